// The rules of sampling on rows of logits: penalties for tokens that occur in front, biases, masks, temperature; with the row's log-sum and
// its best token on the way (gfx950).
//
// Memory bounds it: a row is read once and written once, 2 V elements, and everything else is lists that are short beside it.  A workgroup
// has chunks of 8192 tokens of a row.  Which of these occur in front of the row's token it finds out by itself: it goes through the lists (whose
// first entries its threads keep) and counts those of its tokens in LDS, while the chunk's logits and mask bits are on their way.  Then eight
// logits at a time are in a lane's registers; the rules are applied there, and the row's largest and its sum of exponentials come from the
// same registers.  A second kernel joins the parts of a row.
//
// Rows of 151936 in bf16: 1339 under masks alone, read and not written, 80 to 86 us (4.8 to 5.1 TB/s, a large copy 4.9); 682 rewritten without lists 87 us
// (5.0 TB/s), with prompts, own tokens and drafted paths 103, with biases too 110 to 114: the lists' atomics, barriers and branches.
#include "kv_common.hpp"

#include <math.h>

#include <type_traits>

namespace atg {

namespace {

constexpr int kRuleThreads = 256, kRuleSteps = 4, kStepTokens = 8 * kRuleThreads, kRuleChunk = kRuleSteps * kStepTokens, kMostChunks = 8;
// A token's word in LDS: whether the prompt has it, the number of its bias among the sequence's, from 1 on, or 0, and how often it occurs behind
// the prompt.  Where lists may be longer than that counts the biases go through LDS first, and the count has all other bits.
constexpr uint32_t kInPrompt = 0x80000000u;
constexpr int kBiasShift = 16, kMostBiases = 0x7fff, kMostTokens = 0xffff, kNearBiases = 512;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Up to where the largest's multiple is subtracted from the others': rounded, it is off by half a unit of its last place, which is in every exponent
// then.  Here that is at most 2^-5, and never more than half a unit of the log-sum; at 2^32 it is past 127, where sums are infinite or 0.
constexpr float kMostScaled = 0x1p20f;

// Of a workgroup's tokens: the largest x, where it is first, and sum exp((x - reference(top)) to_out).
struct RulePart {
  float top, sum, to_out;
  int best;
};

// What exponents are taken relative to.  x itself, not its multiple by log2e: a row of the type's lowest values would be infinite so.
__device__ __forceinline__ float reference(float top) { return fabsf(top) < INFINITY ? top : 0.f; }

// The temperature's reciprocal for exponents to the base 2: finite, since differences of 0 are multiplied by it.
__device__ __forceinline__ float exponents(float to_out) { return fminf(to_out * kLog2e, 0x1.fffffep127f); }

// A sum relative to `of` as one relative to `to`.  An empty one stays: its reference says nothing.
__device__ __forceinline__ float moved(float sum, float of, float to, float to_log2) {
  return sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((reference(of) - reference(to)) * to_log2);
}

struct RuleArgs {
  at_grpo_sampling_rules r;
  int n_rows, chunks, splits, per;      // workgroups of a row, chunks that each of them goes through
  const void* logits;
  int64_t logits_stride;
  void* out;
  int64_t out_stride;
  float* lse;
  int32_t *best, *data_error;
  RulePart* parts;      // workspace: [n_rows][splits], or null where neither lse nor best is asked for
};

// What belongs to a row.
struct RowRules {
  const int32_t *own, *prompt, *drafted, *bias_token;
  const float* bias;
  int n_own, n_prompt, n_drafted, n_bias;
  uint64_t path;
  float repetition, presence, frequency, to_out;      // to_out: 1 / temperature
  const uint8_t* allowed;                             // bits, or null
};

__device__ __forceinline__ float checked(float x, float otherwise, bool positive, int* error) {
  const bool fine = fabsf(x) < INFINITY && (!positive || (x > 0.f && 1.f / x < INFINITY));
  if (!fine) *error |= AT_GRPO_DATA_RULE;
  return fine ? x : otherwise;
}

__device__ __forceinline__ RowRules rules_of(const RuleArgs& a, int row, int* error) {
  const at_grpo_sampling_rules& r = a.r;
  RowRules x{};
  x.repetition = 1.f;
  x.to_out = 1.f;
  // Everything that can be asked for at once is, and looked at behind that: one after the other these loads are what a short call takes.
  const int m = r.allowed ? r.mask_row[row] : -1;
  if (r.ancestors) x.path = r.ancestors[row];
  int s = row, t0 = row, t1 = row + 1;
  bool of_one = true;
  if (r.cu_q) {
    s = wave_upper_bound(r.cu_q, r.n_seq + 1, row) - 1;
    of_one = s >= 0 && s < r.n_seq;
    s = of_one ? s : 0;
    if (of_one) {
      t0 = r.cu_q[s];
      t1 = r.cu_q[s + 1];
    }
  }
  float repetition = 1.f, presence = 0.f, frequency = 0.f, temperature = 1.f;
  int n_own = 0, b0 = 0, b1 = 0, g = -1, n_prompt = 0, s0 = 0, s1 = 0;
  if (of_one) {
    if (r.repetition) repetition = r.repetition[s];
    if (r.presence) presence = r.presence[s];
    if (r.frequency) frequency = r.frequency[s];
    if (r.temperature) temperature = r.temperature[s];
    if (r.tokens) n_own = r.length[s];
    if (r.bias_cu) {
      b0 = r.bias_cu[s];
      b1 = r.bias_cu[s + 1];
    }
    if (r.prompt) {
      g = wave_upper_bound(r.group_seq, r.n_group + 1, s) - 1;
      if (g >= 0 && g < r.n_group) {
        n_prompt = r.prompt_len[g];
        s0 = r.group_seq[g];
        s1 = r.group_seq[g + 1];
      }
    }
  }
  if (m < -1 || m >= r.n_mask) {
    if (r.allowed) *error |= AT_GRPO_DATA_RULE;
  } else if (m >= 0) {
    x.allowed = reinterpret_cast<const uint8_t*>(r.allowed + static_cast<int64_t>(m) * ((r.V + 31) >> 5));
  }
  if (!of_one) return x;
  if (t0 < 0 || t0 > row || t1 <= row || t1 > a.n_rows) {      // of no sequence either
    *error |= AT_GRPO_DATA_SEQLENS;
    return x;
  }
  x.repetition = checked(repetition, 1.f, true, error);
  x.presence = checked(presence, 0.f, false, error);
  x.frequency = checked(frequency, 0.f, false, error);
  x.to_out = 1.f / checked(temperature, 1.f, true, error);
  if (r.tokens) {
    x.own = r.tokens + static_cast<int64_t>(s) * r.max_tokens;
    x.n_own = n_own;
    if (n_own < 0 || n_own > r.max_tokens) {
      *error |= AT_GRPO_DATA_SEQLENS;
      x.n_own = 0;
    }
  }
  if (g >= 0 && g < r.n_group) {
    x.prompt = r.prompt + static_cast<int64_t>(g) * r.max_prompt;
    x.n_prompt = n_prompt;
    if (n_prompt < 0 || n_prompt > r.max_prompt || s0 < 0 || s0 > s || s1 <= s || s1 > r.n_seq) {
      *error |= AT_GRPO_DATA_SEQLENS;
      x.n_prompt = 0;
    }
  }
  if (r.ancestors) {
    x.drafted = r.drafted + t0;
    x.n_drafted = min(64, t1 - t0);
  }
  if (b0 < 0 || b1 < b0 || b1 > r.n_bias) {
    *error |= AT_GRPO_DATA_SEQLENS;
  } else if (r.bias_cu) {
    x.bias_token = r.bias_token + b0;
    x.bias = r.bias + b0;
    x.n_bias = b1 - b0;
  }
  return x;
}

// Eight logits of a lane; rows begin at any element.
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef Words4 Words4At2 __attribute__((aligned(2)));
typedef Words4 Words4At4 __attribute__((aligned(4)));
template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
  Words4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const Words4At2*>(p); }
  __device__ __forceinline__ float at(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16); }
};
template <>
struct Eight<float> {
  Words4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = reinterpret_cast<const Words4At4*>(p)[0];
    w[1] = reinterpret_cast<const Words4At4*>(p)[1];
  }
  __device__ __forceinline__ float at(int j) const { return __uint_as_float(w[j >> 2][j & 3]); }
};
__device__ __forceinline__ void store_eight(bf16_t* p, const float* y) {
  *reinterpret_cast<Words4At2*>(p) = Words4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
}
__device__ __forceinline__ void store_eight(float* p, const float* y) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    reinterpret_cast<Words4At4*>(p)[i] = Words4{__float_as_uint(y[4 * i]), __float_as_uint(y[4 * i + 1]), __float_as_uint(y[4 * i + 2]), __float_as_uint(y[4 * i + 3])};
}

// The entries of a list, the first K of each thread in registers.
template <int K>
struct List {
  const int32_t* from;
  int n, held[K];
  __device__ __forceinline__ List(const int32_t* list, int count) : from(list), n(count) {
#pragma unroll
    for (int k = 0; k < K; ++k) held[k] = static_cast<int>(threadIdx.x) + k * kRuleThreads < n ? list[threadIdx.x + k * kRuleThreads] : -1;
  }
  // f(token - base, i) for the entries i that name one of `count` tokens from base on.
  template <typename F>
  __device__ __forceinline__ void each(int base, int count, int V, bool look, int* error, F f) const {
    auto one = [&](int token, int i) {
      if (static_cast<unsigned>(token - base) < static_cast<unsigned>(count)) f(token - base, i);
      if (look && i < n && static_cast<unsigned>(token) >= static_cast<unsigned>(V)) *error |= AT_GRPO_DATA_TOKEN_RANGE;
    };
#pragma unroll
    for (int k = 0; k < K; ++k) one(held[k], threadIdx.x + k * kRuleThreads);
    for (int i0 = threadIdx.x + K * kRuleThreads; i0 < n; i0 += 4 * kRuleThreads) {
      int token[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) token[k] = i0 + k * kRuleThreads < n ? from[i0 + k * kRuleThreads] : -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) one(token[k], i0 + k * kRuleThreads);
    }
  }
};

// The largest of three, or NaN where one of them is NaN of either kind: v_maximum3_f32.  v_max3_f32 passes NaN over, and what it has seen in front of
// a signalling one with it.
__device__ __forceinline__ float maximum3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}
__device__ __forceinline__ float wave_sum_all(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o, 64));
  return x;
}

// x / d, rounded once, for x of any kind: the product with the reciprocal `one_over` (itself rounded once), corrected by what is left over.
__device__ __forceinline__ float divided(float x, float d, float one_over) {
  const float q = x * one_over;
  return __builtin_amdgcn_div_fixupf(__builtin_fmaf(__builtin_fmaf(-q, d, x), one_over, q), d, x);
}

// What lists there are to go through: none, those of tokens, of biases too, of any length.
enum Lists { NONE, TOKENS, BIASES, LONG };

template <typename T, typename O, int LISTS>
__global__ __launch_bounds__(kRuleThreads, LISTS == LONG ? 2 : 4) void k_rules(RuleArgs a) {
#pragma clang fp contract(off)
  __shared__ __attribute__((aligned(16))) uint32_t words[LISTS != NONE ? kRuleChunk : 4];
  __shared__ float bias_near[LISTS == BIASES ? kNearBiases : 1];      // values of the first biases
  __shared__ float tops[kRuleThreads / 64], sums[kRuleThreads / 64];
  __shared__ int firsts[kRuleThreads / 64];
  const uint32_t block = flat_block();
  const int row = static_cast<int>(block / static_cast<uint32_t>(a.splits)), split = static_cast<int>(block - static_cast<uint32_t>(row) * a.splits);
  if (row >= a.n_rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.r.V, chunk0 = split * a.per, chunk1 = min(a.chunks, chunk0 + a.per);
  const T* const logits = static_cast<const T*>(a.logits) + row * a.logits_stride;
  // The whole steps of a chunk, 2048 tokens each, are asked for ahead; what is left of a row behind them is read token by token.
  Eight<T> raw[kRuleSteps];
  auto whole_steps = [&](int chunk) { return chunk < chunk1 ? min(kRuleSteps, (V - chunk * kRuleChunk) / kStepTokens) : 0; };
  int bits[kRuleSteps];      // of the row's mask: 8 tokens from a multiple of 8 are a byte
  auto load = [&](int chunk, int i) { raw[i].load(logits + chunk * kRuleChunk + i * kStepTokens + 8 * tid); };
  const int whole0 = whole_steps(chunk0);
#pragma unroll
  for (int i = 0; i < kRuleSteps; ++i)
    if (i < whole0) load(chunk0, i);
  int error = 0;
  const RowRules rules = rules_of(a, row, &error);
  const List<LISTS != NONE ? 4 : 1> prompt(rules.prompt, LISTS != NONE ? rules.n_prompt : 0), own(rules.own, LISTS != NONE ? rules.n_own : 0);
  const List<LISTS >= BIASES ? 2 : 1> biased(rules.bias_token, LISTS >= BIASES ? rules.n_bias : 0);
  if constexpr (LISTS == BIASES)
    for (int i = tid; i < min(rules.n_bias, kNearBiases); i += kRuleThreads) bias_near[i] = rules.bias[i];
  const bool on_path = LISTS != NONE && tid < rules.n_drafted && (rules.path >> (tid & 63) & 1);
  const int drafted = on_path ? rules.drafted[tid] : -1;
  // A thread's own words of a step, which it leaves as 0 for the next chunk.  Those of its first four tokens lie in one half of the step's, those of
  // the others in the other, so that neighbours' lie side by side and no bank is met twice.
  auto take_words = [&](int of, uint32_t (&w)[8]) {      // of: the first one's place in the chunk
    uint4* const at = reinterpret_cast<uint4*>(words + (of - 4 * tid));
    const uint4 lo = at[0], hi = at[kStepTokens / 8];
    at[0] = at[kStepTokens / 8] = make_uint4(0, 0, 0, 0);
    w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w, w[4] = hi.x, w[5] = hi.y, w[6] = hi.z, w[7] = hi.w;
  };
  auto word_of = [&](int at) {
    const int in = at & (kStepTokens - 1);
    return words + (at - in) + (in >> 2 & 1) * (kStepTokens / 2) + (in >> 3 << 2) + (in & 3);
  };
  if constexpr (LISTS != NONE) {
#pragma unroll
    for (int i = 0; i < kRuleSteps; ++i) {
      uint32_t unused[8];
      take_words(i * kStepTokens + 8 * tid, unused);
    }
  }
  auto load_bits = [&](int chunk, int i) { bits[i] = rules.allowed ? rules.allowed[(chunk * kRuleChunk + i * kStepTokens) / 8 + tid] : 0xff; };
#pragma unroll
  for (int i = 0; i < kRuleSteps; ++i)
    if (i < whole0) load_bits(chunk0, i);
  const float one_over = 1.f / rules.repetition, to_log2 = exponents(rules.to_out);
  float top = -INFINITY, scaled = 0.f, sum = 0.f;      // of the wavefront's tokens, its multiple as exponents have it, and of this thread's
  int first = 0x7fffffff;
  // The rules on eight tokens from `token` on, of which the row has `have`; `at` is their place in the chunk.
  auto step = [&](float (&z)[8], const float* bias, int bits, int at, int token, int have, auto is_whole) {
    constexpr bool whole = decltype(is_whole)::value;
    if constexpr (LISTS != NONE) {
      uint32_t w[8];
      take_words(at, w);
      if (__any((w[0] | w[1] | w[2] | w[3]) | (w[4] | w[5] | w[6] | w[7]))) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (w[j]) {
            float x = z[j];
            const uint32_t count = LISTS == BIASES ? w[j] & kMostTokens : w[j] & ~kInPrompt;
            if (LISTS != BIASES || count || w[j] >= kInPrompt) x = x > 0.f ? divided(x, rules.repetition, one_over) : x * rules.repetition;
            if (count) x = (x - rules.frequency * static_cast<float>(count)) - rules.presence;
            if constexpr (LISTS == BIASES) {
              const int entry = w[j] >> kBiasShift & kMostBiases;
              if (entry) x += entry <= kNearBiases ? bias_near[entry - 1] : rules.bias[entry - 1];
            }
            z[j] = x;
          }
      }
    }
    if constexpr (LISTS == LONG) {
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += bias[j];
    }
    if (rules.allowed || !whole) {
      if (!whole) bits &= have >= 8 ? 0xff : have > 0 ? (1 << have) - 1 : 0;           // behind the last token: as if masked
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t on = static_cast<uint32_t>(static_cast<int>(static_cast<uint32_t>(bits) << (31 - j)) >> 31);
        z[j] = __uint_as_float((__float_as_uint(z[j]) & on) | (0xff800000u & ~on));
      }
    }
    if (a.out) {
      O* const to = static_cast<O*>(a.out) + row * a.out_stride + token;
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = z[j] * rules.to_out;
      if constexpr (whole) {
        store_eight(to, y);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < have) to[j] = from_f32<O>(y[j]);
      }
    }
    if (!a.parts) return;
    // Four instructions; fmaxf, which has to quiet signalling NaN first, takes fifteen.  A NaN comes out as one, and is looked at as a larger one is.
    if (__any(!(maximum3(maximum3(maximum3(z[0], z[1], z[2]), z[3], z[4]), z[5], maximum3(z[6], z[7], z[7])) <= top))) {      // seldom, once a wavefront has seen some of its tokens
      float high = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) high = z[j] > high ? z[j] : high;      // NaN of either kind is passed over; of several fmaxf the compiler makes v_max3_f32
      const float now = wave_max(high);
      if (now > top) {
        sum = moved(sum, top, now, to_log2);
        top = now;
        scaled = reference(top) * to_log2;
        first = 0x7fffffff;
#pragma unroll
        for (int j = 7; j >= 0; --j) first = z[j] == now ? token + j : first;
      }
    }
    if (a.lse) {
      if (fabsf(scaled) < kMostScaled) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], to_log2, -scaled));
      } else {      // differences first: 0 for the largest itself, also where multiples are infinite
        const float ref = reference(top);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f((z[j] - ref) * to_log2);
      }
    }
  };
  for (int chunk = chunk0; chunk < chunk1; ++chunk) {
    const int base = chunk * kRuleChunk, n = min(kRuleChunk, V - base);
    const bool look = chunk == 0;
    float bias[LISTS == LONG ? kRuleSteps : 1][8];
    if constexpr (LISTS != NONE) __syncthreads();
    if constexpr (LISTS == LONG) {      // of several entries for a token the last: the largest number
      biased.each(base, n, V, look, &error, [&](int at, int i) { atomicMax(word_of(at), static_cast<uint32_t>(i) + 1); });
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRuleSteps; ++i) {
        uint32_t w[8];
        take_words(i * kStepTokens + 8 * tid, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[i][j] = w[j] ? rules.bias[w[j] - 1] : 0.f;
      }
      __syncthreads();
    }
    if constexpr (LISTS == BIASES) {
      biased.each(base, n, V, look, &error, [&](int at, int i) { atomicMax(word_of(at), static_cast<uint32_t>(i + 1) << kBiasShift); });
      __syncthreads();
    }
    if constexpr (LISTS != NONE) {
      prompt.each(base, n, V, look, &error, [&](int at, int) { atomicOr(word_of(at), kInPrompt); });
      own.each(base, n, V, look, &error, [&](int at, int) { atomicAdd(word_of(at), 1u); });
      if (static_cast<unsigned>(drafted - base) < static_cast<unsigned>(n)) atomicAdd(word_of(drafted - base), 1u);
      if (look && on_path && static_cast<unsigned>(drafted) >= static_cast<unsigned>(V)) error |= AT_GRPO_DATA_TOKEN_RANGE;
      __syncthreads();
    }

    const int whole = whole_steps(chunk), whole_next = whole_steps(chunk + 1);
#pragma unroll
    for (int i = 0; i < kRuleSteps; ++i)
      if (i < whole) {
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = raw[i].at(j);
        const int allowed = bits[i];
        if (i < whole_next) {
          load(chunk + 1, i);
          load_bits(chunk + 1, i);
        }
        const int at = i * kStepTokens + 8 * tid;
        step(z, bias[LISTS == LONG ? i : 0], allowed, at, base + at, 8, std::true_type{});
      }
    if (whole < kRuleSteps && whole * kStepTokens < n) {      // the row's last tokens
      const int at = whole * kStepTokens + 8 * tid, token = base + at, have = V - token;
      float z[8], b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[j] = j < have ? to_f32(logits[token + j]) : 0.f;
        if constexpr (LISTS == LONG) b[j] = whole == 0 ? bias[0][j] : whole == 1 ? bias[1][j] : whole == 2 ? bias[2][j] : bias[3][j];
      }
      step(z, b, rules.allowed && have > 0 ? rules.allowed[token >> 3] : 0xff, at, token, have, std::false_type{});
    }
  }
  if (chunk0 == 0) raise_data_error(a.data_error, error);
  if (!a.parts) return;
  sum = wave_sum_all(sum);
  first = wave_min(first);
  if (lane == 0) {
    tops[wave] = top;
    sums[wave] = sum;
    firsts[wave] = first;
  }
  __syncthreads();
  if (tid == 0) {
    RulePart p{fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), 0.f, rules.to_out, 0x7fffffff};
    for (int w = 0; w < kRuleThreads / 64; ++w) {
      p.sum += moved(sums[w], tops[w], p.top, to_log2);
      if (tops[w] == p.top) p.best = min(p.best, firsts[w]);
    }
    a.parts[static_cast<int64_t>(row) * a.splits + split] = p;
  }
}

// A wavefront for each row.
__global__ __launch_bounds__(256) void k_rules_join(RuleArgs a) {
  const int64_t row = static_cast<int64_t>(flat_block()) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.n_rows) return;
  const RulePart* const parts = a.parts + row * a.splits;
  float top = -INFINITY;
  for (int c = lane; c < a.splits; c += 64) top = fmaxf(top, parts[c].top);
  top = wave_max(top);
  const float to_out = parts[0].to_out;
  float sum = 0.f;
  int first = 0x7fffffff;
  for (int c = lane; c < a.splits; c += 64) {
    const RulePart p = parts[c];
    sum += moved(p.sum, p.top, top, exponents(to_out));
    if (p.top == top) first = min(first, p.best);
  }
  sum = wave_sum_all(sum);
  first = wave_min(first);
  if (lane) return;
  if (a.lse) a.lse[row] = reference(top) * to_out + __builtin_amdgcn_logf(sum) * kLn2;      // nothing left: log2 0
  if (a.best) a.best[row] = top == -INFINITY ? -1 : first;
}

int check_rules(const at_grpo_sampling_rules* r, int32_t n_rows) {
  if (!r || n_rows < 0 || r->V <= 0 || r->n_seq < 0 || r->n_group < 0 || r->max_tokens < 0 || r->max_prompt < 0 || r->n_bias < 0 || r->n_mask < 0)
    return AT_GRPO_EINVAL;
  if (r->dtype != AT_GRPO_F32 && r->dtype != AT_GRPO_BF16) return AT_GRPO_EUNSUPPORTED;
  if (r->out_dtype != r->dtype && r->out_dtype != AT_GRPO_F32) return AT_GRPO_EUNSUPPORTED;
  // tokens, places in lists, sequences, groups and the workgroups of a launch are counted in 32 bits; places go past a list's end by less than 2^16
  const int32_t most = 0x7fff0000;
  if (r->max_tokens > most || r->max_prompt > most || r->n_bias > most || r->n_seq > most || r->n_group > most) return AT_GRPO_EUNSUPPORTED;
  return r->V <= 0x40000000 && ceil_div(r->V, kRuleChunk) * n_rows < 0x7f000000 ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

size_t rule_parts(const at_grpo_sampling_rules* r, int32_t n_rows, void* workspace, RulePart** parts) {
  WsAlloc ws(workspace);
  *parts = ws.take<RulePart>(ceil_div(r->V, kRuleChunk) * n_rows);
  return ws.bytes();
}

template <typename T, typename O>
void launch_rules(const RuleArgs& a, int lists, hipStream_t s) {
  const dim3 grid = grid_of(static_cast<int64_t>(a.splits) * a.n_rows);
  const auto kernel = lists == LONG ? k_rules<T, O, LONG> : lists == BIASES ? k_rules<T, O, BIASES> : lists == TOKENS ? k_rules<T, O, TOKENS> : k_rules<T, O, NONE>;
  hipLaunchKernelGGL(kernel, grid, dim3(kRuleThreads), 0, s, a);
}

}  // namespace
}  // namespace atg

using namespace atg;

extern "C" size_t at_grpo_logit_rules_workspace_bytes(const at_grpo_sampling_rules* rules, int32_t n_rows) {
  RulePart* parts;
  return check_rules(rules, n_rows) == AT_GRPO_OK ? rule_parts(rules, n_rows, nullptr, &parts) + 256 : 0;
}

extern "C" int at_grpo_logit_rules(const at_grpo_sampling_rules* rules, int32_t n_rows, const void* logits, int64_t logits_stride, void* out,
                                   int64_t out_stride, float* lse, int32_t* best, int32_t* data_error, void* workspace, size_t workspace_bytes,
                                   void* hip_stream) {
  ATG_TRY(check_rules(rules, n_rows));
  const at_grpo_sampling_rules& r = *rules;
  if (!r.cu_q && n_rows != r.n_seq) return AT_GRPO_EINVAL;
  if (n_rows == 0) return AT_GRPO_OK;
  if (!logits || (!out && !lse && !best) || (n_rows > 1 && logits_stride < r.V) || (out && n_rows > 1 && out_stride < r.V)) return AT_GRPO_EINVAL;
  if ((r.tokens && !r.length) || (r.prompt && (!r.group_seq || !r.prompt_len)) || (r.ancestors && !r.drafted)) return AT_GRPO_EINVAL;
  if ((r.bias_cu && r.n_bias > 0 && (!r.bias_token || !r.bias)) || (r.allowed && !r.mask_row)) return AT_GRPO_EINVAL;
  const int64_t e = elem_size(r.dtype), eo = elem_size(r.out_dtype);
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (at(logits) % e || at(out) % eo) return AT_GRPO_EINVAL;
  if (out) {      // the logits themselves, or apart from them
    const uintptr_t in0 = at(logits), in1 = in0 + ((n_rows - 1) * logits_stride + r.V) * e, out0 = at(out), out1 = out0 + ((n_rows - 1) * out_stride + r.V) * eo;
    const bool itself = out == logits && r.out_dtype == r.dtype && (n_rows == 1 || out_stride == logits_stride);
    bool beside = false;      // in rows of one buffer
    if (n_rows > 1 && logits_stride * e == out_stride * eo) {
      const int64_t step = logits_stride * e, apart = ((static_cast<int64_t>(out0) - static_cast<int64_t>(in0)) % step + step) % step;
      beside = apart >= r.V * e && apart + r.V * eo <= step;
    }
    if (!itself && !beside && in0 < out1 && out0 < in1) return AT_GRPO_EINVAL;
  }
  const int chunks = static_cast<int>(ceil_div(r.V, kRuleChunk));
  RuleArgs a{r, n_rows, chunks, chunks, 1, logits, logits_stride, out, out_stride, lse, best, data_error, nullptr};
  const bool penalties = r.repetition || r.presence || r.frequency;
  if (!penalties) a.r.tokens = a.r.prompt = a.r.drafted = nullptr, a.r.ancestors = nullptr;
  const bool tokens = a.r.tokens || a.r.prompt || a.r.ancestors, bias = r.bias_cu && r.n_bias > 0;
  if (!bias) a.r.bias_cu = nullptr;
  const int64_t most = (a.r.tokens ? r.max_tokens : 0) + (a.r.ancestors ? int64_t{64} : 0);
  const int lists = !bias ? tokens ? TOKENS : NONE : r.n_bias <= kMostBiases && most <= kMostTokens ? BIASES : LONG;
  // As many chunks a workgroup as leave two rounds of four workgroups a compute unit: what belongs to a row is looked up once for them and a chunk's
  // logits come beside the work on the one in front.  682 rows of 151936 with all rules: a chunk each 146 us, three 124, five 119, seven 114,
  // ten 160 (not two rounds); 1339 rows under masks alone: 103, 88, 89, 86.
  const int64_t share = ceil_div(static_cast<int64_t>(chunks) * n_rows, int64_t{8} * device_cu_count());
  a.per = static_cast<int>(share < kMostChunks ? share : kMostChunks);
  a.splits = static_cast<int>(ceil_div(chunks, a.per));
  a.per = static_cast<int>(ceil_div(chunks, a.splits));
  if (lse || best) {
    const size_t bytes = rule_parts(rules, n_rows, workspace, &a.parts);
    if (!workspace || (at(workspace) & 255) || workspace_bytes < bytes) return AT_GRPO_EWORKSPACE;
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  ProfScope ps(PROF_RULES, s);
  if (r.dtype == AT_GRPO_F32) launch_rules<float, float>(a, lists, s);
  else if (r.out_dtype == AT_GRPO_F32) launch_rules<bf16_t, float>(a, lists, s);
  else launch_rules<bf16_t, bf16_t>(a, lists, s);
  ATG_LAUNCH_CHECK();
  if (a.parts) {
    hipLaunchKernelGGL(k_rules_join, grid_of(ceil_div(n_rows, 4)), dim3(256), 0, s, a);
    ATG_LAUNCH_CHECK();
  }
  return AT_GRPO_OK;
}
