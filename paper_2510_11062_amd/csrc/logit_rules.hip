// The rules of sampling on rows of logits: penalties for tokens that occur in front, biases, masks, temperature; with the row's log-sum and
// its best token on the way (gfx950).
//
// Memory bounds it: a row is read once and written once, 2 V elements, and everything else is lists that are short beside it.  A workgroup
// has 8192 tokens of a row.  Which of them occur in front of the row's token it finds out by itself: it goes through the lists (from the
// cache, where the row's other workgroups read them too) and counts those of its tokens in LDS, while its logits are on their way.  Then
// every logit is in a register, the rules are applied there, and the row's largest and its sum of exponentials come from the same
// registers.  A second kernel joins the parts of a row.
#include "kv_common.hpp"

#include <math.h>

#include <type_traits>

namespace atg {

namespace {

constexpr int kRuleThreads = 256, kRuleSteps = 4, kStepTokens = 8 * kRuleThreads, kRuleChunk = kRuleSteps * kStepTokens;
constexpr uint32_t kInPrompt = 0x80000000u;      // of a token's word in LDS; the rest counts it behind the prompt
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Of a workgroup's tokens: the largest x, where it is first, and sum exp((x - reference(top)) to_out).
struct RulePart {
  float top, sum, to_out;
  int best;
};

// What exponents are taken relative to.  x itself, not its multiple by log2e: a row of the type's lowest values would be infinite so.
__device__ __forceinline__ float reference(float top) { return fabsf(top) < INFINITY ? top : 0.f; }

// A sum relative to `of` as one relative to `to`.  An empty one stays: its reference says nothing.
__device__ __forceinline__ float moved(float sum, float of, float to, float to_log2) {
  return sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((reference(of) - reference(to)) * to_log2);
}

struct RuleArgs {
  at_grpo_sampling_rules r;
  int n_rows, chunks;
  const void* logits;
  int64_t logits_stride;
  void* out;
  int64_t out_stride;
  float* lse;
  int32_t *best, *data_error;
  RulePart* parts;      // workspace: [n_rows][chunks], or null where neither lse nor best is asked for
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

__device__ __forceinline__ float setting(const float* of, int s, float otherwise, bool positive, int* error) {
  if (!of) return otherwise;
  const float x = of[s];
  const bool fine = fabsf(x) < INFINITY && (!positive || x > 0.f);
  if (!fine) *error |= AT_GRPO_DATA_RULE;
  return fine ? x : otherwise;
}

__device__ __forceinline__ RowRules rules_of(const RuleArgs& a, int row, int* error) {
  const at_grpo_sampling_rules& r = a.r;
  RowRules x{};
  x.repetition = 1.f;
  x.to_out = 1.f;
  if (r.allowed) {
    const int m = r.mask_row[row];
    if (m < -1 || m >= r.n_mask) *error |= AT_GRPO_DATA_RULE;
    else if (m >= 0) x.allowed = reinterpret_cast<const uint8_t*>(r.allowed + static_cast<int64_t>(m) * ((r.V + 31) >> 5));
  }
  int s = row, t0 = row, t1 = row + 1;
  if (r.cu_q) {
    s = wave_upper_bound(r.cu_q, r.n_seq + 1, row) - 1;
    if (s < 0 || s >= r.n_seq) return x;      // of no sequence
    t0 = r.cu_q[s];
    t1 = r.cu_q[s + 1];
    if (t0 < 0 || t0 > row || t1 <= row || t1 > a.n_rows) {
      *error |= AT_GRPO_DATA_SEQLENS;
      return x;
    }
  }
  x.repetition = setting(r.repetition, s, 1.f, true, error);
  x.presence = setting(r.presence, s, 0.f, false, error);
  x.frequency = setting(r.frequency, s, 0.f, false, error);
  x.to_out = 1.f / setting(r.temperature, s, 1.f, true, error);
  if (r.tokens) {
    x.own = r.tokens + static_cast<int64_t>(s) * r.max_tokens;
    x.n_own = r.length[s];
    if (x.n_own < 0 || x.n_own > r.max_tokens) {
      *error |= AT_GRPO_DATA_SEQLENS;
      x.n_own = 0;
    }
  }
  if (r.prompt) {
    const int g = wave_upper_bound(r.group_seq, r.n_group + 1, s) - 1;
    if (g >= 0 && g < r.n_group) {
      x.prompt = r.prompt + static_cast<int64_t>(g) * r.max_prompt;
      x.n_prompt = r.prompt_len[g];
      if (x.n_prompt < 0 || x.n_prompt > r.max_prompt || r.group_seq[g] < 0 || r.group_seq[g] > s || r.group_seq[g + 1] <= s || r.group_seq[g + 1] > r.n_seq) {
        *error |= AT_GRPO_DATA_SEQLENS;
        x.n_prompt = 0;
      }
    }
  }
  if (r.ancestors) {
    x.path = r.ancestors[row];
    x.drafted = r.drafted + t0;
    x.n_drafted = min(64, t1 - t0);
  }
  if (r.bias_cu) {
    const int b0 = r.bias_cu[s], b1 = r.bias_cu[s + 1];
    if (b0 < 0 || b1 < b0 || b1 > r.n_bias) {
      *error |= AT_GRPO_DATA_SEQLENS;
    } else {
      x.bias_token = r.bias_token + b0;
      x.bias = r.bias + b0;
      x.n_bias = b1 - b0;
    }
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
  __device__ __forceinline__ void set(int j, bf16_t x) { w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | static_cast<uint32_t>(x.bits) << 16 : x.bits; }
  __device__ __forceinline__ float at(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16); }
};
template <>
struct Eight<float> {
  Words4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = reinterpret_cast<const Words4At4*>(p)[0];
    w[1] = reinterpret_cast<const Words4At4*>(p)[1];
  }
  __device__ __forceinline__ void set(int j, float x) { w[j >> 2][j & 3] = __float_as_uint(x); }
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

// f(token - base, i) for the entries i of a list that name one of a workgroup's tokens.
template <typename F>
__device__ __forceinline__ void go_through(const int32_t* list, int n, int base, int count, int V, bool look, int* error, F f) {
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * kRuleThreads) {
    int token[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) token[k] = i0 + k * kRuleThreads < n ? list[i0 + k * kRuleThreads] : base - 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = token[k] - base;
      if (static_cast<unsigned>(at) < static_cast<unsigned>(count)) f(at, i0 + k * kRuleThreads);
      if (look && i0 + k * kRuleThreads < n && static_cast<unsigned>(token[k]) >= static_cast<unsigned>(V)) *error |= AT_GRPO_DATA_TOKEN_RANGE;
    }
  }
}

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

// LISTS: there are lists to go through; BIAS: biases among them.
template <typename T, typename O, bool LISTS, bool BIAS>
__global__ __launch_bounds__(kRuleThreads) void k_rules(RuleArgs a) {
#pragma clang fp contract(off)
  __shared__ __attribute__((aligned(16))) uint32_t words[LISTS ? kRuleChunk : 4];
  __shared__ float tops[kRuleThreads / 64], sums[kRuleThreads / 64];
  __shared__ int firsts[kRuleThreads / 64];
  const uint32_t block = flat_block();
  const int row = static_cast<int>(block / static_cast<uint32_t>(a.chunks)), chunk = static_cast<int>(block - static_cast<uint32_t>(row) * a.chunks);
  if (row >= a.n_rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.r.V, base = chunk * kRuleChunk, n = min(kRuleChunk, V - base);
  Eight<T> raw[kRuleSteps];
  const T* from = static_cast<const T*>(a.logits) + row * a.logits_stride + base + 8 * tid;
#pragma unroll
  for (int i = 0; i < kRuleSteps; ++i) {
    if ((i + 1) * kStepTokens <= n) {
      raw[i].load(from + i * kStepTokens);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) raw[i].set(j, i * kStepTokens + 8 * tid + j < n ? from[i * kStepTokens + j] : T{});
    }
  }
  int error = 0;
  const RowRules rules = rules_of(a, row, &error);
  const bool look = chunk == 0;
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < kRuleChunk / (4 * kRuleThreads); ++i) *reinterpret_cast<uint4*>(words + 4 * (tid + i * kRuleThreads)) = make_uint4(0, 0, 0, 0);
  };
  auto own_words = [&](int i, uint32_t (&w)[8]) {
    const uint4 lo = *reinterpret_cast<const uint4*>(words + i * kStepTokens + 8 * tid), hi = *reinterpret_cast<const uint4*>(words + i * kStepTokens + 8 * tid + 4);
    w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w, w[4] = hi.x, w[5] = hi.y, w[6] = hi.z, w[7] = hi.w;
  };
  float bias[BIAS ? kRuleSteps : 1][8];
  if constexpr (BIAS) {      // of several entries for a token the last: the largest number
    clear();
    __syncthreads();
    go_through(rules.bias_token, rules.n_bias, base, n, V, look, &error, [&](int at, int i) { atomicMax(words + at, static_cast<uint32_t>(i) + 1); });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRuleSteps; ++i) {
      uint32_t w[8];
      own_words(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) bias[i][j] = w[j] ? rules.bias[w[j] - 1] : 0.f;
    }
    __syncthreads();
  }
  if constexpr (LISTS) {
    clear();
    __syncthreads();
    go_through(rules.prompt, rules.n_prompt, base, n, V, look, &error, [&](int at, int) { atomicOr(words + at, kInPrompt); });
    go_through(rules.own, rules.n_own, base, n, V, look, &error, [&](int at, int) { atomicAdd(words + at, 1u); });
    if (tid < rules.n_drafted && (rules.path >> tid & 1)) {
      const int token = rules.drafted[tid], at = token - base;
      if (static_cast<unsigned>(at) < static_cast<unsigned>(n)) atomicAdd(words + at, 1u);
      if (look && static_cast<unsigned>(token) >= static_cast<unsigned>(V)) error |= AT_GRPO_DATA_TOKEN_RANGE;
    }
    __syncthreads();
  }
  if (look) raise_data_error(a.data_error, error);

  float z[kRuleSteps][8];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kRuleSteps; ++i) {
    const int at = i * kStepTokens + 8 * tid;
    uint32_t bits = 0xff;
    if (rules.allowed) bits = at < n ? rules.allowed[(base + at) >> 3] : 0;      // 8 tokens from a multiple of 8: a byte
    if ((i + 1) * kStepTokens > n) bits &= at + 8 <= n ? 0xffu : at < n ? (1u << (n - at)) - 1 : 0u;      // behind the last token: as if masked
#pragma unroll
    for (int j = 0; j < 8; ++j) z[i][j] = raw[i].at(j);
    if constexpr (LISTS) {
      uint32_t w[8];
      own_words(i, w);
      if ((w[0] | w[1] | w[2] | w[3]) | (w[4] | w[5] | w[6] | w[7])) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t count = w[j] & ~kInPrompt;
          const float x = z[i][j], y = w[j] ? (x > 0.f ? x / rules.repetition : x * rules.repetition) : x;
          z[i][j] = count ? (y - rules.frequency * static_cast<float>(count)) - rules.presence : y;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (BIAS) z[i][j] += bias[i][j];
      z[i][j] = bits >> j & 1 ? z[i][j] : -INFINITY;
      top = fmaxf(top, z[i][j]);
    }
  }
  if (a.out) {
    O* to = static_cast<O*>(a.out) + row * a.out_stride + base + 8 * tid;
#pragma unroll
    for (int i = 0; i < kRuleSteps; ++i) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = z[i][j] * rules.to_out;
      if ((i + 1) * kStepTokens <= n) {
        store_eight(to + i * kStepTokens, y);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i * kStepTokens + 8 * tid + j < n) to[i * kStepTokens + j] = from_f32<O>(y[j]);
      }
    }
  }
  if (!a.parts) return;
  top = wave_max(top);
  if (lane == 0) tops[wave] = top;
  const float to_log2 = rules.to_out * kLog2e, ref = reference(top);
  if (a.lse) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kRuleSteps; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f((z[i][j] - ref) * to_log2);
    sum = wave_sum_all(sum);
    if (lane == 0) sums[wave] = sum;
  }
  __syncthreads();
  const float all = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  int first = 0x7fffffff;
  if (a.best && top == all && all > -INFINITY) {
#pragma unroll
    for (int i = kRuleSteps - 1; i >= 0; --i)
#pragma unroll
      for (int j = 7; j >= 0; --j) first = z[i][j] == all ? base + i * kStepTokens + 8 * tid + j : first;
    first = wave_min(first);
  }
  if (lane == 0) firsts[wave] = first;
  __syncthreads();
  if (tid == 0) {
    RulePart p{all, 0.f, rules.to_out, min(min(firsts[0], firsts[1]), min(firsts[2], firsts[3]))};
    if (a.lse)
      for (int w = 0; w < kRuleThreads / 64; ++w) p.sum += moved(sums[w], tops[w], all, to_log2);
    a.parts[static_cast<int64_t>(row) * a.chunks + chunk] = p;
  }
}

// A wavefront for each row.
__global__ __launch_bounds__(256) void k_rules_join(RuleArgs a) {
  const int64_t row = static_cast<int64_t>(flat_block()) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.n_rows) return;
  const RulePart* const parts = a.parts + row * a.chunks;
  float top = -INFINITY;
  for (int c = lane; c < a.chunks; c += 64) top = fmaxf(top, parts[c].top);
  top = wave_max(top);
  const float to_out = parts[0].to_out;
  float sum = 0.f;
  int first = 0x7fffffff;
  for (int c = lane; c < a.chunks; c += 64) {
    const RulePart p = parts[c];
    sum += moved(p.sum, p.top, top, to_out * kLog2e);
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
  // tokens, and the workgroups of a launch, are counted in 32 bits
  return r->V <= 0x40000000 && ceil_div(r->V, kRuleChunk) * n_rows < 0x7f000000 ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

size_t rule_parts(const at_grpo_sampling_rules* r, int32_t n_rows, void* workspace, RulePart** parts) {
  WsAlloc ws(workspace);
  *parts = ws.take<RulePart>(ceil_div(r->V, kRuleChunk) * n_rows);
  return ws.bytes();
}

template <typename T, typename O>
void launch_rules(const RuleArgs& a, bool lists, bool bias, hipStream_t s) {
  const dim3 grid = grid_of(static_cast<int64_t>(a.chunks) * a.n_rows);
  const auto kernel = bias ? k_rules<T, O, true, true> : lists ? k_rules<T, O, true, false> : k_rules<T, O, false, false>;
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
    if (!itself && in0 < out1 && out0 < in1) return AT_GRPO_EINVAL;
  }
  RuleArgs a{r, n_rows, static_cast<int>(ceil_div(r.V, kRuleChunk)), logits, logits_stride, out, out_stride, lse, best, data_error, nullptr};
  const bool penalties = r.repetition || r.presence || r.frequency;
  if (!penalties) a.r.tokens = a.r.prompt = a.r.drafted = nullptr, a.r.ancestors = nullptr;
  const bool lists = a.r.tokens || a.r.prompt || a.r.ancestors, bias = r.bias_cu && r.n_bias > 0;
  if (!bias) a.r.bias_cu = nullptr;
  if (lse || best) {
    const size_t bytes = rule_parts(rules, n_rows, workspace, &a.parts);
    if (!workspace || (at(workspace) & 255) || workspace_bytes < bytes) return AT_GRPO_EWORKSPACE;
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  ProfScope ps(PROF_RULES, s);
  if (r.dtype == AT_GRPO_F32) launch_rules<float, float>(a, lists, bias, s);
  else if (r.out_dtype == AT_GRPO_F32) launch_rules<bf16_t, float>(a, lists, bias, s);
  else launch_rules<bf16_t, bf16_t>(a, lists, bias, s);
  ATG_LAUNCH_CHECK();
  if (a.parts) {
    hipLaunchKernelGGL(k_rules_join, grid_of(ceil_div(n_rows, 4)), dim3(256), 0, s, a);
    ATG_LAUNCH_CHECK();
  }
  return AT_GRPO_OK;
}
