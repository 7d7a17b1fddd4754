// Page tables, slots and positions of a step's new tokens, from the sequences' lengths (gfx950).
//
// A sequence holds ceil(tokens / page) pages, so a step takes or gives the difference of two such counts, and where in the ring a
// sequence's pages come from is a sum over the sequences in front of it, as is the place of its tokens among the new ones.  There is next
// to nothing to move (12 bytes a sequence read, 16 with `keep`, and 8 written; a token's parent read, 4, and up to 24 written): what a call takes is launches and loads
// one behind the other.
//   k_plan             up to 2048 sequences, in one launch: every workgroup adds up all sequences by itself, keeps the sums in LDS, and writes its
//                      share of the tokens, the sequences and the pages moved; a new page's id it reads where it stands in the ring.  Where an output is its
//                      input itself it may only be written once every workgroup has read that: by a single workgroup then, while the tokens are few
// Otherwise two:
//   k_plan_sequences   a workgroup for 1024 sequences.  Each adds up all sequences, since every one has to know whether the pool suffices, and
//                      those in front of its own; then pages are moved, a thread for each
//   k_plan_tokens      a thread for each new token and for each sequence's length, which the first still reads
// Four candidates 4.3 us (two launches 7.5 and 2.2), 1339 with 11000 drafted tokens 10.3 (10.5 and 6.2), 512 prompts of 374000 tokens 14.6 (11.5 and 5.6,
// and the gap between them).
#include "kv_common.hpp"

namespace atg {

namespace {

constexpr int kPlanBlock = 1024;
constexpr int kMostDrafted = 64;      // tokens of a tree: bits of a word

struct PlanArgs {
  int shift, n_pages, n_seq, max_pages, n_group, n_tok;
  int32_t *pages, *ring;
  const int32_t *group_seq, *prefix_len, *length, *keep, *add, *parent, *state;
  int32_t *length_out, *state_out, *cu_q, *seq, *position;
  int64_t* slot;
  uint64_t* ancestors;
  int32_t* data_error;
  // Workspace, so that the second kernel reads nothing that it writes where an output is its input itself.
  int32_t* verdict;             // whether there are prefixes, the state behind the step
  int32_t *kept, *behind;       // [n_seq]: tokens kept, length behind the step
};

// What the step is for a sequence.
struct Step {
  int keep, add, used, will;
  bool wrong;
};
__device__ __forceinline__ Step step_of(const PlanArgs& a, int s) {
  const int held = a.length[s], keep = a.keep ? a.keep[s] : held, add = a.add[s], most = a.max_pages << a.shift, last = (1 << a.shift) - 1;
  const bool wrong = held < 0 || held > most || keep < 0 || keep > held || add < 0 || add > most - keep || (a.parent && add > kMostDrafted);
  return wrong ? Step{0, 0, 0, 0, true} : Step{keep, add, (held + last) >> a.shift, (keep + add + last) >> a.shift, false};
}

__device__ __forceinline__ int64_t wave_sum64(int64_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// The last of n rising entries that is <= x, the first of which is; between 0 and n - 1 whatever they hold.
__device__ __forceinline__ int last_below(const int32_t* a, int n, int x) {
  int s = 0;
  for (int k = n; k > 1;) {
    const int half = k >> 1;
    if (a[s + half] <= x) s += half;
    k -= half;
  }
  return s;
}

// Sums over all sequences, and over those in front of a workgroup's.
struct Sums {
  int taken, given, taken_before, given_before;
  int64_t added, added_before;
  int wrong;
};

// The state of a ring that can be, and a step that it can take: 0, or the bits of what is wrong.
__device__ __forceinline__ int verdict_of(const PlanArgs& a, int first, int count, const Sums& x) {
  if (x.wrong || x.added > a.n_tok) return AT_GRPO_DATA_SEQLENS;
  if (first < 0 || first >= a.n_pages || count < 0 || count > a.n_pages || x.taken > count || x.given > a.n_pages - count) return AT_GRPO_DATA_POOL;
  return 0;
}

__device__ __forceinline__ int ring_at(const PlanArgs& a, int first, int i) {      // first, i < n_pages <= 2^31
  const uint32_t at = static_cast<uint32_t>(first) + static_cast<uint32_t>(i);
  return static_cast<int>(at >= static_cast<uint32_t>(a.n_pages) ? at - a.n_pages : at);
}

__global__ __launch_bounds__(kPlanBlock) void k_plan_sequences(PlanArgs a) {
  __shared__ Sums waves[kPlanBlock / 64];
  __shared__ int scan_lds[kPlanBlock / 64], used[kPlanBlock], will[kPlanBlock], take[kPlanBlock], give[kPlanBlock];
  __shared__ int group_wrong;
  const int tid = threadIdx.x, wave = tid >> 6, begin = blockIdx.x * kPlanBlock;
  const int first = a.state[0], count = a.state[1];
  if (tid == 0) group_wrong = 0;
  Sums x{};
  for (int s = tid; s < a.n_seq; s += kPlanBlock) {
    const Step y = step_of(a, s);
    const int taken = max(0, y.will - y.used), given = max(0, y.used - y.will);
    x.wrong |= y.wrong;
    x.taken += taken;
    x.given += given;
    x.added += y.add;
    if (s < begin) {
      x.taken_before += taken;
      x.given_before += given;
      x.added_before += y.add;
    }
  }
  x.taken = wave_total(x.taken);
  x.given = wave_total(x.given);
  x.taken_before = wave_total(x.taken_before);
  x.given_before = wave_total(x.given_before);
  x.added = wave_sum64(x.added);
  x.added_before = wave_sum64(x.added_before);
  x.wrong = __any(x.wrong);
  if ((tid & 63) == 0) waves[wave] = x;
  __syncthreads();
  x = Sums{};
  for (int w = 0; w < kPlanBlock / 64; ++w) {
    x.taken += waves[w].taken;
    x.given += waves[w].given;
    x.taken_before += waves[w].taken_before;
    x.given_before += waves[w].given_before;
    x.added += waves[w].added;
    x.added_before += waves[w].added_before;
    x.wrong |= waves[w].wrong;
  }
  const int refused = verdict_of(a, first, count, x);
  if (blockIdx.x == 0) {
    int error = refused, falls = 0;
    for (int g = tid; g < a.n_group; g += kPlanBlock) {
      falls |= a.group_seq[g] < 0 || a.group_seq[g + 1] < a.group_seq[g] || a.group_seq[g + 1] > a.n_seq;
      if (a.prefix_len[g] < 0 || a.prefix_len[g] > 1 << 30) error |= AT_GRPO_DATA_SEQLENS;
    }
    if (falls) atomicOr(&group_wrong, 1);
    __syncthreads();
    if (falls) error |= AT_GRPO_DATA_SEQLENS;
    raise_data_error(a.data_error, error);
    if (tid == 0) {
      a.verdict[0] = group_wrong == 0;
      a.verdict[1] = refused ? first : ring_at(a, first, x.taken);
      a.verdict[2] = refused ? count : count - x.taken + x.given;
      a.cu_q[a.n_seq] = refused ? 0 : static_cast<int>(x.added);
    }
  }
  const int s = begin + tid;
  if (refused) {
    if (s < a.n_seq) {
      a.cu_q[s] = 0;
      a.behind[s] = a.length[s];
    }
    return;
  }
  const Step y = s < a.n_seq ? step_of(a, s) : Step{};
  if (s < a.n_seq) {
    a.kept[s] = y.keep;
    a.behind[s] = y.keep + y.add;
  }
  int moved, unused;
  const int new_before = block_exclusive_scan<kPlanBlock>(y.add, scan_lds, &unused);
  if (s < a.n_seq) a.cu_q[s] = static_cast<int>(x.added_before) + new_before;
  used[tid] = y.used;
  will[tid] = y.will;
  take[tid] = block_exclusive_scan<kPlanBlock>(max(0, y.will - y.used), scan_lds, &moved);
  __syncthreads();
  for (int m = tid; m < moved; m += kPlanBlock) {
    const int i = last_below(take, kPlanBlock, m);
    a.pages[static_cast<int64_t>(begin + i) * a.max_pages + used[i] + m - take[i]] = a.ring[ring_at(a, first, x.taken_before + m)];
  }
  give[tid] = block_exclusive_scan<kPlanBlock>(max(0, y.used - y.will), scan_lds, &moved);
  __syncthreads();
  const int end = ring_at(a, first, count);      // count == n_pages: the front, and nothing is given
  for (int m = tid; m < moved; m += kPlanBlock) {
    const int i = last_below(give, kPlanBlock, m);
    a.ring[ring_at(a, end, x.given_before + m)] = a.pages[static_cast<int64_t>(begin + i) * a.max_pages + will[i] + m - give[i]];
  }
}

// The group that sequence s belongs to: its prefix's length.
__device__ __forceinline__ int prefix_of(const PlanArgs& a, int s) {
  if (a.n_group == 0 || s < a.group_seq[0] || s >= a.group_seq[a.n_group]) return 0;
  const int n = a.prefix_len[last_below(a.group_seq, a.n_group, s)];
  return n < 0 || n > 1 << 30 ? 0 : n;
}

// Parents of a workgroup's tokens and of the 64 in front of them, in which the trees that it has a part of begin.
struct Parents {
  int of[256 + kMostDrafted];
};

// The way from token j of a tree to its root, `here` the token's place in the list.
__device__ __forceinline__ uint64_t path_of(const int* here, int j, int* error) {
  uint64_t bits = 0;
  for (int i = j;;) {
    bits |= uint64_t{1} << i;
    const int up = here[i - j];
    if (up < -1 || up >= i) *error |= AT_GRPO_DATA_TREE;
    if (up < 0 || up >= i) return bits;
    i = up;
  }
}

__global__ __launch_bounds__(256) void k_plan_tokens(PlanArgs a) {
  __shared__ Parents parents;
  const int tid = threadIdx.x;
  const int64_t begin = static_cast<int64_t>(flat_block()) * 256, at = begin + tid;
  if (at == 0) {
    a.state_out[0] = a.verdict[1];
    a.state_out[1] = a.verdict[2];
  }
  if (at < a.n_seq) a.length_out[at] = a.behind[at];
  const int total = a.cu_q[a.n_seq];      // 0 where the step is refused
  if (a.parent && begin < total) {
    for (int i = tid; i < 256 + kMostDrafted; i += 256) {
      const int64_t t = begin - kMostDrafted + i;
      parents.of[i] = t >= 0 && t < total ? a.parent[t] : -1;
    }
  }
  __syncthreads();
  int error = 0;
  if (at < total) {
    const int t = static_cast<int>(at), s = last_below(a.cu_q, a.n_seq + 1, t), j = t - a.cu_q[s], keep = a.kept[s], place = keep + j;
    int depth = j;
    if (a.parent) {
      const uint64_t bits = path_of(parents.of + kMostDrafted + tid, j, &error);
      depth = __popcll(bits) - 1;
      if (a.ancestors) a.ancestors[t] = bits;
    }
    if (a.seq) a.seq[t] = s;
    if (a.position) a.position[t] = (a.verdict[0] ? prefix_of(a, s) : 0) + keep + depth;
    if (a.slot)
      a.slot[t] = (static_cast<int64_t>(a.pages[static_cast<int64_t>(s) * a.max_pages + (place >> a.shift)]) << a.shift) + (place & ((1 << a.shift) - 1));
  }
  raise_data_error(a.data_error, error);
}

// ---- in one launch ------------------------------------------------------------------------------------
constexpr int kPlanAlone = 8 * kPlanBlock;

template <int BLOCK>
struct PlanLds {
  static constexpr int kSeqs = 2 * BLOCK;
  int cu[kSeqs], take[kSeqs], give[kSeqs], group[kSeqs];      // in front of each sequence; the last group that begins there or in front
  int keep[kSeqs], used[kSeqs];
  int wave_take[BLOCK / 64], wave_give[BLOCK / 64], wave_group[BLOCK / 64], wave_wrong[BLOCK / 64], wave_falls[BLOCK / 64];
  int64_t wave_add[BLOCK / 64];
  int parents[BLOCK + kMostDrafted];
};

// BLOCK threads for 2 BLOCK sequences.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_plan(PlanArgs a, int64_t per) {
  __shared__ PlanLds<BLOCK> lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = a.state[0], count = a.state[1];
  for (int s = tid; s < 2 * BLOCK; s += BLOCK) lds.group[s] = -1;
  Step of[2];
  int take = 0, give = 0, wrong = 0;
  int64_t add = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {      // two sequences side by side a thread
    const int s = 2 * tid + k;
    of[k] = s < a.n_seq ? step_of(a, s) : Step{};
    take += max(0, of[k].will - of[k].used);
    give += max(0, of[k].used - of[k].will);
    add += of[k].add;
    wrong |= of[k].wrong;
  }
  __syncthreads();
  // Where groups begin: of several that begin with a sequence the last, which is the one that has it.
  int falls = 0, error = 0;
  for (int g = tid; g < a.n_group; g += BLOCK) {
    const int s0 = a.group_seq[g], s1 = a.group_seq[g + 1], n = a.prefix_len[g];
    falls |= s0 < 0 || s1 < s0 || s1 > a.n_seq;
    if (n < 0 || n > 1 << 30) error |= AT_GRPO_DATA_SEQLENS;
    if (s0 >= 0 && s0 < a.n_seq) atomicMax(&lds.group[s0], g);
  }
  if (falls) error |= AT_GRPO_DATA_SEQLENS;
  __syncthreads();
  const int own_group[2] = {lds.group[2 * tid], max(lds.group[2 * tid], lds.group[2 * tid + 1])};
  int take_up = take, give_up = give, group_up = own_group[1];      // up to this thread
  int64_t add_up = add;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(take_up, o, 64), g = __shfl_up(give_up, o, 64), m = __shfl_up(group_up, o, 64);
    const int64_t d = __shfl_up(add_up, o, 64);
    if (lane >= o) {
      take_up += t;
      give_up += g;
      add_up += d;
      group_up = max(group_up, m);
    }
  }
  wrong = __any(wrong);
  falls = __any(falls);
  if (lane == 63) {
    lds.wave_take[wave] = take_up;
    lds.wave_give[wave] = give_up;
    lds.wave_add[wave] = add_up;
    lds.wave_group[wave] = group_up;
    lds.wave_wrong[wave] = wrong;
    lds.wave_falls[wave] = falls;
  }
  __syncthreads();
  Sums all{};
  int take0 = take_up - take, give0 = give_up - give, group0 = -1;
  int64_t add0 = add_up - add;
  falls = 0;
#pragma unroll
  for (int w = 0; w < BLOCK / 64; ++w) {
    if (w < wave) {
      take0 += lds.wave_take[w];
      give0 += lds.wave_give[w];
      add0 += lds.wave_add[w];
      group0 = max(group0, lds.wave_group[w]);
    }
    all.taken += lds.wave_take[w];
    all.given += lds.wave_give[w];
    all.added += lds.wave_add[w];
    all.wrong |= lds.wave_wrong[w];
    falls |= lds.wave_falls[w];
  }
  // of the lanes in front in the wavefront
  const int lane_before = __shfl_up(group_up, 1, 64);
  if (lane > 0) group0 = max(group0, lane_before);
  const int refused = verdict_of(a, first, count, all);
  if (blockIdx.x == 0) raise_data_error(a.data_error, error | (tid == 0 ? refused : 0));
  const int total = refused ? 0 : static_cast<int>(all.added);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = 2 * tid + k;
    lds.cu[s] = refused ? 0 : static_cast<int>(add0);
    lds.take[s] = take0;
    lds.give[s] = give0;
    lds.keep[s] = of[k].keep;
    lds.used[s] = of[k].used;
    add0 += of[k].add;
    take0 += max(0, of[k].will - of[k].used);
    give0 += max(0, of[k].used - of[k].will);
  }
  __syncthreads();      // every thread has read which groups begin where
  lds.group[2 * tid] = max(group0, own_group[0]);
  lds.group[2 * tid + 1] = max(group0, own_group[1]);
  __syncthreads();

  const int64_t step = static_cast<int64_t>(gridDim.x) * BLOCK, here = static_cast<int64_t>(blockIdx.x) * BLOCK + tid;
  // the tokens
  const int64_t t0 = blockIdx.x * per, t1 = min<int64_t>(total, t0 + per);
  for (int64_t begin = t0; begin < t1; begin += BLOCK) {
    if (a.parent) {
      __syncthreads();
      for (int i = tid; i < BLOCK + kMostDrafted; i += BLOCK) {
        const int64_t t = begin - kMostDrafted + i;
        lds.parents[i] = t >= 0 && t < total ? a.parent[t] : -1;
      }
      __syncthreads();
    }
    const int64_t at = begin + tid;
    if (at >= t1) continue;
    const int t = static_cast<int>(at), s = last_below(lds.cu, a.n_seq, t), j = t - lds.cu[s], place = lds.keep[s] + j, page = place >> a.shift;
    int depth = j, wrong_parent = 0;
    const int g = lds.group[s];
    int64_t id = 0;
    if (a.slot) {
      const int from_ring = page - lds.used[s];
      id = from_ring < 0 ? a.pages[static_cast<int64_t>(s) * a.max_pages + page] : a.ring[ring_at(a, first, lds.take[s] + from_ring)];
    }
    int prefix = 0;
    if (a.position && !falls && g >= 0 && s < a.group_seq[g + 1]) {
      prefix = a.prefix_len[g];
      if (prefix < 0 || prefix > 1 << 30) prefix = 0;
    }
    if (a.parent) {
      const uint64_t bits = path_of(lds.parents + kMostDrafted + tid, j, &wrong_parent);
      depth = __popcll(bits) - 1;
      if (a.ancestors) a.ancestors[t] = bits;
      raise_data_error(a.data_error, wrong_parent);
    }
    if (a.seq) a.seq[t] = s;
    if (a.position) a.position[t] = prefix + lds.keep[s] + depth;
    if (a.slot) a.slot[t] = (id << a.shift) + (place & ((1 << a.shift) - 1));
  }
  // pages moved
  if (!refused) {
    for (int64_t m = here; m < all.taken; m += step) {
      const int s = last_below(lds.take, a.n_seq, static_cast<int>(m));
      a.pages[static_cast<int64_t>(s) * a.max_pages + lds.used[s] + m - lds.take[s]] = a.ring[ring_at(a, first, static_cast<int>(m))];
    }
    const int end = all.given ? ring_at(a, first, count) : 0;
    for (int64_t m = here; m < all.given; m += step) {
      const int s = last_below(lds.give, a.n_seq, static_cast<int>(m));
      const int will = (lds.keep[s] + (s + 1 < a.n_seq ? lds.cu[s + 1] : total) - lds.cu[s] + (1 << a.shift) - 1) >> a.shift;
      a.ring[ring_at(a, end, static_cast<int>(m))] = a.pages[static_cast<int64_t>(s) * a.max_pages + will + m - lds.give[s]];
    }
  }
  // the sequences: behind everything that has read their lengths, where there is one workgroup
  __syncthreads();
  for (int64_t s = here; s < a.n_seq; s += step) {
    a.cu_q[s] = lds.cu[s];
    if (refused) a.length_out[s] = a.length[s];
    else a.length_out[s] = lds.keep[s] + (s + 1 < a.n_seq ? lds.cu[s + 1] : total) - lds.cu[s];
  }
  if (here == 0) {
    a.cu_q[a.n_seq] = total;
    a.state_out[0] = refused ? first : ring_at(a, first, all.taken);
    a.state_out[1] = refused ? count : count - all.taken + all.given;
  }
}

struct Span {
  const void* at;
  size_t bytes;
  bool meets(const Span& o) const {
    const uintptr_t x = reinterpret_cast<uintptr_t>(at), y = reinterpret_cast<uintptr_t>(o.at);
    return at && o.at && bytes && o.bytes && x < y + o.bytes && y < x + bytes;
  }
};

size_t lay_out(int32_t n_seq, void* workspace, PlanArgs* a) {
  WsAlloc ws(workspace);
  a->verdict = ws.take<int32_t>(4);
  a->kept = ws.take<int32_t>(n_seq);
  a->behind = ws.take<int32_t>(n_seq);
  return ws.bytes();
}

}  // namespace
}  // namespace atg

using namespace atg;

extern "C" size_t at_grpo_kv_plan_workspace_bytes(int32_t n_seq) {
  PlanArgs a;
  return n_seq < 0 ? 0 : lay_out(n_seq, nullptr, &a);
}

extern "C" int at_grpo_kv_plan(const at_grpo_page_pool* pool, int32_t n_tok, const int32_t* length, const int32_t* keep, const int32_t* add,
                               const int32_t* parent, const int32_t* state, int32_t* length_out, int32_t* state_out, int32_t* cu_q, int32_t* seq,
                               int32_t* position, int64_t* slot, uint64_t* ancestors, int32_t* data_error, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
  if (!pool || n_tok < 0 || pool->n_pages <= 0 || pool->n_seq < 0 || pool->max_pages < 0 || pool->n_group < 0) return AT_GRPO_EINVAL;
  if (pool->page_size < 8 || pool->page_size > 65536 || (pool->page_size & (pool->page_size - 1))) return AT_GRPO_EUNSUPPORTED;
  // places, pages of all sequences, groups (a thread's next is up to 1024 further) and threads of a launch are counted in 32 bits
  if (static_cast<int64_t>(pool->max_pages) * pool->page_size > 1 << 30 || static_cast<int64_t>(pool->n_seq) * pool->max_pages > 0x7fffffff ||
      n_tok > 0x7fffff00 || pool->n_seq > 0x3fffff00 || pool->n_group > 0x3fffff00)
    return AT_GRPO_EUNSUPPORTED;
  const size_t S = pool->n_seq, T = n_tok, word = sizeof(int32_t);
  if (!pool->ring || !state || !state_out || !cu_q || (S > 0 && (!length || !add || !length_out || (pool->max_pages > 0 && !pool->pages)))) return AT_GRPO_EINVAL;
  if (pool->n_group > 0 && (!pool->group_seq || !pool->prefix_len)) return AT_GRPO_EINVAL;
  if (ancestors && !parent) return AT_GRPO_EINVAL;
  if (keep == length) keep = nullptr;
  const Span in[] = {{length, S * word}, {state, 2 * word}, {keep, S * word}, {add, S * word}, {parent, T * word},
                     {pool->group_seq, pool->n_group ? (pool->n_group + size_t{1}) * word : 0}, {pool->prefix_len, pool->n_group * word}};
  const Span out[] = {{length_out, S * word}, {state_out, 2 * word}, {cu_q, (S + 1) * word}, {seq, T * word}, {position, T * word}, {slot, 2 * T * word},
                      {ancestors, 2 * T * word}, {pool->pages, S * pool->max_pages * word}, {pool->ring, pool->n_pages * word}, {data_error, word}};
  const int n_in = sizeof(in) / sizeof(in[0]), n_out = sizeof(out) / sizeof(out[0]);
  for (int o = 0; o < n_out; ++o) {
    for (int i = 0; i < n_in; ++i)
      if (out[o].meets(in[i]) && !(o == i && o < 2 && out[o].at == in[i].at)) return AT_GRPO_EINVAL;
    for (int i = 0; i < o; ++i)
      if (out[o].meets(out[i])) return AT_GRPO_EINVAL;
  }
  int shift = 0;
  while ((1 << shift) < pool->page_size) ++shift;
  PlanArgs a{shift, pool->n_pages, pool->n_seq, pool->max_pages, pool->n_group, n_tok, pool->pages, pool->ring, pool->group_seq, pool->prefix_len, length, keep,
             add, parent, state, length_out, state_out, cu_q, seq, position, slot, ancestors, data_error, nullptr, nullptr, nullptr};
  const size_t bytes = lay_out(pool->n_seq, workspace, &a);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < bytes) return AT_GRPO_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  ProfScope ps(PROF_PLAN, s);
  // One launch for few sequences; in place by one workgroup, which has a share of at most 8192 tokens.  The smaller workgroup for few of both: four
  // candidates 6.7 us by 1024 threads, 4.3 by 256.
  const bool in_place = length_out == length || state_out == state;
  const bool small = pool->n_seq <= 512 && n_tok <= 1024;
  const int block = small ? 256 : kPlanBlock;
  if (pool->n_seq <= 2 * kPlanBlock && (!in_place || n_tok <= kPlanAlone)) {
    const int64_t per = in_place ? (n_tok > block ? n_tok : block) : block * (1 + n_tok / (int64_t{block} * 512));
    const int64_t blocks = n_tok ? ceil_div(n_tok, per) : 1;
    hipLaunchKernelGGL(small ? k_plan<256> : k_plan<kPlanBlock>, dim3(static_cast<unsigned>(blocks)), dim3(block), 0, s, a, per);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  }
  hipLaunchKernelGGL(k_plan_sequences, dim3(static_cast<unsigned>(S ? ceil_div(S, kPlanBlock) : 1)), dim3(kPlanBlock), 0, s, a);
  ATG_LAUNCH_CHECK();
  const int64_t threads = static_cast<int64_t>(T > S ? T : S);
  hipLaunchKernelGGL(k_plan_tokens, grid_of(threads ? ceil_div(threads, 256) : 1), dim3(256), 0, s, a);
  ATG_LAUNCH_CHECK();
  return AT_GRPO_OK;
}
