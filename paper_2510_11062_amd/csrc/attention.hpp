// Attention of new tokens over a paged cache, the prompts of groups of candidates among it (gfx950).
//
//   out = sum_i p_i v_i / sum_i p_i,  p_i = exp(scale <q, k_i> - m)  over the visible tokens i
//
// in one pass with a running maximum m.  What there is to read is the keys and values, and where few queries read them their passage
// from memory bounds the call; with many queries the products do.  Hence units of work that read a token once for all queries that see
// it.  A unit's rows are its queries times the Hq / Hk heads that share a key head, cut into tiles of 16 to 128; a tile's passage over a
// unit's tokens for one key head is a run.  The runs of the whole batch, one behind the other, are dealt to the workgroups in shares of
// equal cost, wherever that cuts a run: long prompts and ragged responses fill the chip alike, whatever their lengths, which only the
// device knows.  A second kernel joins the parts of a row.  Three kernels, by the rows of a sequence:
//   k_decode        at most 16: a unit is a group, whose rows read its prefix and then its sequences' own tokens as one stream
//   k_attend_wide   more, in bf16: units are the prefix of a group with the queries of all its sequences, and a sequence's own tokens with its
//                   queries; tiles of 128 rows
//   k_attend        the same in fp32, and where k_decode's tables end; tiles of 16 or 32 rows
// and, for trees, k_tree_near where there is little of everything.
//
// In the first and the last a wavefront holds a tile's queries, takes 32 tokens at a time (16 in fp32) and keeps everything in registers:
//   S^T = K Q^T     MFMA 16x16: tokens down, queries across, so that a lane has four consecutive tokens of one query
//   P^T             is at once the second product's operand: no lane needs a weight that another one computed
//   O^T += V^T P^T  a lane loads whole rows of V, eight elements of eight tokens, and transposes that block by itself
// The four wavefronts of a workgroup take turns in a run's tokens and add up at its end.
//
// With TREE a sequence's new tokens are a tree: each has a word of bits for those of them that it sees (see tree_bits), in place of an order.
#pragma once

#include "gemm_bf16.hpp"
#include "kv_common.hpp"

#include <math.h>

#include <type_traits>

namespace atg {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMostGroups = 1024;     // workgroups of a launch
constexpr int kCachedUnits = 512;     // units whose sizes are kept in LDS
// A run's beginning and end (queries, first loads, adding up) take about as long as 128 tokens and count as that.
constexpr int kRunCost = 16, kMinShare = 16;
// A tree's run has two tiles that not all see, and few rows to a tile: 6.8 us beside 2.2 to 2.5 for 64 tokens.  220 candidates with 16 drafted tokens
// 275 us with 16, 265 with 32, 278 with 56; two prompts of 40000 tokens 249, 219 and 225.
constexpr int kTreeRunCost = 32;
constexpr int kPageSlots = 1024;     // page ids of a chunk in LDS at a time
constexpr int kMaxRows = 128;        // rows of the largest tile
constexpr int kWideRows = 128;       // of the tiles below that four wavefronts share by rows
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The running maximum is raised where a score passes it by more than this (in powers of two): weights of at most 2^8 lose nothing in
// fp32 sums, nor in bf16, whose error is relative, and most tokens then leave the sums as they are.
constexpr float kSlack = 8.f;
// Up to where a row's exponents are its scores' multiples less the largest's, in one instruction: that multiple is rounded, and half a unit of its last
// place, here at most 2^-5, is in every exponent.  From 2^32 on it is past 127, where all weights are infinite or 0.
// Differences for all rows would take an instruction a score: trees of 24 conversations, heads of 64, 81.6 us, by this branch 80.8, by neither 77.8; elsewhere
// a tile's check costs up to 1 %, 0.1 to 0.6 us of calls of 8 to 20.
constexpr float kFar = 0x1p20f;

// x / d for 0 <= x < 2^31 by a product: ceil(2^(31 + k) / d) with 2^k >= d is off by less than one part in 2^31.
struct Divisor {
  uint32_t d, mul, shift;      // shift: k - 1; d == 1 has no product
};
Divisor divisor(int d) {
  int k = 0;
  while ((int64_t{1} << k) < d) ++k;
  return Divisor{static_cast<uint32_t>(d), d == 1 ? 0 : static_cast<uint32_t>(((uint64_t{1} << (31 + k)) + d - 1) / d), static_cast<uint32_t>(k - 1)};
}
__device__ __forceinline__ int operator/(int x, const Divisor& by) {
  return by.d == 1 ? x : static_cast<int>(__umulhi(static_cast<uint32_t>(x), by.mul) >> by.shift);
}

struct Args {
  int n_tok, Hq, share;      // share: Hq / Hk
  Divisor by_share;
  int coarse, rise, quantum; // of the costs below; rise: by how much from one causal tile to the next
  int causal, run_cost;      // run_cost: of a run's beginning and end
  float scale;
  Rows q, out;
  float* lse;                // [n_tok, Hq] or null
  const uint64_t* ancestors; // [n_tok]: with TREE
  int32_t* data_error;
  int4* units;               // workspace: [n_group + n_seq] cost in front of the unit, its length, first token, tokens; then {share, all cost, whether an index falls}
  // Parts, each divided by its own sum.  A run's first part lies by its query and head, those of prefixes first: [2 or 1][n_tok][Hq].
  // A workgroup's first part, where it begins inside a run, lies behind them: [workgroup][row of the tile].
  float* part_lse;
  float* part_out;           // .. [D]
};

// A unit: queries tok0 .. tok0 + ntok - 1 over the first `len` tokens of a page table.  Units 0 .. n_group - 1 are the prefixes.
struct Unit {
  int tok0, ntok, len, row;      // row: of the page table
};

// Of 64 tokens, the first of which is number `from` of a sequence's new ones, those that one of these sees: all in front of the new ones, of these
// the ones that its bits name, and none behind the 64th.
__device__ __forceinline__ uint64_t tree_bits(uint64_t path, int from) {
  if (from >= 0) return from < 64 ? path >> from : 0;
  return from <= -64 ? ~uint64_t{0} : path << -from | ((uint64_t{1} << -from) - 1);
}
constexpr int kMostTree = 64;

// Without sequences nothing else looks at the one entry of cu_q, up to which and from which on rows belong to nobody.
__device__ __forceinline__ bool no_sequence_falls(const KvView& kv, int n_tok) {
  return kv.n_seq == 0 && kv.cu_q && (kv.cu_q[0] < 0 || kv.cu_q[0] > n_tok);
}

__device__ __forceinline__ Unit unit_of(const KvView& kv, int u, int n_tok, int* error, bool* falls) {
  int s0 = u - kv.n_group, s1 = s0 + 1, len, most;
  if (u < kv.n_group) {
    s0 = kv.group_seq[u];
    s1 = kv.group_seq[u + 1];
    if (s0 < 0 || s1 < s0 || s1 > kv.n_seq) {
      *falls = true;
      return Unit{0, 0, 0, 0};
    }
    len = kv.prefix_len[u];
    most = kv.max_prefix_pages << kv.page_shift;
  } else {
    len = kv.length[s0];
    most = kv.max_pages << kv.page_shift;
  }
  const int t0 = kv.cu_q ? kv.cu_q[s0] : s0, t1 = kv.cu_q ? kv.cu_q[s1] : s1;
  if (t0 < 0 || t1 < t0 || t1 > n_tok) {
    *falls = true;
    return Unit{0, 0, 0, 0};
  }
  if (len < 0 || len > most) {
    *error |= AT_GRPO_DATA_SEQLENS;
    len = 0;
  }
  return Unit{t0, t1 - t0, len, u < kv.n_group ? u : s0};
}

__device__ __forceinline__ int tiles_of(int ntok, int share, int rows) { return (ntok * share + rows - 1) / rows; }

// A unit's tokens up to the last that a tile sees: those of causal tiles rise.
__device__ __forceinline__ int end_of(const Unit& u, bool steps, const Args& a, int tile, int rows) {
  const int last = (min(u.ntok * a.share, (tile + 1) * rows) - 1) / a.by_share;
  return steps ? max(0, min(u.len, u.len - u.ntok + 1 + last)) : u.len;
}
// Costs are counted in eights of tokens (<< coarse).  Those of a unit's tiles rise by `step` from one to the next, by which sums over tiles
// are closed forms; with causal tiles of a whole number of tokens they rise as their tokens do.
struct Cost {
  int first, step;
  __device__ __forceinline__ int of(int tile) const { return first + tile * step; }
  __device__ __forceinline__ int in_front(int tile) const { return tile * first + step * (tile * (tile - 1) / 2); }
};
__device__ __forceinline__ Cost cost_of(const Unit& u, bool steps, const Args& a, int rows) {
  if (u.len == 0 || u.ntok == 0) return Cost{0, 0};
  const bool rises = steps && a.rise && u.ntok <= u.len;
  const int first = (((rises ? end_of(u, true, a, 0, rows) : u.len) + 7) >> 3 >> a.coarse) + a.run_cost;
  return Cost{(first + a.quantum - 1) & -a.quantum, rises ? a.rise : 0};
}
__device__ __forceinline__ int head_cost(const Unit& u, bool steps, const Args& a, int rows) {
  return cost_of(u, steps, a, rows).in_front(tiles_of(u.ntok, a.share, rows));
}

// Where a run of `cost` over tokens 0 .. end - 1 is cut: the block of 64 tokens that stands at `at` of its cost.
__device__ __forceinline__ int cut(int at, int cost, int end) {
  if (at >= cost) return end;
  return min(end, static_cast<int>(static_cast<float>((end + 63) >> 6) * (static_cast<float>(at) / static_cast<float>(cost))) << 6);
}

// A workgroup's share of the runs.
struct Schedule {
  int wave_cost[4], wave_falls[4];
  int unit, base;      // the unit that the workgroup begins in, and the cost in front of it
  Unit cache[kCachedUnits];
};

struct Share {
  int number, at, stop;
};

// The costs of all units, a contiguous part of them on each thread, and the workgroup's share of them; the same in every workgroup.
template <int R>
__device__ Share make_schedule(const KvView& kv, const Args& a, Schedule& S) {
  const int n = kv.n_group + kv.n_seq, per = (n + 255) / 256, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int u0 = min(n, tid * per), u1 = min(n, u0 + per);
  int error = 0, mine = 0;
  bool falls = no_sequence_falls(kv, a.n_tok);
  for (int u = u0; u < u1; ++u) {
    const Unit x = unit_of(kv, u, a.n_tok, &error, &falls);
    if (u < kCachedUnits) S.cache[u] = x;
    mine += head_cost(x, a.causal && u >= kv.n_group, a, R) * kv.Hk;
  }
  int sum = mine;      // of the threads up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(sum, o, 64);
    if (lane >= o) sum += up;
  }
  const bool wave_falls = __any(falls);
  if (lane == 63) {
    S.wave_cost[wave] = sum;
    S.wave_falls[wave] = wave_falls;
  }
  __syncthreads();
  const bool none = S.wave_falls[0] | S.wave_falls[1] | S.wave_falls[2] | S.wave_falls[3];
  int total = 0, first = sum - mine;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) first += S.wave_cost[w];
    total += S.wave_cost[w];
  }
  if (none) total = 0;
  total = __builtin_amdgcn_readfirstlane(total);
  const int share = max(kMinShare, (total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x));
  // neighbouring shares go to one XCD
  const int per_xcd = gridDim.x >> 3, w = per_xcd << 3 == gridDim.x ? (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3) : blockIdx.x;
  const int at = static_cast<int>(min<int64_t>(total, static_cast<int64_t>(w) * share));
  if (blockIdx.x == 0) {       // for the kernel that joins the parts
    if (none) error |= AT_GRPO_DATA_SEQLENS;
    raise_data_error(a.data_error, error);
    int base = first;
    for (int u = u0; u < u1; ++u) {
      Unit x{0, 0, 0, 0};
      if (!none) x = u < kCachedUnits ? S.cache[u] : unit_of(kv, u, a.n_tok, &error, &falls);
      const int c = head_cost(x, a.causal && u >= kv.n_group, a, R);
      a.units[u] = make_int4(base, x.len, x.tok0, x.ntok);
      base += c * kv.Hk;
    }
    if (tid == 0) a.units[n] = make_int4(share, total, none, 0);
  }
  if (at < total && first <= at && at - first < mine) {
    int base = first, u = u0;
    for (;; ++u) {
      const Unit x = u < kCachedUnits ? S.cache[u] : unit_of(kv, u, a.n_tok, &error, &falls);
      const int c = head_cost(x, a.causal && u >= kv.n_group, a, R) * kv.Hk;
      if (at < base + c) break;
      base += c;
    }
    S.unit = u;
    S.base = base;
  }
  __syncthreads();
  return Share{w, at, min(total, at + share)};
}

// The runs of a workgroup's share, one after the other: everything in it is uniform.
template <int R>
struct Runs {
  const KvView& kv;
  const Args& a;
  const Schedule& S;
  int number, at, stop;      // of the workgroup; the cost at hand, the end of its share
  int u, base, unit_stop;    // the unit, the costs in front of it and of the share in it
  Unit x;
  bool own, steps;
  Cost costs;
  int tiles, hk, tile, run0, cost;

  __device__ __forceinline__ Runs(const KvView& kv_, const Args& a_, const Schedule& S_, const Share& mine)
      : kv(kv_), a(a_), S(S_), number(mine.number), at(mine.at), stop(mine.stop) {
    if (!valid()) return;
    u = __builtin_amdgcn_readfirstlane(S.unit);
    base = __builtin_amdgcn_readfirstlane(S.base);
    enter();
    const int head = costs.in_front(tiles);
    hk = (at - base) / head;
    run0 = base + hk * head;
    tile = 0;
    if (costs.step == 0) {
      tile = (at - run0) / cost;
      run0 += tile * cost;
    }
    for (; at >= run0 + cost; ++tile, cost += costs.step) run0 += cost;
  }
  __device__ __forceinline__ bool valid() const { return at < stop; }
  __device__ __forceinline__ int from() const { return at - run0; }                      // the part of the run's cost
  __device__ __forceinline__ int to() const { return min(unit_stop, run0 + cost) - run0; }

  __device__ __forceinline__ void next() {
    at = min(unit_stop, run0 + cost);
    if (!valid()) return;
    run0 += cost;
    cost += costs.step;
    if (++tile == tiles) {
      tile = 0;
      ++hk;
      cost = costs.first;
    }
    while (at >= unit_stop) {
      base = unit_stop;
      ++u;
      enter();
      hk = tile = 0;
      run0 = base;
    }
  }

 private:
  __device__ __forceinline__ void enter() {      // unit u, first run
    int error = 0;
    bool falls = false;
    x = u < kCachedUnits ? S.cache[u] : unit_of(kv, u, a.n_tok, &error, &falls);
    x.tok0 = __builtin_amdgcn_readfirstlane(x.tok0);
    x.ntok = __builtin_amdgcn_readfirstlane(x.ntok);
    x.len = __builtin_amdgcn_readfirstlane(x.len);
    x.row = __builtin_amdgcn_readfirstlane(x.row);
    own = u >= kv.n_group;
    steps = own && a.causal;
    tiles = tiles_of(x.ntok, a.share, R);
    costs = cost_of(x, steps, a, R);
    cost = costs.first;
    unit_stop = min(stop, base + costs.in_front(tiles) * kv.Hk);
  }
};

// A run of a tile: key head, first row, and the tokens that the workgroup has of it.
struct TileRun {
  int hk, r0, k0, k1;
};
template <int R>
__device__ __forceinline__ TileRun tile_run(const Runs<R>& r, const Args& a) {
  const int end = end_of(r.x, r.steps, a, r.tile, R);
  return TileRun{r.hk, r.tile * R, cut(r.from(), r.cost, end), cut(r.to(), r.cost, end)};
}

// What a lane (m, g) = (lane & 15, lane >> 4) holds of a tile of TOK tokens.
//   bf16: K elements 32 c + 8 g .. + 7 of tokens m and 16 + m; V elements 128 b + 8 m .. + 7 (64-wide heads: 4 m .. + 3) of the tokens
//         4 g .. + 3 and 16 + 4 g .. + 3.
//   fp32: K elements 16 c + 4 g .. + 3 of token m; V elements 64 b + 4 m .. + 3 of tokens 4 g .. + 3.
// E: elements of V in a lane's row; NB: blocks of 16 E in a head.
template <typename T, int D>
struct Shape;
template <int D>
struct Shape<bf16_t, D> {
  static constexpr int TOK = 32, SUB = 2, KC = D / 32, KE = 8, E = D >= 128 ? 8 : 4, NB = D / (16 * E);
  typedef uint4 KV;
  typedef typename std::conditional<E == 8, uint4, uint2>::type VV;
};
template <int D>
struct Shape<float, D> {
  static constexpr int TOK = 16, SUB = 1, KC = D / 16, KE = 4, E = 4, NB = D / 64;
  typedef f32x4 KV;
  typedef f32x4 VV;
};

__device__ __forceinline__ uint32_t dword(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t dword(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

// Element e of eight tokens' rows, side by side: an operand of V^T.
template <typename VV>
__device__ __forceinline__ bf16x8 transposed(const VV (&v)[8], int e) {
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = __builtin_amdgcn_perm(dword(v[2 * j + 1], e >> 1), dword(v[2 * j], e >> 1), e & 1 ? 0x07060302u : 0x05040100u);
  return __builtin_bit_cast(bf16x8, make_uint4(o[0], o[1], o[2], o[3]));
}

// The largest magnitude as an integer, of two bfloat16 a word or of float32: infinities and NaN are above every number.
typedef unsigned short Halves __attribute__((ext_vector_type(2)));
template <typename V>
__device__ __forceinline__ uint32_t largest_bits(uint32_t high, const V& v) {
  if constexpr (std::is_same<V, f32x4>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i) high = max(high, __float_as_uint(v[i]) & 0x7fffffffu);
  } else {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(V) / 4); ++i)
      high = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Halves, high), __builtin_bit_cast(Halves, dword(v, i) & 0x7fff7fffu)));
  }
  return high;
}
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t high) {
  return sizeof(T) == 4 ? high >= 0x7f800000u : (high & 0xffffu) >= 0x7f80u || high >= 0x7f800000u;
}

__device__ __forceinline__ float element(const f32x4& v, int e) { return v[e]; }
template <typename V>
__device__ __forceinline__ float element(const V& v, int e) {
  return __uint_as_float(e & 1 ? dword(v, e >> 1) & 0xffff0000u : dword(v, e >> 1) << 16);
}
// The largest of three, or NaN: v_maximum3_f32, where fmaxf takes an instruction more for each number that might be a signalling NaN.  Not in asm: what a matrix
// instruction writes may be read only some cycles later, and the compiler waits for its own instructions alone.
__device__ __forceinline__ float maximum3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// 0 in place of infinities and NaN
__device__ __forceinline__ uint32_t finite_halves(uint32_t x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0 : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0 : x & 0xffff0000u);
}
__device__ __forceinline__ uint4 finite_of(const uint4& v) { return make_uint4(finite_halves(v.x), finite_halves(v.y), finite_halves(v.z), finite_halves(v.w)); }
__device__ __forceinline__ uint2 finite_of(const uint2& v) { return make_uint2(finite_halves(v.x), finite_halves(v.y)); }
__device__ __forceinline__ f32x4 finite_of(const f32x4& v) {
  f32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = not_finite(v[i]) ? 0.f : v[i];
  return x;
}

struct Lds {
  Schedule S;
  int pages[2][kPageSlots];
  int holes[2][4];
  float ml[4][64][2];
  float slab[4][16][128 + 4];
};

// 16 or 8 bytes that nothing reads again while the caches hold them: keys and values of a decode, 117 us for 32 groups, then 106.
template <typename V>
__device__ __forceinline__ V load_once(const void* p) {
  typedef float Words __attribute__((ext_vector_type(sizeof(V) / 4)));
  return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const Words*>(p)));
}

// S^T = K Q^T of a tile.
template <typename T, int D, int NR>
__device__ __forceinline__ void scores(const typename Shape<T, D>::KV (&k)[Shape<T, D>::SUB][Shape<T, D>::KC],
                                       const typename Shape<T, D>::KV (&q)[NR][Shape<T, D>::KC], f32x4 (&s)[NR][Shape<T, D>::SUB]) {
  constexpr int SUB = Shape<T, D>::SUB, KC = Shape<T, D>::KC;
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      s[n][y] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        if constexpr (sizeof(T) == 2) {
          s[n][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[y][x]), __builtin_bit_cast(bf16x8, q[n][x]), s[n][y], 0, 0, 0);
        } else {
#pragma unroll
          for (int z = 0; z < 4; ++z) s[n][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[y][x][z], q[n][x][z], s[n][y], 0, 0, 0);
        }
      }
    }
}

// A weight of 0 does not keep an infinite or NaN value out of a product.  In a tile that some rows do not see in full such values are added to
// the rows that see them, one by one, and the products get 0 in their place.  `slab`: a wavefront's part of LDS for 32 tokens of 128 elements.
template <typename T, int D, int NR, typename Sees>
__device__ __forceinline__ void set_apart(float* slab, typename Shape<T, D>::VV (&v)[Shape<T, D>::NB][4 * Shape<T, D>::SUB],
                                          f32x4 (&acc)[NR][Shape<T, D>::NB][Shape<T, D>::E], Sees sees) {
  typedef Shape<T, D> Z;
  typedef typename Z::VV VV;
  uint32_t high = 0;
#pragma unroll
  for (int b = 0; b < Z::NB; ++b)
#pragma unroll
    for (int j = 0; j < 4 * Z::SUB; ++j) high = largest_bits(high, v[b][j]);
  if (!__any(not_finite<T>(high))) return;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  VV* const at = reinterpret_cast<VV*>(slab);
#pragma unroll
  for (int b = 0; b < Z::NB; ++b) {
#pragma unroll
    for (int j = 0; j < 4 * Z::SUB; ++j) {
      at[(16 * (j >> 2) + 4 * g + (j & 3)) * 16 + m] = v[b][j];
      v[b][j] = finite_of(v[b][j]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int i = 0; i < 16 * Z::TOK; ++i) {
      const VV x = at[i];
      if (!__any(not_finite<T>(largest_bits(0u, x)))) continue;
      const int token = i >> 4, of = i & 15;      // whose elements E of .. are those of the fourth of the lanes of / 4
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const bool on = g == of >> 2 && sees(n, token);
#pragma unroll
        for (int e = 0; e < Z::E; ++e) {
          const float y = element(x, e), add = on && not_finite(y) ? y : 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[n][b][e][c] += c == (of & 3) ? add : 0.f;
        }
      }
    }
    asm volatile("" ::: "memory");
  }
}

// What a row's weights are relative to: `top`, its largest score at some time (-inf: none yet), and `lead`, that times log2 e and the scale.  Raises them to `high`,
// the largest of a tile; returns what sums up to there are multiplied by.
template <bool EACH>
__device__ __forceinline__ float raise_top(float high, float to_log2, float& top, float& lead) {
  if (EACH && !(high * to_log2 > lead + kSlack)) high = top;
  top = fmaxf(high, top);
  const float now = top * to_log2, keep = __builtin_amdgcn_exp2f(lead - (now == -INFINITY ? 0.f : now));
  lead = now;
  return keep;
}
// Far from 0 the scores of a tile become differences from the largest before their exponents are taken, so that it has none, and any larger one raises it.
// `less` is what they are less by, `lead` 0 then.
__device__ __forceinline__ bool is_far(float top, float lead) { return fabsf(lead) > kFar && top > -INFINITY; }
__device__ __forceinline__ float raise_far(float high, float to_log2, float& top, float& lead, float& less) {
  const bool far = is_far(top, lead);
  const float now = far ? fmaxf(high, top) : top, keep = far ? __builtin_amdgcn_exp2f((top - now) * to_log2) : 1.f;
  top = now;
  less = far ? now : 0.f;
  lead = far ? 0.f : lead;
  return keep;
}
// The largest score's multiple; a number where the product is none.
__device__ __forceinline__ float top_log2(float top, float to_log2) {
  return top == -INFINITY ? top : fminf(fmaxf(top * to_log2, -0x1.fffffep127f), 0x1.fffffep127f);
}

// The tile's weights into the sums, and their products with its values into the accumulators; `before` the products, once these are scaled.
// The matrix instruction takes bf16 weights with bf16 values, so a weight is rounded to 8 bits there (the sums take it as it is): an error
// of up to 2^-8 of each term, of the order of the result's own rounding.  Against 64 bits bf16 results are off by 0.0023 (rounded once from
// 32 bits 0.0017).  Weights in two parts would take twice the products.
// EACH: a row's maximum is raised where its own score asks for it and not where another row's in the wavefront does, so that what one row sees
// leaves the others' bits as they are.
template <typename T, int D, bool EACH, int NR, typename Before>
__device__ __forceinline__ void weigh_and_add(const typename Shape<T, D>::VV (&v)[Shape<T, D>::NB][4 * Shape<T, D>::SUB], f32x4 (&s)[NR][Shape<T, D>::SUB],
                                              float to_log2, f32x4 (&acc)[NR][Shape<T, D>::NB][Shape<T, D>::E], float (&top)[NR], float (&sum)[NR],
                                              Before before) {
  typedef Shape<T, D> Z;
  constexpr int E = Z::E, NB = Z::NB, SUB = Z::SUB;
  constexpr bool kBf16 = sizeof(T) == 2;
  uint32_t w16[NR][4];
  float w32[NR][4];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float high = -INFINITY;
#pragma unroll
    for (int y = 0; y < SUB; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) high = fmaxf(high, s[n][y][i]);
    float lead = top[n] * to_log2;
    const auto keep = [&](float x) {
      sum[n] *= x;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[n][b][e] *= x;
    };
    const auto of_row = [&] {
      const float x = fmaxf(high, __shfl_xor(high, 16, 64));
      return fmaxf(x, __shfl_xor(x, 32, 64));
    };
    if (__any(high * to_log2 > lead + kSlack)) keep(raise_top<EACH>(of_row(), to_log2, top[n], lead));
    if (__any(is_far(top[n], lead))) {
      float less;
      keep(raise_far(of_row(), to_log2, top[n], lead, less));
#pragma unroll
      for (int y = 0; y < SUB; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][y][i] -= less;
    }
    const float minus = top[n] == -INFINITY ? 0.f : lead;
    float p[4 * SUB];
#pragma unroll
    for (int y = 0; y < SUB; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * y + i] = __builtin_amdgcn_exp2f(fmaf(s[n][y][i], to_log2, -minus));
        sum[n] += p[4 * y + i];
      }
    if constexpr (kBf16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w16[n][j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w32[n][j] = p[j];
    }
  }
  before();
  auto product = [&](int n, int b, int e, bf16x8 vt, f32x4 x) {
    if constexpr (kBf16) {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, make_uint4(w16[n][0], w16[n][1], w16[n][2], w16[n][3])), x, 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b][i][e], w32[n][i], x, 0, 0, 0);
      return x;
    }
  };
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      bf16x8 vt;
      if constexpr (kBf16) vt = transposed(v[b], e);
#pragma unroll
      for (int n = 0; n < NR; ++n) acc[n][b][e] = product(n, b, e, vt, acc[n][b][e]);
    }
}

// Rows r0 .. rows - 1 (at most a tile) of the queries from tok0 on for key head hk.
struct RowsOf {
  int tok0, hk, r0, rows;
};

// The wavefronts' maxima and sums, and their products, which sixteen threads a row weigh and add up.  Into the output, or into a part: by
// query and head (group < 0), or with the workgroup.
template <typename T, bool EXACT, typename L, int NR, int NB, int E>
__device__ __forceinline__ void finish(const Args& a, L& lds, const f32x4 (&acc)[NR][NB][E], const float (&top)[NR], float (&sum)[NR], const RowsOf& of,
                                       bool direct, int group, int64_t by_query, int64_t by_group, int dim) {
  constexpr bool kBf16 = sizeof(T) == 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    sum[n] += __shfl_xor(sum[n], 16, 64);
    sum[n] += __shfl_xor(sum[n], 32, 64);
    if (g == 0) {
      lds.ml[wave][16 * n + m][0] = top_log2(top[n], a.scale * kLog2e);
      lds.ml[wave][16 * n + m][1] = sum[n];
    }
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = tid >> 4, r = of.r0 + 16 * n + row, tq = r / a.by_share, h = of.hk * a.share + r - tq * a.share;
    const int64_t part = group < 0 ? by_query + static_cast<int64_t>(of.tok0 + tq) * a.Hq + h : by_group + static_cast<int64_t>(group) * kMaxRows + (r - of.r0);
    float f[4];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (n || b) lds_barrier();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<f32x4*>(&lds.slab[wave][m][E * (4 * g + i) + e]) =
              f32x4{acc[n][b][e][i], acc[n][b][e + 1][i], acc[n][b][e + 2][i], acc[n][b][e + 3][i]};
      lds_barrier();
      if (b == 0) {
        float high = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) high = fmaxf(high, lds.ml[w][16 * n + row][0]);
        const float now = high == -INFINITY ? 0.f : high;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          f[w] = __builtin_amdgcn_exp2f(lds.ml[w][16 * n + row][0] - now);
          total = fmaf(f[w], lds.ml[w][16 * n + row][1], total);
        }
        const float one = total == 0.f ? 0.f : __builtin_amdgcn_rcpf(total);
#pragma unroll
        for (int w = 0; w < 4; ++w) f[w] *= one;
        if ((tid & 15) == 0 && r < of.rows) {
          const float x = total == 0.f ? -INFINITY : (now + __builtin_amdgcn_logf(total)) * kLn2;
          if (!direct) a.part_lse[part] = x;
          else if (a.lse) a.lse[static_cast<int64_t>(of.tok0 + tq) * a.Hq + h] = x;
        }
      }
      const int d = E * (tid & 15);
      if (r < of.rows && (EXACT || 16 * E * b + d < dim)) {
        f32x4 o[E / 4];
#pragma unroll
        for (int e = 0; e < E / 4; ++e) {
          f32x4 x[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) x[w] = *reinterpret_cast<const f32x4*>(&lds.slab[w][row][d + 4 * e]) * f[w];
          o[e] = (x[0] + x[1]) + (x[2] + x[3]);
        }
        if (direct) {
          T* to = static_cast<T*>(a.out.data) + (of.tok0 + tq) * a.out.ts + h * a.out.hs + 16 * E * b + d;
#pragma unroll
          for (int e = 0; e < E / 4; ++e) {
            if constexpr (kBf16) *reinterpret_cast<uint2*>(to + 4 * e) = make_uint2(pack_bf16x2(o[e][0], o[e][1]), pack_bf16x2(o[e][2], o[e][3]));
            else *reinterpret_cast<f32x4*>(to + 4 * e) = o[e];
          }
        } else {
          float* to = a.part_out + part * dim + 16 * E * b + d;
#pragma unroll
          for (int e = 0; e < E / 4; ++e) *reinterpret_cast<f32x4*>(to + 4 * e) = o[e];
        }
      }
    }
  }
}

// Workgroups on a compute unit, by the registers of a wavefront.
template <int D, int NR>
constexpr int kPerUnit = D == 256 || D * NR >= 512 ? 1 : 2;

// ---- one new token, or few, in each sequence ---------------------------------------------------------
// Here a sequence has no more rows than a tile, and all rows of a group read one stream of tokens: the prefix, then the own tokens of its
// sequences that have new ones, one behind the other, each beginning a block of 32; a row's scores for other sequences' tokens have no weight.  A unit is a
// group, or a sequence in none; with as many tiles of rows as it has, each reads the prefix and its own sequences.  What a row needs is
// in one run, so rows of runs that one workgroup had whole are done, and a run for each sequence and head, most of whose time would be
// its beginning and end, is saved: 32 groups of up to 8 take 108 us
// (540 MB, 5.0 TB/s) and 7 for their joining, with runs of prefixes and of sequences 120 and 11; two groups behind 40000 tokens 62 and 9 (5.3 TB/s),
// one group of four 10 and 4.
// Sequences whose places are kept in LDS, which is at most 64 KB so.  1280 behind prefixes of 600 tokens with 64 of their own, 32 heads on 8 of
// 128: 175 us, by k_attend 268.
constexpr int kDecodeSeqs = 1792;
constexpr int kDecodeUnits = 256;     // units
constexpr int kDecodeSlots = 2048;    // page ids of a share of a run; beyond that they are read where they lie

struct DecodeUnit {
  int tok0, ntok, seq0, seq1, prefix, blocks;      // blocks of 32: of the whole stream
};

struct DecodeLds {
  int wave_sum[4][2], wave_falls[4];
  int unit, base;
  int place[kDecodeSeqs + 1];      // blocks in front of each sequence, times 32, and how many tokens its last block has, if not 32; of the stream's tokens
  int pages_before[kDecodeSeqs + 1];
  DecodeUnit cache[kDecodeUnits];
  int pages[kDecodeSlots];
  int holes[4];
  float ml[4][64][2];
  float slab[4][16][128 + 4];
};

__device__ __forceinline__ int blocks_before(const DecodeLds& lds, int s) { return lds.place[s] >> 5; }
__device__ __forceinline__ int length_of(const DecodeLds& lds, int s) {
  const int part = lds.place[s] & 31, blocks = blocks_before(lds, s + 1) - blocks_before(lds, s);
  return 32 * blocks - (part ? 32 - part : 0);
}

struct GroupSizes {
  int seq0, seq1, prefix;
};
__device__ __forceinline__ GroupSizes group_sizes(const KvView& kv, int g) {
  return g < kv.n_group ? GroupSizes{kv.group_seq[g], kv.group_seq[g + 1], kv.prefix_len[g]} : GroupSizes{0, 0, 0};
}

// group_seq and cu_q are known to rise here.
__device__ __forceinline__ DecodeUnit decode_unit(const KvView& kv, const DecodeLds& lds, int u, const GroupSizes& of, int* error) {
  DecodeUnit x{0, 0, u - kv.n_group, u - kv.n_group + 1, 0, 0};
  if (u < kv.n_group) {
    x.seq0 = of.seq0;
    x.seq1 = of.seq1;
    x.prefix = of.prefix;
    if (x.prefix < 0 || x.prefix > (kv.max_prefix_pages << kv.page_shift)) {
      *error |= AT_GRPO_DATA_SEQLENS;
      x.prefix = 0;
    }
  } else if (kv.n_group && x.seq0 >= kv.group_seq[0] && x.seq0 < kv.group_seq[kv.n_group]) {
    x.seq1 = x.seq0;      // a group's
  }
  x.tok0 = kv.cu_q ? kv.cu_q[x.seq0] : x.seq0;
  x.ntok = (kv.cu_q ? kv.cu_q[x.seq1] : x.seq1) - x.tok0;
  x.blocks = ((x.prefix + 31) >> 5) + blocks_before(lds, x.seq1) - blocks_before(lds, x.seq0);
  return x;
}

// Cost of a run: all alike.
__device__ __forceinline__ int decode_cost(const DecodeUnit& x, const Args& a, int tiles) {
  if (x.blocks == 0 || x.ntok == 0) return 0;
  const int prefix = (x.prefix + 31) >> 5, own = x.blocks - prefix;
  return (4 * (prefix + (own + tiles - 1) / tiles) + kRunCost + a.quantum - 1) & -a.quantum;
}

template <int R>
__device__ Share decode_schedule(const KvView& kv, const Args& a, DecodeLds& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = kv.n_group + kv.n_seq;
  int error = 0;
  bool falls = no_sequence_falls(kv, a.n_tok);
  // Two sums over all threads, in front of this one's share of them.
  auto scan = [&](int& x, int& y, int* total) {
    int sx = x, sy = y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int ux = __shfl_up(sx, o, 64), uy = __shfl_up(sy, o, 64);
      if (lane >= o) {
        sx += ux;
        sy += uy;
      }
    }
    if (lane == 63) {
      lds.wave_sum[wave][0] = sx;
      lds.wave_sum[wave][1] = sy;
    }
    __syncthreads();
    x = sx - x;
    y = sy - y;
    *total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) {
        x += lds.wave_sum[w][0];
        y += lds.wave_sum[w][1];
      }
      *total += lds.wave_sum[w][0];
    }
  };
  const int per_seq = (kv.n_seq + 255) / 256, s0 = min(kv.n_seq, tid * per_seq), s1 = min(kv.n_seq, s0 + per_seq), most = kv.max_pages << kv.page_shift;
  const int per = (n + 255) / 256, u0 = min(n, tid * per);
  const GroupSizes ahead = group_sizes(kv, u0);      // on its way while the sequences are counted
  int blocks = 0, page_count = 0, unused;
  for (int s = s0; s < s1; ++s) {
    const int length = kv.length[s], q0 = kv.cu_q ? kv.cu_q[s] : s, q1 = kv.cu_q ? kv.cu_q[s + 1] : s + 1;
    falls |= q0 < 0 || q1 < q0 || q1 > a.n_tok;
    const bool wrong = length < 0 || length > most;
    if (wrong) error |= AT_GRPO_DATA_SEQLENS;
    // Of a sequence without new tokens nothing is read: no query sees it, and its pages may be somebody else's by now.
    const int len = wrong || q1 <= q0 ? 0 : length;
    lds.place[s] = len;
    blocks += (len + 31) >> 5;
    page_count += (len + (1 << kv.page_shift) - 1) >> kv.page_shift;
  }
  for (int g = tid; g < kv.n_group; g += 256) falls |= kv.group_seq[g] < 0 || kv.group_seq[g + 1] < kv.group_seq[g] || kv.group_seq[g + 1] > kv.n_seq;
  const bool wave_falls = __any(falls);
  if (lane == 0) lds.wave_falls[wave] = wave_falls;
  scan(blocks, page_count, &unused);
  const bool none = lds.wave_falls[0] | lds.wave_falls[1] | lds.wave_falls[2] | lds.wave_falls[3];
  for (int s = s0; s < s1; ++s) {
    const int len = lds.place[s];      // this thread's own
    lds.place[s] = blocks << 5 | (len & 31);
    lds.pages_before[s] = page_count;
    blocks += (len + 31) >> 5;
    page_count += (len + (1 << kv.page_shift) - 1) >> kv.page_shift;
    if (s == kv.n_seq - 1) {
      lds.place[s + 1] = blocks << 5;
      lds.pages_before[s + 1] = page_count;
    }
  }
  if (kv.n_seq == 0 && tid == 0) lds.place[0] = lds.pages_before[0] = 0;
  __syncthreads();
  const int u1 = none ? u0 : min(n, u0 + per);
  int mine = 0, zero = 0, total;
  for (int u = u0; u < u1; ++u) {
    const DecodeUnit x = decode_unit(kv, lds, u, u == u0 ? ahead : group_sizes(kv, u), &error);
    if (u < kDecodeUnits) lds.cache[u] = x;
    const int tiles = tiles_of(x.ntok, a.share, R);
    mine += tiles * decode_cost(x, a, max(1, tiles)) * kv.Hk;
  }
  int first = mine;
  scan(first, zero, &total);
  total = __builtin_amdgcn_readfirstlane(total);
  const int share = max(kMinShare, (total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x));
  const int per_xcd = gridDim.x >> 3, w = per_xcd << 3 == gridDim.x ? (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3) : blockIdx.x;
  const int at = static_cast<int>(min<int64_t>(total, static_cast<int64_t>(w) * share));
  if (blockIdx.x == 0) {
    raise_data_error(a.data_error, error | (none ? AT_GRPO_DATA_SEQLENS : 0));
    int base = first;
    for (int u = u0; u < u1; ++u) {
      const DecodeUnit x = u < kDecodeUnits ? lds.cache[u] : decode_unit(kv, lds, u, group_sizes(kv, u), &error);
      const int tiles = tiles_of(x.ntok, a.share, R), c = decode_cost(x, a, max(1, tiles));
      a.units[u] = make_int4(base, c, x.tok0, x.ntok);
      base += tiles * c * kv.Hk;
    }
    if (none)
      for (int u = tid; u < n; u += 256) a.units[u] = make_int4(0, 0, 0, 0);
    if (tid == 0) a.units[n] = make_int4(share, total, none, 0);
  }
  if (at < total && first <= at && at - first < mine) {
    int base = first, u = u0;
    for (;; ++u) {
      const DecodeUnit x = u < kDecodeUnits ? lds.cache[u] : decode_unit(kv, lds, u, group_sizes(kv, u), &error);
      const int tiles = tiles_of(x.ntok, a.share, R), c = tiles * decode_cost(x, a, max(1, tiles)) * kv.Hk;
      if (at < base + c) break;
      base += c;
    }
    lds.unit = u;
    lds.base = base;
  }
  __syncthreads();
  return Share{w, at, min(total, at + share)};
}

template <typename T, int D, int NR, bool EXACT, bool TREE>
__global__ __launch_bounds__(256, (kPerUnit<D, NR>)) void k_decode(KvView kv, Args a) {
  typedef Shape<T, D> Z;
  constexpr int E = Z::E, NB = Z::NB, KC = Z::KC, SUB = Z::SUB, TOK = Z::TOK, VJ = 4 * SUB, R = 16 * NR;
  __shared__ DecodeLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
  const int dim = EXACT ? D : kv.D;
  const Share mine = decode_schedule<R>(kv, a, lds);
  if (mine.at >= mine.stop) return;
  const uint32_t page_step = static_cast<uint32_t>(kv.Hk * dim) << kv.page_shift;
  const int in_page = (1 << kv.page_shift) - 1;
  const float to_log2 = a.scale * kLog2e;
  const int64_t queries = static_cast<int64_t>(a.n_tok) * a.Hq;
  int at = mine.at, un = __builtin_amdgcn_readfirstlane(lds.unit), base = __builtin_amdgcn_readfirstlane(lds.base);

  for (; at < mine.stop; ++un) {
    int error = 0;
    DecodeUnit u = un < kDecodeUnits ? lds.cache[un] : decode_unit(kv, lds, un, group_sizes(kv, un), &error);
    u.tok0 = __builtin_amdgcn_readfirstlane(u.tok0);
    u.ntok = __builtin_amdgcn_readfirstlane(u.ntok);
    u.seq0 = __builtin_amdgcn_readfirstlane(u.seq0);
    u.seq1 = __builtin_amdgcn_readfirstlane(u.seq1);
    u.prefix = __builtin_amdgcn_readfirstlane(u.prefix);
    u.blocks = __builtin_amdgcn_readfirstlane(u.blocks);
    const int rows = u.ntok * a.share, tiles = tiles_of(u.ntok, a.share, R), cost = decode_cost(u, a, max(1, tiles)), unit_stop = min(mine.stop, base + tiles * cost * kv.Hk);
    const int32_t* const prefix_table = kv.prefix_pages + static_cast<int64_t>(un) * kv.max_prefix_pages;      // of a group
    while (at < unit_stop) {
      const int run = (at - base) / cost, run0 = base + run * cost, stop = min(unit_stop, run0 + cost), hk = run / tiles, r0 = (run - hk * tiles) * R;
      const bool first_part = at == run0, whole = first_part && stop == run0 + cost;
      // the sequences of the tile's rows
      int seq0 = u.seq0, seq1 = u.seq1;
      if (tiles > 1) {
        const int t0 = u.tok0 + r0 / a.by_share, t1 = u.tok0 + (min(rows, r0 + R) - 1) / a.by_share;
        seq0 = kv.cu_q ? __builtin_amdgcn_readfirstlane(wave_upper_bound(kv.cu_q, kv.n_seq + 1, t0)) - 1 : t0;
        seq1 = (kv.cu_q ? __builtin_amdgcn_readfirstlane(wave_upper_bound(kv.cu_q, kv.n_seq + 1, t1)) - 1 : t1) + 1;
      }
      const int own0 = (u.prefix + 31) & ~31, block0 = __builtin_amdgcn_readfirstlane(blocks_before(lds, seq0));
      const int end = own0 + 32 * (__builtin_amdgcn_readfirstlane(blocks_before(lds, seq1)) - block0), k0 = cut(at - run0, cost, end), k1 = cut(stop - run0, cost, end);
      at = stop;
      // the sequence whose block stands at place t of the stream: the last that begins there or in front of it
      auto seq_at = [&](int t) {
        const int y = ((t - own0) >> 5) + block0;
        int s = seq0 - 1;
        for (int i = seq0; i < seq1; i += 64) s += __popcll(__ballot(i + lane < seq1 && blocks_before(lds, min(i + lane, seq1)) <= y));
        return __builtin_amdgcn_readfirstlane(s);
      };
      auto begin_of = [&](int s) { return own0 + 32 * (__builtin_amdgcn_readfirstlane(blocks_before(lds, s)) - block0); };

      // Page ids of this part of the stream: those of the prefix, then those of its sequences, the first from `skip` on.
      const int page0 = k0 >> kv.page_shift, prefix_slots = k0 < u.prefix && k0 < k1 ? ((min(k1, u.prefix) - 1) >> kv.page_shift) - page0 + 1 : 0;
      int s0 = seq0, s1 = seq0, skip = 0, slots = prefix_slots;
      if (k1 > own0 && k0 < k1) {
        s0 = seq_at(max(k0, own0));
        s1 = seq_at(k1 - 32) + 1;
        skip = max(0, k0 - begin_of(s0)) >> kv.page_shift;
        slots += __builtin_amdgcn_readfirstlane(lds.pages_before[s1] - lds.pages_before[s0]) - skip;
      }
      const bool listed = slots <= kDecodeSlots;
      auto slot0_of = [&](int s) { return prefix_slots + __builtin_amdgcn_readfirstlane(lds.pages_before[s] - lds.pages_before[s0]) - skip; };
      lds_barrier();      // the last run has read its list and what was added up
      bool missing = false;
      if (listed) {
        auto put = [&](int slot, int id) {
          const bool none = static_cast<unsigned>(id) >= static_cast<unsigned>(kv.n_pages);
          lds.pages[slot] = none ? -1 : id;
          missing |= none;
        };
        for (int i = tid; i < prefix_slots; i += 256) put(i, prefix_table[page0 + i]);
        for (int s = s0 + wave; s < s1; s += 4) {
          const int from = s == s0 ? skip : 0, count = __builtin_amdgcn_readfirstlane(lds.pages_before[s + 1] - lds.pages_before[s]), slot0 = slot0_of(s);
          for (int i = from + lane; i < count; i += 64) put(slot0 + i, kv.pages[static_cast<int64_t>(s) * kv.max_pages + i]);
        }
      } else {      // every tile's are looked at as if one were missing
        missing = true;
      }
      if (missing && listed) raise_data_error(a.data_error, AT_GRPO_DATA_PAGE);
      const bool any = __any(missing);
      if (lane == 0) lds.holes[wave] = any;

      typename Z::KV q[NR][KC], k[SUB][KC];
      typename Z::VV v[NB][VJ];
      int row_tok[NR];
      uint64_t path[TREE ? NR : 1];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int r = min(r0 + 16 * n + m, rows - 1), tq = r / a.by_share, h = hk * a.share + r - tq * a.share;
        const T* from = static_cast<const T*>(a.q.data) + (u.tok0 + tq) * a.q.ts + h * a.q.hs;
        row_tok[n] = u.tok0 + tq;
        if constexpr (TREE) path[n] = a.ancestors[u.tok0 + tq];
#pragma unroll
        for (int x = 0; x < KC; ++x) {
          const int d = 4 * Z::KE * x + Z::KE * g;
          typename Z::KV z{};
          if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::KV*>(from + d);
          q[n][x] = z;
        }
      }
      lds_barrier();
      asm volatile("" ::: "memory");
      const bool holes = (lds.holes[0] | lds.holes[1] | lds.holes[2] | lds.holes[3]) != 0;

      // A tile of the stream: tokens token .. of a sequence (or of the prefix: -1), of which there are `last`; where its page ids are listed.
      struct Tile {
        int seq, token, last, slot0;
        int q0, q1;      // the sequence's queries
      };
      auto tile_at = [&](int t) {
        Tile x{-1, t, u.prefix, -page0, 0, 0};
        if (t >= own0) {
          x.seq = seq_at(t);
          x.q0 = kv.cu_q ? kv.cu_q[x.seq] : x.seq;
          x.q1 = kv.cu_q ? kv.cu_q[x.seq + 1] : x.seq + 1;
          x.token = t - begin_of(x.seq);
          x.last = __builtin_amdgcn_readfirstlane(length_of(lds, x.seq));
          x.slot0 = slot0_of(x.seq);
        }
        return x;
      };
      auto id_of = [&](const Tile& x, int token) {      // negative: none
        const int page = token >> kv.page_shift;
        if (listed) return lds.pages[x.slot0 + page];
        const int id = x.seq < 0 ? prefix_table[page] : kv.pages[static_cast<int64_t>(x.seq) * kv.max_pages + page];
        const bool none = static_cast<unsigned>(id) >= static_cast<unsigned>(kv.n_pages);
        if (none) raise_data_error(a.data_error, AT_GRPO_DATA_PAGE);
        return none ? -1 : id;
      };
      auto row_of = [&](const Tile& x, int token) {
        return static_cast<uint64_t>(static_cast<uint32_t>(max(0, id_of(x, token)))) * page_step + static_cast<uint32_t>((token & in_page) * dim);
      };
      const T* const kbase = static_cast<const T*>(kv.k) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
      const T* const vbase = static_cast<const T*>(kv.v) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
      auto load_k = [&](const Tile& tile) {      // a token behind the last stands for it
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
          const T* p = kbase + row_of(tile, min(tile.token + 16 * s + m, tile.last - 1));
#pragma unroll
          for (int x = 0; x < KC; ++x) {
            const int d = 4 * Z::KE * x + Z::KE * g;
            typename Z::KV z{};
            if (EXACT || d < dim) z = load_once<typename Z::KV>(p + d);
            k[s][x] = z;
          }
        }
      };
      auto load_v = [&](const Tile& tile) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
          const T* p = vbase + row_of(tile, min(tile.token + 16 * s + 4 * g, (tile.last - 1) & ~3));
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int d = 16 * E * b + E * m;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              typename Z::VV z{};
              if (EXACT || d < dim) z = load_once<typename Z::VV>(p + static_cast<int64_t>(j) * dim + d);
              v[b][4 * s + j] = z;
            }
          }
        }
      };

      f32x4 acc[NR][NB][E];
      float top[NR], sum[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[n][b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      int t = k0 + TOK * wave;
      if (t < k1) {
        Tile tile = tile_at(t);
        load_k(tile);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load_v(tile);
        for (;;) {      // loads are not behind a branch (see k_attend): behind the last tile it is the one that is asked for again
          const bool more = t + 4 * TOK < k1;
          const Tile next = more ? tile_at(t + 4 * TOK) : tile;
          f32x4 s[NR][SUB];
          scores<T, D>(k, q, s);
          load_k(next);
          int left[NR];
          uint32_t sees[TREE ? NR : 1];      // of the tile's tokens
          if (tile.seq >= 0 || tile.token + TOK > tile.last || holes) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              left[n] = tile.last - tile.token;
              if constexpr (TREE) sees[n] = ~0u;
            }
            if (tile.seq >= 0) {
              const int q0 = tile.q0, q1 = tile.q1;
#pragma unroll
              for (int n = 0; n < NR; ++n) {
                const bool of_it = row_tok[n] >= q0 && row_tok[n] < q1;
                if constexpr (TREE) sees[n] = of_it ? static_cast<uint32_t>(tree_bits(path[n], tile.token - (tile.last - (q1 - q0)))) : 0u;
                else left[n] = of_it ? left[n] - (a.causal ? q1 - 1 - row_tok[n] : 0) : 0;
              }
              if (TREE && q1 - q0 > kMostTree) raise_data_error(a.data_error, AT_GRPO_DATA_TREE);
            }
#pragma unroll
            for (int y = 0; y < SUB; ++y) {
              const int at = 16 * y + 4 * g, t4 = tile.token + at, last = tile.last - t4;
              const int seen = last > 0 && id_of(tile, min(t4, tile.last - 1)) >= 0 ? last : 0;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                  bool on = i < min(seen, left[n] - at);
                  if constexpr (TREE) on = on && (sees[n] >> (at + i) & 1);
                  s[n][y][i] = on ? s[n][y][i] : -INFINITY;
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) v[b][4 * y + i] = i < seen ? v[b][4 * y + i] : typename Z::VV{};
              }
            }
          }
          weigh_and_add<T, D, TREE>(v, s, to_log2, acc, top, sum, [&] {
            // the one new token of a unit sees its stream whole: that of its sequence alone (in a tree itself only where its bit says so)
            if (tile.seq >= 0 && (TREE || u.ntok > 1))
              set_apart<T, D>(lds.slab[wave][0], v, acc, [&](int n, int token) {
                if constexpr (TREE) return token < left[n] && (sees[n] >> token & 1);
                else return token < left[n];
              });
          });
          load_v(next);
          asm volatile("" ::: "memory");
          if (!more) break;
          tile = next;
          t += 4 * TOK;
        }
      }
      finish<T, EXACT>(a, lds, acc, top, sum, RowsOf{u.tok0, hk, r0, rows}, whole, first_part ? -1 : mine.number, 0, queries, dim);
    }
    base += tiles * cost * kv.Hk;
  }
}

// ---- many queries ----------------------------------------------------------------------------------
// Where a tile has 128 rows the products bound the call, not the tokens' passage.  Each wavefront then has 32 rows of its own, and the
// four read the same 64 tokens from LDS, into which they come by direct loads, one tile ahead.  MFMA 32x32: a lane has 16 tokens of one
// query in S^T, which are P^T's operand as they are, and V^T's operand comes from rows of V by transposing reads.  Eight prompts of 763 to
// 2048 tokens, 16 heads on 8 of 128: 88 us and 16 for joining what was cut, 600 TFLOP/s in the kernel; a large product makes 1216.  Eight of
// 2000 tokens, 16 heads on 4 of 256: 704 us whole, 370 TFLOP/s (by k_attend 1640); on 8 of 96: 331 (576).
//
// A token's row is 2 D bytes in LDS; its 16-byte pieces are exchanged so that the reads meet no bank twice: piece c of K's row r lies at
// c ^ (r & 15) (64-wide heads, whose rows take turns in the banks' halves: c ^ ((r >> 1) & 7)), of V's at c ^ 2 (r & 7) (c ^ 2 ((r >> 1) & 3)).
constexpr int kWideTok = 64;

struct WideLds {
  Schedule S;
  int not_finite[4];
  int pages[kPageSlots];
};

// Workgroups on a compute unit: heads of 256 take 128 KB of LDS.
template <int D>
constexpr int kWidePerUnit = D == 256 ? 1 : 2;

template <int D>
__device__ __forceinline__ int swizzle_k(int r) { return D >= 128 ? r & 15 : (r >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swizzle_v(int r) { return D >= 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }

template <int D, bool EXACT, bool TREE>
__global__ __launch_bounds__(256, kWidePerUnit<D>) void k_attend_wide(KvView kv, Args a) {
  constexpr int KC = D / 16, DT = D / 32, TB = kWideTok * D * 2, NL = TB / 4096, PIECES = D / 8, LROWS = 64 / PIECES, VG = DT > 4 ? 2 : 1, DB = DT / VG;
  extern __shared__ __attribute__((aligned(1024))) char smem[];      // two tiles of keys and values, then the rest
  WideLds& lds = *reinterpret_cast<WideLds*>(smem + 4 * TB);
  const int dim = EXACT ? D : kv.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 31, g = lane >> 5;
  const Share mine = make_schedule<kWideRows>(kv, a, lds.S);
  Runs<kWideRows> run(kv, a, lds.S, mine);
  if (!run.valid()) return;
  if (!EXACT) {      // what no load writes: the elements behind a head's last count as 0
    for (int i = tid; i < 4 * TB / 16; i += 256) *reinterpret_cast<uint4*>(smem + i * 16) = make_uint4(0, 0, 0, 0);
    lds_barrier();
    asm volatile("" ::: "memory");
  }

  // where this lane reads: K piece 2 c + g of row m (XOR 32 c), V four elements of row 4 g + (lane & 15) / 4 (XOR 64 t)
  const int read_k = m * (2 * D) + ((g ^ swizzle_k<D>(m)) << 4);
  const int i16 = lane & 15, row_v = 4 * g + (i16 >> 2);
  const int read_v = row_v * (2 * D) + (((2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1)) ^ swizzle_v<D>(row_v)) << 4) + (i16 & 1) * 8;
  const float to_log2 = a.scale * kLog2e;
  const uint32_t page_bytes = (static_cast<uint32_t>(kv.Hk) * dim * 2) << kv.page_shift;      // of all heads
  const int in_page = (1 << kv.page_shift) - 1;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr32(smem)) + wave * NL * 1024;

  // Page ids of tokens page0 << page_shift .. in LDS: a unit's all, where they fit, for all its runs.
  int page0 = 0, staged = -1;
  bool holes = false;
  auto stage = [&](const int32_t* table, int first_token, int to) {
    page0 = first_token >> kv.page_shift;
    const int n_slots = to > first_token ? ((to - 1) >> kv.page_shift) - page0 + 1 : 0;
    bool missing = false;
    lds_barrier();
    for (int i = tid; i < n_slots; i += 256) {
      int id = table[page0 + i];
      if (static_cast<unsigned>(id) >= static_cast<unsigned>(kv.n_pages)) {
        id = -1;
        missing = true;
      }
      lds.pages[i] = id;
    }
    if (missing) raise_data_error(a.data_error, AT_GRPO_DATA_PAGE);
    holes = __syncthreads_or(missing);
  };
  // A tile of tokens t .. into a buffer; rows behind the last token are the last.
  auto request = [&](int hk, int t, int to, int buffer) {
    const char* const kbase = static_cast<const char*>(kv.k) + ((static_cast<int64_t>(hk) * dim * 2) << kv.page_shift);
    const char* const vbase = static_cast<const char*>(kv.v) + ((static_cast<int64_t>(hk) * dim * 2) << kv.page_shift);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = (wave * NL + i) * LROWS + lane / PIECES, piece = lane & (PIECES - 1), token = min(t + row, to - 1);
      const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(max(0, lds.pages[(token >> kv.page_shift) - page0]))) * page_bytes;
      const uint32_t in = static_cast<uint32_t>(token & in_page) * (2 * dim);
      const int of_k = piece ^ swizzle_k<D>(row), of_v = piece ^ swizzle_v<D>(row);
      if (EXACT || 8 * of_k < dim) direct_load_v(kbase + (at + (in + 16 * of_k)), lds0 + buffer * 2 * TB + i * 1024);
      if (EXACT || 8 * of_v < dim) direct_load_v(vbase + (at + (in + 16 * of_v)), lds0 + buffer * 2 * TB + TB + i * 1024);
    }
  };
  uint4 q[KC];
  auto load_q = [&](const Unit& x, const TileRun& w) {
    const int r = min(w.r0 + 32 * wave + m, x.ntok * a.share - 1), tq = r / a.by_share, h = w.hk * a.share + r - tq * a.share;
    const bf16_t* from = static_cast<const bf16_t*>(a.q.data) + (x.tok0 + tq) * a.q.ts + h * a.q.hs + 8 * g;
#pragma unroll
    for (int c = 0; c < KC; ++c) q[c] = EXACT || 16 * c + 8 * g < dim ? *reinterpret_cast<const uint4*>(from + 16 * c) : make_uint4(0, 0, 0, 0);
  };
  int buffer = 0;
  bool requested = false;      // the run's first tile, by the run in front of it
  TileRun w = tile_run(run, a);
  load_q(run.x, w);
  for (;;) {
    const Unit u = run.x;
    const bool steps = run.steps, own = run.own, fits = ((u.len - 1) >> kv.page_shift) < kPageSlots;
    const int rows = u.ntok * a.share;
    const int first = u.len - u.ntok + 1, k1 = w.k1;      // a causal query sees the own tokens in front of `first + its number among the new tokens`
    // What is needed at a run's end alone, or for few tiles, is computed there: the loop has no register left.
    auto token_of = [&] { return min(w.r0 + 32 * wave + m, rows - 1) / a.by_share; };
    const int limit = steps ? min(k1, first + token_of()) : k1;
    // a first row sees least: the tile's, and the wavefront's; in a tree, what is in front of it
    const bool tree = TREE && own;
    const int all_see = tree ? first - 1 : steps ? first + w.r0 / a.by_share : k1;
    const int wave_sees = tree ? first - 1 : steps ? first + min(w.r0 + 32 * wave, rows - 1) / a.by_share : k1;
    if (tree && u.ntok > kMostTree) raise_data_error(a.data_error, AT_GRPO_DATA_TREE);
    const bool direct = kv.n_group == 0 && run.from() == 0 && run.to() == run.cost, first_part = run.from() == 0;
    const int group = run.number;
    const int32_t* const table = own ? kv.pages + static_cast<int64_t>(u.row) * kv.max_pages : kv.prefix_pages + static_cast<int64_t>(u.row) * kv.max_prefix_pages;
    if (fits && staged != run.u) {
      stage(table, 0, u.len);
      staged = run.u;
    }
    run.next();
    const bool more = run.valid();
    TileRun next{};
    if (more) next = tile_run(run, a);
    const bool ahead = more && run.u == staged && next.k0 < next.k1;      // with the same page ids
    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
    float top = -INFINITY, sum = 0.f;
    const bool idle = TREE && w.r0 + 32 * wave >= rows;      // no rows: it loads and waits with the others

    for (int from = w.k0; from < k1;) {
      int to = k1;
      if (!fits) {
        to = min(k1, ((from >> kv.page_shift) + kPageSlots) << kv.page_shift);
        stage(table, from, to);
        staged = -1;
      }
      if (!requested) request(w.hk, from, to, buffer);
      requested = false;
      for (int t = from; t < to; t += kWideTok, buffer ^= 1) {
        asm volatile("" ::: "memory");
        wait_loads_but<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // The next tile, or the next run's first: its buffer is free, since who has passed this barrier has read the tile in front.  Asked for in one
        // place: in two it takes 12 registers more (trees, heads of 128: 116 bytes of them in memory and not 28).
        const bool inside = t + kWideTok < to;
        if (inside || (ahead && to == k1)) request(inside ? w.hk : next.hk, inside ? t + kWideTok : next.k0, inside ? to : next.k1, buffer ^ 1);
        uint64_t path = 0;
        if constexpr (TREE)
          if (tree && t + kWideTok > all_see) path = a.ancestors[u.tok0 + token_of()];
        const char* const kt = smem + buffer * 2 * TB;
        char* const vt = smem + buffer * 2 * TB + TB;
        if (holes || t + kWideTok > to) {      // what stands for a token behind the last or of no page counts as 0
          for (int i = tid; i < kWideTok * PIECES; i += 256) {
            const int token = t + i / PIECES;
            if (token >= to || lds.pages[(token >> kv.page_shift) - page0] < 0) *reinterpret_cast<uint4*>(vt + i * 16) = make_uint4(0, 0, 0, 0);
          }
          lds_barrier();
          asm volatile("" ::: "memory");
        }
        const bool partly = t + kWideTok > all_see;      // as in set_apart; each wavefront looks at a fourth of the values
        if (partly) {
          uint32_t high = 0;
#pragma unroll
          for (int i = 0; i < kWideTok * PIECES / 256; ++i) high = largest_bits(high, *reinterpret_cast<const uint4*>(vt + (tid + 256 * i) * 16));
          const bool any = __any(not_finite<bf16_t>(high));
          if (lane == 0) lds.not_finite[wave] = any;
        }
        f32x16 s[2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
        // Fragments are read a group ahead of the products that take them: left to itself the compiler reads each right in front of its own,
        // and every product waits for LDS (103 us for eight prompts of up to 2048 tokens, then 90).
        bf16x8 f[2][4];
        auto read_k_group = [&](int x) {      // two steps of 16 elements, two blocks of 32 tokens
#pragma unroll
          for (int i = 0; i < 4; ++i) f[x & 1][i] = *reinterpret_cast<const bf16x8*>(kt + (read_k ^ ((2 * x + (i >> 1)) << 5)) + (i & 1) * 32 * 2 * D);
        };
        if (!idle) {
          read_k_group(0);
#pragma unroll
          for (int x = 0; x < KC / 2; ++x) {
            if (x + 1 < KC / 2) read_k_group(x + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[x & 1][i], __builtin_bit_cast(bf16x8, q[2 * x + (i >> 1)]), s[i & 1], 0, 0, 0);
          }
        }
        if (more && t + kWideTok >= k1) load_q(run.x, next);      // the last scores of this run are on their way
        auto read_v_group = [&](int k) {      // 16 tokens, all blocks of 32 elements or half of them
#pragma unroll
          for (int x = 0; x < DB; ++x) {
            const char* p = vt + (read_v ^ ((DB * (k % VG) + x) << 6)) + k / VG * 16 * 2 * D;
            const uint2 lo = lds_read_tr(p), hi = lds_read_tr(p + 8 * 2 * D);
            f[k & 1][x] = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
          }
        };
        if (!idle) read_v_group(0);
        uint64_t sees = ~uint64_t{0};      // of the tile's tokens
        if constexpr (TREE)
          if (tree && t + kWideTok > all_see) sees = tree_bits(path, t - (first - 1));
        if (!idle && (t + kWideTok > min(to, wave_sees) || holes)) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int b = 0; b < 4; ++b) {      // four tokens that start at a multiple of four share a page
              const int t4 = t + 32 * y + 8 * b + 4 * g;
              int left = limit - t4;
              if (holes) left = lds.pages[(min(t4, to - 1) >> kv.page_shift) - page0] < 0 ? 0 : left;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                bool on = i < left;
                if constexpr (TREE) on = on && (static_cast<uint32_t>(sees >> 32 * y) >> (8 * b + 4 * g + i) & 1);
                s[y][4 * b + i] = on ? s[y][4 * b + i] : -INFINITY;
              }
            }
        }
        float lead = 0.f;
        if (!idle) {
          float high = -INFINITY;
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; i += 2) high = maximum3(high, s[y][i], s[y][i + 1]);
          lead = top * to_log2;
          const auto keep = [&](float f) {
            sum *= f;
#pragma unroll
            for (int x = 0; x < DT; ++x) acc[x] *= f;
          };
          if (__any(high * to_log2 > lead + kSlack)) keep(raise_top<TREE>(fmaxf(high, __shfl_xor(high, 32, 64)), to_log2, top, lead));
          if (__any(is_far(top, lead))) {
            float less;
            keep(raise_far(fmaxf(high, __shfl_xor(high, 32, 64)), to_log2, top, lead, less));
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < 16; ++i) s[y][i] -= less;
          }
          lead = top == -INFINITY ? 0.f : lead;
        }
        bool apart = false;
        if (partly) {
          lds_barrier();
          asm volatile("" ::: "memory");
          apart = (lds.not_finite[0] | lds.not_finite[1] | lds.not_finite[2] | lds.not_finite[3]) != 0;
        }
        if (apart) {
#pragma unroll 1
          for (int i = 0; i < (idle ? 0 : kWideTok * PIECES); ++i) {
            const int token = i / PIECES, c = i & (PIECES - 1);      // elements 8 c ..
            const uint4 x = *reinterpret_cast<const uint4*>(vt + (token * PIECES + (c ^ swizzle_v<D>(token))) * 16);
            if (!__any(not_finite<bf16_t>(largest_bits(0u, x)))) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {      // of this lane's four
              const float y = g ? element(x, 4 + j) : element(x, j), add = not_finite(y) && t + token < limit && (!TREE || (sees >> token & 1)) ? y : 0.f;
#pragma unroll
              for (int d = 0; d < 4 * DT; ++d) acc[d >> 2][4 * (d & 3) + j] += d == c ? add : 0.f;
            }
          }
          lds_barrier();
          for (int i = tid; i < kWideTok * PIECES; i += 256) {
            uint4* const piece = reinterpret_cast<uint4*>(vt + i * 16);
            *piece = finite_of(*piece);
          }
          lds_barrier();
          asm volatile("" ::: "memory");
          if (!idle) read_v_group(0);
        }
        if (!idle) {
          uint4 w[2];
          auto weigh = [&](int ks) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              p[j] = __builtin_amdgcn_exp2f(fmaf(s[ks >> 1][8 * (ks & 1) + j], to_log2, -lead));
              sum += p[j];
            }
            w[ks & 1] = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
          };
          weigh(0);
#pragma unroll
          for (int k = 0; k < 4 * VG; ++k) {
            const int ks = k / VG;
            __builtin_amdgcn_sched_barrier(0);
            const bool weighing = k % VG == 0 && ks < 3;
            if (k + 1 < 4 * VG) read_v_group(k + 1);
            if (weighing) weigh(ks + 1);      // the next tokens' weights are computed between this step's products
#pragma unroll
            for (int x = 0; x < DB; ++x)
              acc[DB * (k % VG) + x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[k & 1][x], __builtin_bit_cast(bf16x8, w[ks & 1]), acc[DB * (k % VG) + x], 0, 0, 0);
            if (weighing) {
              __builtin_amdgcn_sched_group_barrier(0x100, 2 * DB, 0);      // LDS reads, then a product and some of the weights in turn
#pragma unroll
              for (int x = 0; x < DB; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x402, 28 / DB, 0);
              }
            }
          }
        }
      }
      from = to;
    }

    sum += __shfl_xor(sum, 32, 64);
    const int r = w.r0 + 32 * wave + m;
    if (r < rows) {
      const int tq = token_of(), h = w.hk * a.share + r - tq * a.share;
      const float f = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum), x = sum == 0.f ? -INFINITY : (top_log2(top, to_log2) + __builtin_amdgcn_logf(sum)) * kLn2;
      const int64_t by_query = static_cast<int64_t>(own && kv.n_group ? a.n_tok : 0) * a.Hq + static_cast<int64_t>(u.tok0 + tq) * a.Hq + h;
      if (direct) {
        if (a.lse && g == 0) a.lse[by_query] = x;
        // two lanes have 8 bytes each of a row's 16: they exchange them for those of the next 16
        bf16_t* to = static_cast<bf16_t*>(a.out.data) + (u.tok0 + tq) * a.out.ts + h * a.out.hs + 8 * g;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; i += 8) {
            uint32_t p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = pack_bf16x2(acc[t][i + 2 * j] * f, acc[t][i + 2 * j + 1] * f);
            const auto lo = __builtin_amdgcn_permlane32_swap(p[0], p[2], false, false), hi = __builtin_amdgcn_permlane32_swap(p[1], p[3], false, false);
            if (EXACT || 32 * t + 2 * i + 8 * g < dim) *reinterpret_cast<uint4*>(to + 32 * t + 2 * i) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
          }
      } else {
        const int64_t part = first_part ? by_query : static_cast<int64_t>(a.n_tok) * a.Hq * (kv.n_group ? 2 : 1) + static_cast<int64_t>(group) * kMaxRows + (r - w.r0);
        if (g == 0) a.part_lse[part] = x;
        float* to = a.part_out + part * dim + 4 * g;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            if (EXACT || 32 * t + 2 * i + 4 * g < dim) *reinterpret_cast<f32x4*>(to + 32 * t + 2 * i) = f32x4{acc[t][i] * f, acc[t][i + 1] * f, acc[t][i + 2] * f, acc[t][i + 3] * f};
      }
    }
    if (!more) break;
    requested = ahead;
    if (w.k0 >= w.k1) {      // no tile, at which they were asked for
      load_q(run.x, next);
      requested = false;
    }
    w = next;
  }
}

template <typename T, int D, int NR, bool EXACT, bool TREE>
__global__ __launch_bounds__(256, (kPerUnit<D, NR>)) void k_attend(KvView kv, Args a) {
  typedef Shape<T, D> Z;
  constexpr int E = Z::E, NB = Z::NB, KC = Z::KC, SUB = Z::SUB, TOK = Z::TOK, VJ = 4 * SUB, R = 16 * NR;
  constexpr bool kBf16 = sizeof(T) == 2;
  __shared__ Lds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
  const int dim = EXACT ? D : kv.D;
  const Share mine = make_schedule<R>(kv, a, lds.S);
  Runs<R> run(kv, a, lds.S, mine);
  if (!run.valid()) return;
  const uint32_t page_step = static_cast<uint32_t>(kv.Hk * dim) << kv.page_shift;      // elements of a page of all heads
  const int in_page = (1 << kv.page_shift) - 1;
  const float to_log2 = a.scale * kLog2e;

  // Page ids of tokens page0 << page_shift .. : a unit's all, where they fit, for all its runs.  Two lists take turns, so that the next
  // unit's comes in beside a run of this one.
  const int* pages = lds.pages[0];
  int page0 = 0, staged = -1, half = 0;
  bool holes = false;
  auto slots = [&](int from, int to) { return to > from ? ((to - 1) >> kv.page_shift) - (from >> kv.page_shift) + 1 : 0; };
  auto put_ids = [&](const int* ids, int n, int at) {      // ids[i]: of slot tid + 256 i; whether one is none, and all lists have been read
    bool missing = false;
#pragma unroll
    for (int i = 0; i < kPageSlots / 256; ++i)
      if (tid + 256 * i < n) {
        const bool none = static_cast<unsigned>(ids[i]) >= static_cast<unsigned>(kv.n_pages);
        lds.pages[at][tid + 256 * i] = none ? -1 : ids[i];
        missing |= none;
      }
    if (missing) raise_data_error(a.data_error, AT_GRPO_DATA_PAGE);
    const bool any = __any(missing);
    if (lane == 0) lds.holes[at][wave] = any;
    lds_barrier();
    asm volatile("" ::: "memory");
    return (lds.holes[at][0] | lds.holes[at][1] | lds.holes[at][2] | lds.holes[at][3]) != 0;
  };
  auto get_ids = [&](int* ids, const int32_t* table, int n) {
#pragma unroll
    for (int i = 0; i < kPageSlots / 256; ++i) ids[i] = tid + 256 * i < n ? table[tid + 256 * i] : 0;
  };
  auto table_of = [&](const Unit& x, bool own) {
    return own ? kv.pages + static_cast<int64_t>(x.row) * kv.max_pages : kv.prefix_pages + static_cast<int64_t>(x.row) * kv.max_prefix_pages;
  };
  auto fits = [&](const Unit& x) { return ((x.len - 1) >> kv.page_shift) < kPageSlots; };

  typename Z::KV q[NR][KC], k[SUB][KC];
  typename Z::VV v[NB][VJ];
  auto row_of = [&](int token, int to) {      // a token behind the last stands for it
    const int i = min(token, to - 1), id = max(0, pages[(i >> kv.page_shift) - page0]);
    return static_cast<uint64_t>(static_cast<uint32_t>(id)) * page_step + static_cast<uint32_t>((i & in_page) * dim);
  };
  auto load_k = [&](int hk, int t, int to) {
    const T* const base = static_cast<const T*>(kv.k) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
      const T* p = base + row_of(t + 16 * s + m, to);
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        const int d = 4 * Z::KE * x + Z::KE * g;
        typename Z::KV z{};
        if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::KV*>(p + d);
        k[s][x] = z;
      }
    }
  };
  auto load_v = [&](int hk, int t, int to) {
    const T* const base = static_cast<const T*>(kv.v) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
      const T* p = base + row_of(min(t + 16 * s + 4 * g, (to - 1) & ~3), to);      // four tokens that start at a multiple of four share a page
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int d = 16 * E * b + E * m;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typename Z::VV z{};
          if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::VV*>(p + static_cast<int64_t>(j) * dim + d);
          v[b][4 * s + j] = z;
        }
      }
    }
  };
  auto load_q = [&](const Unit& u, const TileRun& w) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = min(w.r0 + 16 * n + m, u.ntok * a.share - 1), tq = r / a.by_share, h = w.hk * a.share + r - tq * a.share;
      const T* from = static_cast<const T*>(a.q.data) + (u.tok0 + tq) * a.q.ts + h * a.q.hs;
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        const int d = 4 * Z::KE * x + Z::KE * g;
        typename Z::KV z{};
        if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::KV*>(from + d);
        q[n][x] = z;
      }
    }
  };

  TileRun w = tile_run(run, a);
  for (;;) {
    const Unit u = run.x;
    const bool steps = run.steps, own = run.own, whole = fits(u), first_part = run.from() == 0;
    const bool direct = kv.n_group == 0 && first_part && run.to() == run.cost;
    const int32_t* const table = table_of(u, own);
    if (whole && staged != run.u) {
      int ids[kPageSlots / 256];
      get_ids(ids, table, slots(0, u.len));
      lds_barrier();      // nobody reads the list any more
      holes = put_ids(ids, slots(0, u.len), half);
      pages = lds.pages[half];
      page0 = 0;
      staged = run.u;
    }
    run.next();
    const bool more = run.valid();
    TileRun next{};
    if (more) next = tile_run(run, a);
    const bool turn = more && run.u != staged && fits(run.x);      // another unit: its page ids come meanwhile
    int ids[kPageSlots / 256];
    if (turn) get_ids(ids, table_of(run.x, run.own), slots(0, run.x.len));

    // Twice: where all rows see all tokens nothing is kept for each.  Messages in fp32, heads of 128: 257 us in one, 242 so.
    auto body = [&](auto in_part) {
      constexpr bool part = decltype(in_part)::value, tree = TREE && part, steps = part && !TREE;
      const int rows = u.ntok * a.share, hk = w.hk, r0 = w.r0, k0 = w.k0, k1 = w.k1, first = u.len - u.ntok + 1;
      const int all_see = tree ? first - 1 : steps ? first + r0 / a.by_share : k1;
      int limit[NR];
      uint64_t path[tree ? NR : 1];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int tq = min(r0 + 16 * n + m, rows - 1) / a.by_share;
        limit[n] = steps ? min(k1, first + tq) : k1;
        if constexpr (tree) path[n] = a.ancestors[u.tok0 + tq];
      }
      if (tree && u.ntok > kMostTree) raise_data_error(a.data_error, AT_GRPO_DATA_TREE);
      f32x4 acc[NR][NB][E];
      float top[NR], sum[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[n][b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      load_q(u, w);
      for (int from = k0; from < k1;) {
        int to = k1;
        if (!whole) {      // a part of the list at a time
          page0 = from >> kv.page_shift;
          to = min(k1, (page0 + kPageSlots) << kv.page_shift);
          int part[kPageSlots / 256];
          get_ids(part, table + page0, slots(from, to));
          lds_barrier();
          holes = put_ids(part, slots(from, to), half);
          pages = lds.pages[half];
          staged = -1;
        }
        // The order of the loads is that of their use.
        load_k(hk, from + TOK * wave, to);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load_v(hk, from + TOK * wave, to);
        // Loads are never behind a branch: the compiler could not tell then which of them are still on their way, and would wait for all.
        // What is asked for behind the last tile is the last token's row.
        for (int t = from + TOK * wave; t < to; t += 4 * TOK) {
          f32x4 s[NR][SUB];
          scores<T, D>(k, q, s);
          load_k(hk, t + 4 * TOK, to);
          uint32_t sees[tree ? NR : 1];      // of the tile's tokens
          if constexpr (tree)
#pragma unroll
            for (int n = 0; n < NR; ++n) sees[n] = static_cast<uint32_t>(tree_bits(path[n], t - (first - 1)));
          if (t + TOK > min(to, all_see) || holes) {
            // tokens that a row does not see, and what lies in the cache behind the last or in no page: no weight, and no value
#pragma unroll
            for (int y = 0; y < SUB; ++y) {
              const int t4 = t + 16 * y + 4 * g;
              const int last = to - t4, seen = last > 0 && pages[(min(t4, to - 1) >> kv.page_shift) - page0] >= 0 ? last : 0;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                  bool on = i < min(seen, limit[n] - t4);
                  if constexpr (tree) on = on && (sees[n] >> (16 * y + 4 * g + i) & 1);
                  s[n][y][i] = on ? s[n][y][i] : -INFINITY;
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) v[b][4 * y + i] = i < seen ? v[b][4 * y + i] : typename Z::VV{};
              }
            }
          }
          weigh_and_add<T, D, TREE>(v, s, to_log2, acc, top, sum, [&] {
            if (part && t + TOK > all_see)
              set_apart<T, D>(lds.slab[wave][0], v, acc, [&](int n, int token) {
                if constexpr (tree) return t + token < limit[n] && (sees[n] >> token & 1);
                else return t + token < limit[n];
              });
          });
          load_v(hk, t + 4 * TOK, to);
          asm volatile("" ::: "memory");      // the loads stay on this side of the jump back
        }
        from = to;
      }

      if (turn) {
        half ^= 1;
        holes = put_ids(ids, slots(0, run.x.len), half);
        pages = lds.pages[half];
        page0 = 0;
        staged = run.u;
      }
      const int64_t queries = static_cast<int64_t>(a.n_tok) * a.Hq;
      finish<T, EXACT>(a, lds, acc, top, sum, RowsOf{u.tok0, hk, r0, rows}, direct, first_part ? -1 : run.number, own && kv.n_group ? queries : 0,
                       queries * (kv.n_group ? 2 : 1), dim);
    };
    if (TREE ? own : steps) body(std::true_type{});
    else body(std::false_type{});
    if (!more) break;
    lds_barrier();      // what was added up has been read
    w = next;
  }
}

// ---- joining the parts --------------------------------------------------------------------------------
// out = sum_p exp(lse_p - lse) out_p over the parts of a row.

__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }      // NaN stays

template <typename T>
__device__ __forceinline__ void store8(T* to, const float* y) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
  } else {
    *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]};
    *reinterpret_cast<f32x4*>(to + 4) = f32x4{y[4], y[5], y[6], y[7]};
  }
}

// One row of n parts, by sixteen lanes, eight elements a lane, or where `spread` by a whole wavefront, every fourth part each; by all wavefront's lanes.
template <typename T, typename PartOf>
__device__ __forceinline__ void join_row(const Args& a, int D, int n, bool spread, bool write, PartOf part_of, T* to, float* lse) {
  const int lane = threadIdx.x & 63, l = lane & 15, slot = spread ? lane >> 4 : 0, slots = spread ? 4 : 1;
  float high = -INFINITY;
  for (int p = slot * 16 + l; p < n; p += 16 * slots) high = larger(high, a.part_lse[part_of(p)]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    if (o < 16 * slots) high = larger(high, __shfl_xor(high, o, 64));
  const float ref = high == -INFINITY ? 0.f : high;
  float total = 0.f, acc[kMaxHeadDim / 16] = {};
  for (int p0 = 0; p0 < n; p0 += 2 * slots) {      // two in flight
    float weight[2];
    f32x4 y[2][kMaxHeadDim / 64];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int p = p0 + c * slots + slot;
      const int64_t part = part_of(min(p, n - 1));
      weight[c] = p < n ? a.part_lse[part] : -INFINITY;
#pragma unroll
      for (int x = 0; x < kMaxHeadDim / 128; ++x)
        if (128 * x + 8 * l < D) {
          y[c][2 * x] = *reinterpret_cast<const f32x4*>(a.part_out + part * D + 128 * x + 8 * l);
          y[c][2 * x + 1] = *reinterpret_cast<const f32x4*>(a.part_out + part * D + 128 * x + 8 * l + 4);
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float f = __builtin_amdgcn_exp2f((weight[c] - ref) * kLog2e);
      const bool there = p0 + c * slots + slot < n;      // behind the last not 0 times an infinity of that
      total += f;
#pragma unroll
      for (int x = 0; x < kMaxHeadDim / 128; ++x)
        if (128 * x + 8 * l < D)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[8 * x + e] = fmaf(f, there ? y[c][2 * x + (e >> 2)][e & 3] : 0.f, acc[8 * x + e]);
    }
  }
  if (spread) {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      total += __shfl_xor(total, o, 64);
#pragma unroll
      for (int e = 0; e < kMaxHeadDim / 16; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    }
  }
  if (slot || !write) return;
  const float f = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int e = 0; e < kMaxHeadDim / 16; ++e) acc[e] *= f;
#pragma unroll
  for (int x = 0; x < kMaxHeadDim / 128; ++x)
    if (128 * x + 8 * l < D) store8(to + 128 * x + 8 * l, acc + 8 * x);
  if (lse && l == 0) *lse = total == 0.f ? -INFINITY : high + logf(total);
}

// The units of a token: its group's prefix, and its sequence.
struct UnitsOf {
  int4 prefix, own;
  int share;
};
__device__ __forceinline__ UnitsOf units_of(const KvView& kv, const Args& a, int t) {
  const int s = kv.cu_q ? wave_upper_bound(kv.cu_q, kv.n_seq + 1, t) - 1 : t, g = wave_upper_bound(kv.group_seq, kv.n_group + 1, s) - 1;
  const bool in_seq = s >= 0 && s < kv.n_seq, in_group = in_seq && g >= 0 && g < kv.n_group;
  return UnitsOf{in_group ? a.units[g] : make_int4(0, 0, 0, 0), in_seq ? a.units[kv.n_group + s] : make_int4(0, 0, 0, 0), a.units[kv.n_group + kv.n_seq].x};
}

// The parts of row (t, h): of the prefix, then of its sequence.
struct RowParts {
  int group0[2], count[2], row[2];      // the run's first workgroup, its workgroups, the row in its tile
  int64_t queries, unit;

  __device__ __forceinline__ RowParts(const Args& a, const UnitsOf& units, int t, int h, int tile_rows)
      : queries(static_cast<int64_t>(a.n_tok) * a.Hq), unit(static_cast<int64_t>(t) * a.Hq + h) {
    look_up(0, a, units, units.prefix, false, t, h, tile_rows);
    look_up(1, a, units, units.own, a.causal, t, h, tile_rows);
  }
  __device__ __forceinline__ int parts() const { return count[0] + count[1]; }
  __device__ __forceinline__ int64_t operator()(int p) const {
    const bool own = p >= count[0];
    const int i = own ? p - count[0] : p;
    return i == 0 ? (own ? queries : 0) + unit : 2 * queries + static_cast<int64_t>((own ? group0[1] : group0[0]) + i) * kMaxRows + (own ? row[1] : row[0]);
  }

 private:
  __device__ __forceinline__ void look_up(int which, const Args& a, const UnitsOf& units, const int4& x, bool steps, int t, int h, int rows) {
    group0[which] = count[which] = row[which] = 0;
    const int q = t - x.z, hk = h / a.by_share;
    if (x.y == 0 || q < 0 || q >= x.w) return;
    const Unit of{x.z, x.w, x.y, 0};
    const int r = q * a.share + h - hk * a.share, tile = r / rows;
    const Cost costs = cost_of(of, steps, a, rows);
    const int run0 = x.x + hk * head_cost(of, steps, a, rows) + costs.in_front(tile), run1 = run0 + costs.of(tile);
    group0[which] = run0 / units.share;
    count[which] = (run1 - 1) / units.share - group0[which] + 1;
    row[which] = r - tile * rows;
  }
};

// Rows behind prefixes: a wavefront for four heads of a token, so that what belongs to the token is looked up once.  3840 tokens of 32 heads of 128
// 50 us; a wavefront for each row 111.
template <typename T>
__global__ __launch_bounds__(256) void k_join_heads(KvView kv, Args a, int tile_rows, int heads) {
  const int lane = threadIdx.x & 63, per_token = (a.Hq + heads - 1) / heads;
  const int64_t unit = static_cast<int64_t>(flat_block()) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= static_cast<int64_t>(a.n_tok) * per_token) return;
  const int t = static_cast<int>(unit / per_token), h0 = heads * static_cast<int>(unit - static_cast<int64_t>(t) * per_token);
  const UnitsOf units = units_of(kv, a, t);
  if (heads == 1) {
    const RowParts of(a, units, t, h0, tile_rows);
    join_row(a, kv.D, of.parts(), true, true, of, static_cast<T*>(a.out.data) + t * a.out.ts + h0 * a.out.hs, a.lse ? a.lse + of.unit : nullptr);
    return;
  }
  const RowParts of_slot(a, units, t, min(h0 + (lane >> 4), a.Hq - 1), tile_rows);
  T* const to = static_cast<T*>(a.out.data) + t * a.out.ts;
  if (!__any(of_slot.parts() > 8)) {
    const int h = h0 + (lane >> 4);
    join_row(a, kv.D, of_slot.parts(), false, h < a.Hq, of_slot, to + h * a.out.hs, a.lse ? a.lse + of_slot.unit : nullptr);
    return;
  }
  for (int h = h0; h < min(h0 + 4, a.Hq); ++h) {
    const RowParts of(a, units, t, h, tile_rows);
    join_row(a, kv.D, of.parts(), true, true, of, to + h * a.out.hs, a.lse ? a.lse + of.unit : nullptr);
  }
}

// The same for few rows: a workgroup for each, four parts at a time by each of its wavefronts.
template <typename T>
__global__ __launch_bounds__(256) void k_join(KvView kv, Args a, int tile_rows) {
  __shared__ float lds[4][kMaxHeadDim + 1];
  const int lane = threadIdx.x & 63, l = lane & 15, slot = lane >> 4, wave = threadIdx.x >> 6, D = kv.D;
  const int64_t unit = blockIdx.x;
  const int t = static_cast<int>(unit / a.Hq), h = static_cast<int>(unit - static_cast<int64_t>(t) * a.Hq);
  const RowParts part_of(a, units_of(kv, a, t), t, h, tile_rows);
  const int n = part_of.parts();
  float high = -INFINITY, total = 0.f, acc[kMaxHeadDim / 16] = {};
  for (int p0 = 0; p0 < n; p0 += 64) {
    const int count_here = min(64, n - p0);
    const float x = lane < count_here ? a.part_lse[part_of(p0 + lane)] : -INFINITY;
    float now = larger(high, x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) now = larger(now, __shfl_xor(now, o, 64));
    const float ref = now == -INFINITY ? 0.f : now, keep = __builtin_amdgcn_exp2f((high - ref) * kLog2e), weight = __builtin_amdgcn_exp2f((x - ref) * kLog2e);
    high = now;
    total *= keep;
#pragma unroll
    for (int i = 0; i < kMaxHeadDim / 16; ++i) acc[i] *= keep;
    for (int c0 = 4 * wave; c0 < count_here; c0 += 16) {
      const int c = c0 + slot;
      const float w = __shfl(weight, c, 64);      // 0 behind the last
      const float* from = a.part_out + part_of(p0 + min(c, count_here - 1)) * D;
      total += w;
#pragma unroll
      for (int x2 = 0; x2 < kMaxHeadDim / 128; ++x2) {
        const int d = 128 * x2 + 8 * l;
        if (d < D) {
          const f32x4 y0 = *reinterpret_cast<const f32x4*>(from + d), y1 = *reinterpret_cast<const f32x4*>(from + d + 4);
          const bool there = c < count_here;      // behind the last not 0 times an infinity of that
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[8 * x2 + i] = fmaf(w, there ? y0[i] : 0.f, acc[8 * x2 + i]);
            acc[8 * x2 + 4 + i] = fmaf(w, there ? y1[i] : 0.f, acc[8 * x2 + 4 + i]);
          }
        }
      }
    }
  }
  total += __shfl_xor(total, 16, 64);
  total += __shfl_xor(total, 32, 64);
#pragma unroll
  for (int i = 0; i < kMaxHeadDim / 16; ++i) {
    acc[i] += __shfl_xor(acc[i], 16, 64);
    acc[i] += __shfl_xor(acc[i], 32, 64);
  }
  if (slot == 0) {
#pragma unroll
    for (int x = 0; x < kMaxHeadDim / 128; ++x)
#pragma unroll
      for (int i = 0; i < 8; ++i) lds[wave][128 * x + 8 * l + i] = acc[8 * x + i];
    if (l == 0) lds[wave][kMaxHeadDim] = total;
  }
  __syncthreads();
  if (wave) return;
  total = (lds[0][kMaxHeadDim] + lds[1][kMaxHeadDim]) + (lds[2][kMaxHeadDim] + lds[3][kMaxHeadDim]);
#pragma unroll
  for (int x = 0; x < kMaxHeadDim / 128; ++x)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = 128 * x + 8 * l + i;
      acc[8 * x + i] = (lds[0][d] + lds[1][d]) + (lds[2][d] + lds[3][d]);
    }
  if (slot == 0) {
    const float f = total == 0.f ? 0.f : 1.f / total;
    T* to = static_cast<T*>(a.out.data) + t * a.out.ts + h * a.out.hs;
#pragma unroll
    for (int i = 0; i < kMaxHeadDim / 16; ++i) acc[i] *= f;
#pragma unroll
    for (int x = 0; x < kMaxHeadDim / 128; ++x)
      if (128 * x + 8 * l < D) store8(to + 128 * x + 8 * l, acc + 8 * x);
    if (a.lse && l == 0) a.lse[unit] = total == 0.f ? -INFINITY : high + logf(total);
  }
}

// A wavefront clears a token's rows.
template <typename T>
__device__ void clear_token(const Args& a, int D, int t) {
  const int lane = threadIdx.x & 63, pieces = D / 8;
  const float zeros[8] = {};
  for (int i = lane; i < a.Hq * pieces; i += 64) {
    const int h = i / pieces;
    store8(static_cast<T*>(a.out.data) + t * a.out.ts + h * a.out.hs + 8 * (i - h * pieces), zeros);
  }
  if (a.lse)
    for (int h = lane; h < a.Hq; h += 64) a.lse[static_cast<int64_t>(t) * a.Hq + h] = -INFINITY;
}

// Where rows have no prefix, or it is in their own run, most runs are one workgroup's, and their rows in place.  The workgroups (w, y), w < joins, share the rows of the
// run that workgroup w + 1 of the kernel before began inside, if it was the first to.  The others clear the rows
// that no run has: those of sequences that have nothing to see, and of no sequence.
template <typename T>
__global__ __launch_bounds__(256) void k_join_runs(KvView kv, Args a, int tile_rows, int joins, int n_units, int decode) {
  const int D = kv.D, w = blockIdx.x + 1;
  const int4 all = a.units[n_units];
  if (blockIdx.x >= joins) {
    const int wave = threadIdx.x >> 6, first = ((blockIdx.x - joins) * gridDim.y + blockIdx.y) * 4 + wave, step = (gridDim.x - joins) * gridDim.y * 4;
    const int t0 = all.z ? a.n_tok : kv.cu_q ? kv.cu_q[0] : 0, t1 = all.z ? a.n_tok : kv.cu_q ? kv.cu_q[kv.n_seq] : a.n_tok;
    for (int t = first; t < t0; t += step) clear_token<T>(a, D, t);
    for (int t = t1 + first; t < a.n_tok; t += step) clear_token<T>(a, D, t);
    for (int s = first; s < n_units; s += step) {
      const int4 of = a.units[s];
      for (int t = of.z; of.y == 0 && t < of.z + of.w; ++t) clear_token<T>(a, D, t);      // nothing to see
    }
    return;
  }
  const int share = all.x, total_cost = all.y;
  if (static_cast<int64_t>(w) * share >= total_cost) return;
  const int x = w * share;
  int u = 0;
  for (int n = n_units; n > 1;) {      // the last unit that begins at x or in front of it
    const int step = (n + 63) >> 6, lane = threadIdx.x & 63, at = lane * step;
    const int c = __popcll(__ballot(at < n && a.units[u + (at < n ? at : 0)].x <= x));
    u += (max(c, 1) - 1) * step;
    n = min(step, n - (max(c, 1) - 1) * step);
  }
  const int4 of = a.units[u];
  const Unit unit{of.z, of.w, of.y, 0};
  const Cost costs = decode ? Cost{of.y, 0} : cost_of(unit, a.causal, a, tile_rows);      // a decode's unit has its runs' cost for its length
  const int head = costs.in_front(tiles_of(of.w, a.share, tile_rows)), hk = (x - of.x) / head;
  int run0 = of.x + hk * head, tile = 0, cost = costs.first;
  if (costs.step == 0) {
    tile = (x - run0) / cost;
    run0 += tile * cost;
  }
  for (; x >= run0 + cost; ++tile, cost += costs.step) run0 += cost;
  if (run0 == x || run0 / share != w - 1) return;
  const int rows = of.w * a.share, r0 = tile * tile_rows;
  const int n = (run0 + cost - 1) / share - w + 2;      // parts
  const int64_t queries = static_cast<int64_t>(a.n_tok) * a.Hq;
  // Few parts: sixteen lanes a row; many: a wavefront, four parts at a time.
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, slots = n <= 8 ? 1 : 4, rows_wave = 4 / slots;
  for (int i0 = (blockIdx.y * 4 + wave) * rows_wave; i0 < tile_rows && r0 + i0 < rows; i0 += gridDim.y * 4 * rows_wave) {
    const int i = min(i0 + (slots == 1 ? lane >> 4 : 0), min(tile_rows, rows - r0) - 1);      // behind the last: the last, once more
    const int tq = (r0 + i) / a.by_share, h = hk * a.share + r0 + i - tq * a.share;
    const int64_t row = static_cast<int64_t>(of.z + tq) * a.Hq + h;
    auto part_of = [&](int p) { return p == 0 ? row : queries + static_cast<int64_t>(w - 1 + p) * kMaxRows + i; };
    join_row(a, D, n, slots == 4, true, part_of, static_cast<T*>(a.out.data) + (of.z + tq) * a.out.ts + h * a.out.hs, a.lse ? a.lse + row : nullptr);
  }
}

// ---- few short sequences ------------------------------------------------------------------------------
// With few rows and short contexts a call is its loads one behind the other, and a schedule is some of them, as is a second launch.  Here a
// workgroup has a tile of rows of one sequence for one key head and reads the prefix and the own tokens whole, its four wavefronts in turns:
// bounds, lengths and page ids are asked for together, then queries and keys.  A group's prefix is read by each of its sequences, from the caches.
// Lengths are only on the device, so what the tables have room for says whether it is taken (four candidates in tables for 2048 tokens of their own 25.5 us); by the
// other kernels (heads of 128 on 8, bf16):
//   four candidates behind 197 tokens, 64 rows a group        8.2 us  21.8      120 sequences of up to 2000, 16 rows each        121 us  132
//   22 behind prompts of 300, 64 rows each                   20     43          60 behind prompts of 1000, 64 rows each          56.8    57.0
//   220 behind prompts of 300                                95    111          110 of them                                      92.8    93.1
//   six of up to 3500                                        36.7   37.3        four behind 3500                                 36.6    30.8
// fp32, heads of 64 on 2: 11 behind 300 tokens 9.7 and 20.5, behind 1500 25.8 and 27.1, 56 behind 1500 42.5 and 42.1, 50 of up to 1900 46 and 38.
constexpr int kNearSlots = 512, kNearSeqs = 1024, kNearRoom = 2048;
constexpr int64_t kNearWork = 5 << 19;      // tiles of rows and key heads, times the room

struct NearLds {
  int group, holes[4];
  int pages[2][kNearSlots];      // of the prefix, and the sequence's
  float ml[4][64][2];
  float slab[4][16][128 + 4];
};

template <typename T>
__device__ void clear_token(const Args& a, int D, int t);

template <typename T, int D, int NR, bool EXACT>
__global__ __launch_bounds__(256, (kPerUnit<D, NR>)) void k_tree_near(KvView kv, Args a) {
  typedef Shape<T, D> Z;
  constexpr int E = Z::E, NB = Z::NB, KC = Z::KC, SUB = Z::SUB, TOK = Z::TOK, VJ = 4 * SUB, R = 16 * NR;
  __shared__ NearLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
  const int dim = EXACT ? D : kv.D, hk = blockIdx.y, s = blockIdx.z, last_page = (1 << kv.page_shift) - 1;
  if (tid == 0) lds.group = -1;
  const int32_t* const own_table = kv.pages + static_cast<int64_t>(s) * kv.max_pages;
  int own_id[2], prefix_id[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) own_id[i] = tid + 256 * i < kv.max_pages ? own_table[tid + 256 * i] : 0;
  const int length = kv.length[s], q0 = kv.cu_q ? kv.cu_q[s] : s, q1 = kv.cu_q ? kv.cu_q[s + 1] : s + 1;
  bool falls = false;
  if (kv.cu_q)
    for (int i = tid; i < kv.n_seq; i += 256) falls |= kv.cu_q[i] < 0 || kv.cu_q[i + 1] < kv.cu_q[i] || kv.cu_q[i + 1] > a.n_tok;
  int mine = -1;
  for (int i = tid; i < kv.n_group; i += 256) {
    const int s0 = kv.group_seq[i], s1 = kv.group_seq[i + 1];
    falls |= s0 < 0 || s1 < s0 || s1 > kv.n_seq;
    if (s >= s0 && s < s1) mine = i;
  }
  __syncthreads();
  if (mine >= 0) lds.group = mine;
  const bool none = __syncthreads_or(falls);
  // rows of nobody
  const int workgroups = gridDim.x * gridDim.y * gridDim.z, number = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
  const int cu0 = none ? a.n_tok : kv.cu_q ? kv.cu_q[0] : 0, cu1 = none ? a.n_tok : kv.cu_q ? kv.cu_q[kv.n_seq] : a.n_tok;
  for (int t = number * 4 + wave; t < cu0; t += workgroups * 4) clear_token<T>(a, dim, t);
  for (int t = cu1 + number * 4 + wave; t < a.n_tok; t += workgroups * 4) clear_token<T>(a, dim, t);
  const bool speaks = blockIdx.x == 0 && blockIdx.y == 0;      // of what is wrong with the sequence
  if (none) {
    if (number == 0 && tid == 0) raise_data_error(a.data_error, AT_GRPO_DATA_SEQLENS);
    return;
  }
  const int group = __builtin_amdgcn_readfirstlane(lds.group), ntok = q1 - q0, rows = ntok * a.share;
  const int32_t* const prefix_table = kv.prefix_pages + static_cast<int64_t>(max(group, 0)) * kv.max_prefix_pages;
  int prefix = group >= 0 ? kv.prefix_len[group] : 0, own = length, error = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) prefix_id[i] = group >= 0 && tid + 256 * i < kv.max_prefix_pages ? prefix_table[tid + 256 * i] : 0;
  if (prefix < 0 || prefix > (kv.max_prefix_pages << kv.page_shift)) {
    error |= AT_GRPO_DATA_SEQLENS;
    prefix = 0;
  }
  if (own < 0 || own > (kv.max_pages << kv.page_shift)) {
    error |= AT_GRPO_DATA_SEQLENS;
    own = 0;
  }
  if (ntok > kMostTree) error |= AT_GRPO_DATA_TREE;
  bool missing = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int slot = tid + 256 * i;
    auto put = [&](int which, int id, int tokens) {
      if (slot >= (tokens + last_page) >> kv.page_shift) return;
      const bool no = static_cast<unsigned>(id) >= static_cast<unsigned>(kv.n_pages);
      lds.pages[which][slot] = no ? -1 : id;
      missing |= no;
    };
    put(0, prefix_id[i], prefix);
    put(1, own_id[i], own);
  }
  if (missing && ntok > 0) error |= AT_GRPO_DATA_PAGE;
  if (speaks) raise_data_error(a.data_error, error);
  const bool any = __any(missing);
  if (lane == 0) lds.holes[wave] = any;
  __syncthreads();
  const bool holes = (lds.holes[0] | lds.holes[1] | lds.holes[2] | lds.holes[3]) != 0;

  const uint32_t page_step = static_cast<uint32_t>(kv.Hk * dim) << kv.page_shift;
  const float to_log2 = a.scale * kLog2e;
  const T* const kbase = static_cast<const T*>(kv.k) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
  const T* const vbase = static_cast<const T*>(kv.v) + ((static_cast<int64_t>(hk) * dim) << kv.page_shift);
  const int own0 = (prefix + TOK - 1) & -TOK, end = own0 + own, tree0 = own - ntok;      // own tokens begin a tile; the first new one of them
  struct Tile {
    int which, token, last;
  };
  auto tile_at = [&](int t) { return t < own0 ? Tile{0, t, prefix} : Tile{1, t - own0, own}; };
  auto row_of = [&](const Tile& x, int token) {
    return static_cast<uint64_t>(static_cast<uint32_t>(max(0, lds.pages[x.which][token >> kv.page_shift]))) * page_step + static_cast<uint32_t>((token & last_page) * dim);
  };
  typename Z::KV q[NR][KC], k[SUB][KC];
  typename Z::VV v[NB][VJ];
  auto load_k = [&](const Tile& x) {      // a token behind the last stands for it
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      const T* p = kbase + row_of(x, min(x.token + 16 * y + m, x.last - 1));
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int d = 4 * Z::KE * c + Z::KE * g;
        typename Z::KV z{};
        if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::KV*>(p + d);
        k[y][c] = z;
      }
    }
  };
  auto load_v = [&](const Tile& x) {
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      const T* p = vbase + row_of(x, min(x.token + 16 * y + 4 * g, (x.last - 1) & ~3));
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int d = 16 * E * b + E * m;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typename Z::VV z{};
          if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::VV*>(p + static_cast<int64_t>(j) * dim + d);
          v[b][4 * y + j] = z;
        }
      }
    }
  };
  for (int r0 = blockIdx.x * R; r0 < rows; r0 += gridDim.x * R) {
    uint64_t path[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = min(r0 + 16 * n + m, rows - 1), tq = r / a.by_share, h = hk * a.share + r - tq * a.share;
      const T* from = static_cast<const T*>(a.q.data) + (q0 + tq) * a.q.ts + h * a.q.hs;
      path[n] = a.ancestors[q0 + tq];
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int d = 4 * Z::KE * c + Z::KE * g;
        typename Z::KV z{};
        if (EXACT || d < dim) z = *reinterpret_cast<const typename Z::KV*>(from + d);
        q[n][c] = z;
      }
    }
    f32x4 acc[NR][NB][E];
    float top[NR], sum[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      top[n] = -INFINITY;
      sum[n] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[n][b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t = TOK * wave;
    if (t < end) {
      Tile tile = tile_at(t);
      load_k(tile);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      load_v(tile);
      for (;;) {      // loads are not behind a branch (see k_attend)
        const bool more = t + 4 * TOK < end;
        const Tile next = more ? tile_at(t + 4 * TOK) : tile;
        f32x4 z[NR][SUB];
        scores<T, D>(k, q, z);
        load_k(next);
        uint32_t sees[NR];      // of the tile's tokens
        const bool partly = tile.which && tile.token + TOK > tree0;
#pragma unroll
        for (int n = 0; n < NR; ++n) sees[n] = partly ? static_cast<uint32_t>(tree_bits(path[n], tile.token - tree0)) : ~0u;
        if (partly || tile.token + TOK > tile.last || holes) {
#pragma unroll
          for (int y = 0; y < SUB; ++y) {
            const int at = 16 * y + 4 * g, t4 = tile.token + at, last = tile.last - t4;
            const int seen = last > 0 && lds.pages[tile.which][min(t4, tile.last - 1) >> kv.page_shift] >= 0 ? last : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
              for (int n = 0; n < NR; ++n) z[n][y][i] = i < seen && (sees[n] >> (at + i) & 1) ? z[n][y][i] : -INFINITY;
#pragma unroll
              for (int b = 0; b < NB; ++b) v[b][4 * y + i] = i < seen ? v[b][4 * y + i] : typename Z::VV{};
            }
          }
        }
        weigh_and_add<T, D, true>(v, z, to_log2, acc, top, sum, [&] {
          if (partly) set_apart<T, D>(lds.slab[wave][0], v, acc, [&](int n, int token) { return token < tile.last - tile.token && (sees[n] >> token & 1); });
        });
        load_v(next);
        asm volatile("" ::: "memory");
        if (!more) break;
        tile = next;
        t += 4 * TOK;
      }
    }
    finish<T, EXACT>(a, lds, acc, top, sum, RowsOf{q0, hk, r0, rows}, true, -1, 0, 0, dim);
    lds_barrier();      // what was added up has been read
  }
}

// ---- host -------------------------------------------------------------------------------------------
int check_sizes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  ATG_TRY(check_kv_sizes(kv, n_tok));
  if (Hq <= 0 || Hq % kv->Hk || max_q < 1) return AT_GRPO_EINVAL;
  // rows of all units and runs are counted in 32 bits
  const int64_t units = static_cast<int64_t>(kv->n_seq) + kv->n_group;
  return static_cast<int64_t>(n_tok) * Hq <= 0x3f000000 && units * kv->Hk <= 0x0f000000 ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

struct Scratch {
  int4* units;
  float *part_lse, *part_out;
};

Scratch lay_out(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, WsAlloc& ws) {
  const size_t rows = static_cast<size_t>(kMostGroups) * kMaxRows + static_cast<size_t>(n_tok) * Hq * (kv->n_group > 0 ? 2 : 1);
  Scratch s;
  s.units = ws.take<int4>(static_cast<size_t>(kv->n_seq) + kv->n_group + 1);
  s.part_lse = ws.take<float>(rows);
  s.part_out = ws.take<float>(rows * kv->D);
  return s;
}

typedef void (*Kernel)(KvView, Args);
struct Choice {
  Kernel kernel;
  int rows, per_unit, lds, run_cost = kRunCost;
};

// Rows of a prefix (or, without prefixes, of a sequence) on average, and of a sequence at most.
template <typename T, int D, bool EXACT, bool TREE>
Choice choose_of(int rows_p, int rows_o, bool decode) {
  if (decode) {
    // Rows in as many registers as leave two workgroups (heads of 256: one) and none in memory.  32 groups of 8, 64 rows, behind 2400 tokens with
    // 800 of their own, heads of 128: 64 rows a tile 355 us, 32 229 (5.0 TB/s), though each reads the prefix; with 64 of their own 105 and 109.
    // 32 rows of heads of 256: 32 a tile 343 us, 16 216 (own 64: 121 and 102), fp32 501 and 222.
    constexpr int kMost = sizeof(T) == 4 && D == 64 ? 2 : 256 / D;
    if constexpr (EXACT && kMost > 1) {
      if (rows_p <= 16) return {k_decode<T, D, 1, true, TREE>, 16, kPerUnit<D, 1>, 0};
      if (rows_p <= 32) return {k_decode<T, D, 2, true, TREE>, 32, kPerUnit<D, 2>, 0};
    }
    return {k_decode<T, D, kMost, EXACT, TREE>, 16 * kMost, kPerUnit<D, kMost>, 0};
  }
  // Here bf16 has few rows a sequence, fp32 all that are not few.  1840 sequences behind 600 tokens with 64 of their own, bf16: tiles of 64 rows (heads of
  // 64) 379 us, of 32 298, of 16 286; heads of 128, 2000 in groups of their own, of 32 720, of 16 626; heads of 256, of 32 577, of 16 391.  fp32 heads
  // of 256, messages of 40 tokens: tiles of 32 rows 394 us, of 16 284.
  constexpr int kMost = sizeof(T) == 2 || D == 256 ? 1 : 2;
  if constexpr (sizeof(T) == 2)
    if (rows_o > 16)
      return {k_attend_wide<D, EXACT, TREE>, kWideRows, kWidePerUnit<D>, 4 * kWideTok * D * 2 + static_cast<int>(sizeof(WideLds)), TREE ? kTreeRunCost : kRunCost};
  return {k_attend<T, D, kMost, EXACT, TREE>, 16 * kMost, kPerUnit<D, kMost>, 0};
}

template <typename T, bool TREE>
Choice choose(int D, int rows_p, int rows_o, bool decode) {
  if (D == 64) return choose_of<T, 64, true, TREE>(rows_p, rows_o, decode);
  if (D == 128) return choose_of<T, 128, true, TREE>(rows_p, rows_o, decode);
  if (D == 256) return choose_of<T, 256, true, TREE>(rows_p, rows_o, decode);
  if (D < 64) return choose_of<T, 64, false, TREE>(rows_p, rows_o, decode);
  if (D < 128) return choose_of<T, 128, false, TREE>(rows_p, rows_o, decode);
  return choose_of<T, 256, false, TREE>(rows_p, rows_o, decode);
}

// Tiles of 32 rows, or of 16 where these are no more than there are compute units: 11 sequences of fp32, 52 rows each, 14.1 us and 9.7.
template <typename T, int D, bool EXACT>
Choice near_of(bool large) {
  if constexpr (D <= 128)
    if (large) return {k_tree_near<T, D, 2, EXACT>, 32, 1, 0};
  return {k_tree_near<T, D, 1, EXACT>, 16, 1, 0};
}
template <typename T>
Choice choose_near(int D, bool large) {
  if (D == 64) return near_of<T, 64, true>(large);
  if (D == 128) return near_of<T, 128, true>(large);
  if (D == 256) return near_of<T, 256, true>(large);
  if (D < 64) return near_of<T, 64, false>(large);
  if (D < 128) return near_of<T, 128, false>(large);
  return near_of<T, 256, false>(large);
}

// Everything that goes by sizes alone.
struct Plan {
  Choice choice;
  bool near, decode;
  int64_t tiles;    // of k_tree_near: the most of a sequence and key head
  int coarse;
  double most;      // an upper bound of all costs together
};

template <bool TREE>
int make_plan(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q, Plan* out) {
  ATG_TRY(check_sizes(kv, n_tok, Hq, max_q));
  const int share = Hq / kv->Hk;
  const int64_t all_rows = static_cast<int64_t>(n_tok) * share;
  const int64_t rows_p = kv->n_group ? ceil_div(all_rows, kv->n_group) : 0, rows_o = static_cast<int64_t>(max_q) * share;
  auto small = [](int64_t x) { return static_cast<int>(x < 1 << 20 ? x : 1 << 20); };
  const auto eights_of = [&](int64_t pages) { return static_cast<double>(pages) * kv->page_size / 8; };
  constexpr int run_cost = TREE ? kTreeRunCost : kRunCost;
  const double fixed = 8 + run_cost + kMinShare;
  out->near = false;
  out->tiles = 0;
  if constexpr (TREE) {
    const int64_t room = (static_cast<int64_t>(kv->max_pages) + kv->max_prefix_pages) * kv->page_size;
    const int64_t rows = rows_o < 64 * share ? rows_o : 64 * share;
    const bool large = kv->D <= 128 && ceil_div(rows, 16) * kv->Hk * kv->n_seq > device_cu_count();
    const int64_t tiles = ceil_div(rows, large ? 32 : 16);
    out->near = kv->n_seq > 0 && kv->n_seq <= kNearSeqs && kv->n_group <= kNearSeqs && kv->Hk <= 65535 && kv->max_pages <= kNearSlots && kv->max_prefix_pages <= kNearSlots &&
                room <= kNearRoom && tiles * kv->Hk * kv->n_seq * room <= kNearWork;
    if (out->near) {
      out->choice = kv->dtype == AT_GRPO_BF16 ? choose_near<bf16_t>(kv->D, large) : choose_near<float>(kv->D, large);
      out->decode = false;
      out->coarse = 0;
      out->tiles = tiles;
      out->most = 0;
      return AT_GRPO_OK;
    }
  }
  // Few rows a sequence, as many sequences as LDS has places for, their blocks counted in 26 bits and all costs in 30.
  const double decode_most = kv->Hk * ((all_rows / 16 + kv->n_group + kv->n_seq) * (eights_of(kv->max_prefix_pages) + fixed) + kv->n_seq * (eights_of(kv->max_pages) + fixed));
  out->decode = rows_o <= 16 && kv->n_seq <= kDecodeSeqs && static_cast<int64_t>(kv->n_seq + 1) * kv->max_pages * kv->page_size < 1 << 30 &&
                decode_most < 1 << 30;
  const int rows_u = small(kv->n_group ? rows_p : rows_o);
  out->choice = kv->dtype == AT_GRPO_BF16 ? choose<bf16_t, TREE>(kv->D, rows_u, small(rows_o), out->decode) : choose<float, TREE>(kv->D, rows_u, small(rows_o), out->decode);
  const int64_t tiles_p = kv->n_group ? all_rows / out->choice.rows + kv->n_group : 0, tiles_o = all_rows / out->choice.rows + kv->n_seq;
  out->coarse = 0;
  if (out->decode) {
    out->most = kv->Hk * ((tiles_o + tiles_p) * (kRunCost + 8.0) + tiles_p * (eights_of(kv->max_prefix_pages) + fixed) + kv->n_seq * (eights_of(kv->max_pages) + fixed));
    return AT_GRPO_OK;
  }
  // Costs are added up in 32 bits.  Those of tokens are counted in larger blocks where need be; what each run costs beside them (kRunCost, and
  // up to 1 by rounding up) does not shrink.
  const double runs = kv->Hk * static_cast<double>(tiles_p + tiles_o), beside = runs * (run_cost + 1);
  double tokens = kv->Hk * (tiles_p * eights_of(kv->max_prefix_pages) + tiles_o * eights_of(kv->max_pages));
  if (beside > 1 << 30) return AT_GRPO_EUNSUPPORTED;
  out->most = tokens + runs * fixed;
  for (; tokens + beside > 3 << 29; tokens /= 2) ++out->coarse;
  return AT_GRPO_OK;
}

template <bool TREE>
size_t attention_workspace(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  Plan plan;
  if (make_plan<TREE>(kv, n_tok, Hq, max_q, &plan) != AT_GRPO_OK) return 0;
  WsAlloc ws(nullptr);
  lay_out(kv, n_tok, Hq, ws);
  return ws.bytes();
}

template <bool TREE>
int attend(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, const at_grpo_rows* q, const uint64_t* ancestors, float scale, int32_t causal, int32_t max_q,
           const at_grpo_rows* out, float* lse, int32_t* data_error, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Plan plan;
  ATG_TRY(make_plan<TREE>(kv, n_tok, Hq, max_q, &plan));
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return AT_GRPO_EINVAL;
  KvView view;
  ATG_TRY(check_kv(kv, n_tok, &view));
  if (n_tok == 0) return AT_GRPO_OK;
  if (TREE && !ancestors) return AT_GRPO_EINVAL;
  ATG_TRY(check_rows(q, kv->dtype));
  ATG_TRY(check_rows(out, kv->dtype));
  WsAlloc ws(workspace);
  const Scratch scratch = lay_out(kv, n_tok, Hq, ws);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < ws.bytes()) return AT_GRPO_EWORKSPACE;
  // a run's rows are stored while other runs still read the same queries
  if (rows_meet(*q, *out, n_tok, Hq, kv->D, elem_size(kv->dtype))) return AT_GRPO_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int share = Hq / kv->Hk;
  const Choice& k = plan.choice;
  const bool decode = plan.decode;
  const unsigned blocks = device_cu_count() * k.per_unit < kMostGroups ? device_cu_count() * k.per_unit : kMostGroups;
  Args args{n_tok, Hq, share, divisor(share), plan.coarse, 0, 1, causal != 0, k.run_cost, scale, rows_of(q), rows_of(out), lse, ancestors, data_error, scratch.units, scratch.part_lse, scratch.part_out};
  args.rise = k.rows / (8 * share) >> args.coarse;
  // Where there are workgroups enough, costs are whole shares, so that a run begins with a workgroup: one group of four by
  // k_attend 13.2 us, then 8.0.
  if (plan.most <= static_cast<double>(kMinShare) * blocks) {
    args.quantum = kMinShare;
    args.rise = 0;
  }
  ProfScope ps(PROF_ATTENTION, s);
  if (plan.near) {
    hipLaunchKernelGGL(k.kernel, dim3(static_cast<unsigned>(plan.tiles), kv->Hk, kv->n_seq), dim3(256), 0, s, view, args);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  }
  if (k.lds) ATG_TRY(allow_big_lds(k.kernel, k.lds));
  hipLaunchKernelGGL(k.kernel, dim3(blocks), dim3(256), k.lds, s, view, args);
  ATG_LAUNCH_CHECK();
  const bool bf16 = kv->dtype == AT_GRPO_BF16;
  const int64_t outputs = static_cast<int64_t>(n_tok) * Hq;
  if (kv->n_group == 0 || decode) {
    const int n_units = kv->n_seq + kv->n_group;
    const int y = 4, joins = static_cast<int>(blocks) - 1;
    const int64_t clears = ceil_div(n_units + 1, 4 * y);
    hipLaunchKernelGGL(bf16 ? k_join_runs<bf16_t> : k_join_runs<float>, dim3(static_cast<unsigned>(joins + (clears < 256 ? clears : 256)), y), dim3(256), 0, s,
                       view, args, k.rows, joins, n_units, decode);
  } else if (outputs <= 1024) {
    // Few rows: a workgroup for each.  960 rows, whole calls: behind 1200 tokens 25.6 us (by four heads of a token 33.0), behind 20000 40.8 (61.6),
    // twelve sequences of fp32 behind 300 22.4 (21.3); 3840 rows 39.6 (38.5), 84.1 (85.5) and 38.4 (29.0).
    hipLaunchKernelGGL(bf16 ? k_join<bf16_t> : k_join<float>, dim3(static_cast<unsigned>(outputs)), dim3(256), 0, s, view, args, k.rows);
  } else {
    // Few rows of trees, with many parts each: a wavefront for a row.  Two prompts of 40000 tokens, 6400 rows 216 us whole, then 211, 3500 rows 117 and
    // 110; 45000 rows 221 and 254.
    const int heads = TREE && outputs <= 16384 ? 1 : 4;
    const int64_t waves = static_cast<int64_t>(n_tok) * ceil_div(Hq, heads);
    hipLaunchKernelGGL(bf16 ? k_join_heads<bf16_t> : k_join_heads<float>, grid_of(ceil_div(waves, 4)), dim3(256), 0, s, view, args, k.rows, heads);
  }
  ATG_LAUNCH_CHECK();
  return AT_GRPO_OK;
}

}  // namespace
}  // namespace atg
