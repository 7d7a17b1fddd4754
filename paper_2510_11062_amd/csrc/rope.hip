// Queries and keys of a layer: norm of every head's row, rotation by position, the gradient of both, and the same on the way into a
// paged cache (gfx950).
//
// A row of D elements x with weight w at position p:  u = x r w, r = 1 / sqrt(mean(x^2) + eps), then the pairs (a, b) of the first
// rot_dim elements turn by the table's angle: y_a = c u_a - s u_b, y_b = c u_b + s u_a.  The gradient turns back, then with n = x r and
// g' = g w:  dx = r (g' - n mean(g' n)),  dw = sum over rows of g n.  All sums are fp32.
//
// Bound by memory: two rows' bytes forward, three backward.  A row belongs to LANES neighbouring lanes with four pairs each, so that a
// pair never leaves its lane in either layout.  A large copy makes 5.0 TB/s.
#include "kv_common.hpp"

#include <math.h>

#include <type_traits>

namespace atg {

namespace {

struct Layer {
  int D, half, interleaved, n_pos;   // half: pairs that turn
  float eps, inv_D;
  const float* table;
  const void *qw, *kw;
};

struct Pairs {
  float a[4], b[4];
};

// A lane's eight elements of a row as they lie in memory: four from `lo` on and four from `hi` on, or, where rot_dim is no multiple of
// eight (VEC false), the first and second elements of its four pairs one by one.
struct Places {
  int at[8];
  bool apart;      // lo holds the pairs' first elements and hi their second; otherwise pairs lie side by side
};

template <bool VEC>
__device__ __forceinline__ Places places_of(const Layer& L, int l) {
  Places p;
  p.apart = !VEC || (!L.interleaved && 4 * l < L.half);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = 4 * l + i;
    const bool far = !L.interleaved && pair < L.half;
    p.at[i] = far ? pair : VEC ? 8 * l + i : 2 * pair;
    p.at[4 + i] = far ? pair + L.half : VEC ? 8 * l + 4 + i : 2 * pair + 1;
  }
  return p;
}

template <typename T>
struct Raw;
template <>
struct Raw<bf16_t> {
  uint2 lo, hi;
};
template <>
struct Raw<float> {
  float4 lo, hi;
};

template <bool VEC, typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* row, const Places& p) {
  Raw<T> r;
  if constexpr (VEC) {
    r.lo = *reinterpret_cast<const decltype(r.lo)*>(row + p.at[0]);
    r.hi = *reinterpret_cast<const decltype(r.hi)*>(row + p.at[4]);
  } else {
    T* x = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = row[p.at[i]];
  }
  return r;
}

template <bool VEC, typename T>
__device__ __forceinline__ void store_raw(T* row, const Places& p, const Raw<T>& r) {
  if constexpr (VEC) {
    *reinterpret_cast<decltype(Raw<T>::lo)*>(row + p.at[0]) = r.lo;
    *reinterpret_cast<decltype(Raw<T>::hi)*>(row + p.at[4]) = r.hi;
  } else {
    const T* x = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int i = 0; i < 8; ++i) row[p.at[i]] = x[i];
  }
}

__device__ __forceinline__ Pairs sorted(const float (&lo)[4], const float (&hi)[4], bool apart) {
  return Pairs{{lo[0], apart ? lo[1] : lo[2], apart ? lo[2] : hi[0], apart ? lo[3] : hi[2]},
               {apart ? hi[0] : lo[1], apart ? hi[1] : lo[3], apart ? hi[2] : hi[1], hi[3]}};
}

__device__ __forceinline__ Pairs pairs_of(const Raw<float>& r, const Places& p) {
  const float lo[4] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w}, hi[4] = {r.hi.x, r.hi.y, r.hi.z, r.hi.w};
  return sorted(lo, hi, p.apart);
}
__device__ __forceinline__ Pairs pairs_of(const Raw<bf16_t>& r, const Places& p) {
  const auto low = [](uint32_t x) { return __uint_as_float(x << 16); };
  const auto high = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
  const float lo[4] = {low(r.lo.x), high(r.lo.x), low(r.lo.y), high(r.lo.y)}, hi[4] = {low(r.hi.x), high(r.hi.x), low(r.hi.y), high(r.hi.y)};
  return sorted(lo, hi, p.apart);
}

// pairs_of backwards
template <typename T>
__device__ __forceinline__ Raw<T> raw_of(const Pairs& x, const Places& p) {
  const float lo[4] = {x.a[0], p.apart ? x.a[1] : x.b[0], p.apart ? x.a[2] : x.a[1], p.apart ? x.a[3] : x.b[1]};
  const float hi[4] = {p.apart ? x.b[0] : x.a[2], p.apart ? x.b[1] : x.b[2], p.apart ? x.b[2] : x.a[3], x.b[3]};
  if constexpr (sizeof(T) == 4) return Raw<T>{make_float4(lo[0], lo[1], lo[2], lo[3]), make_float4(hi[0], hi[1], hi[2], hi[3])};
  else
    return Raw<T>{make_uint2(pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3])), make_uint2(pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3]))};
}

// Cosines and sines of a lane's pairs; 1 and 0 behind the last that turns (such a pair is passed by, not multiplied: 0 times an infinite
// partner would be NaN).
template <bool VEC>
__device__ __forceinline__ Pairs load_turn(const Layer& L, int l, int position) {
  Pairs t{{1.f, 1.f, 1.f, 1.f}, {}};
  const float* e = L.table + 2 * (static_cast<int64_t>(position) * L.half + 4 * l);
  if constexpr (VEC) {
    if (4 * l < L.half) {
      const float4 x = *reinterpret_cast<const float4*>(e), y = *reinterpret_cast<const float4*>(e + 4);
      t = Pairs{{x.x, x.z, y.x, y.z}, {x.y, x.w, y.y, y.w}};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * l + i < L.half) {
        t.a[i] = e[2 * i];
        t.b[i] = e[2 * i + 1];
      }
  }
  return t;
}

template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <int LANES>
__device__ __forceinline__ float inverse_size(const Pairs& x, const Layer& L) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) ss = fmaf(x.a[i], x.a[i], fmaf(x.b[i], x.b[i], ss));
  return rsqrtf(fmaf(row_sum<LANES>(ss), L.inv_D, L.eps));
}

// Where a new token belongs: its position, and its place in the cache (rows between its heads are page_size * D apart).
struct Spot {
  int position;      // -1: nowhere
  int64_t at;
};

// Sequence and group of new token t: one that there is not, or one out of range, is found out by find_spot.
struct Owner {
  int s, g;
};
__device__ __forceinline__ Owner find_owner(const KvView& kv, int t) {
  const int s = kv.cu_q ? __builtin_amdgcn_readfirstlane(wave_upper_bound(kv.cu_q, kv.n_seq + 1, t)) - 1 : t;
  return Owner{s, kv.n_group > 0 ? __builtin_amdgcn_readfirstlane(wave_upper_bound(kv.group_seq, kv.n_group + 1, s)) - 1 : -1};
}

// What depends on nothing is asked for together, without branches in between.
__device__ __forceinline__ Spot find_spot(const KvView& kv, int n_pos, int t, const Owner& of, int32_t* data_error) {
  Spot spot{-1, 0};
  const bool there = of.s >= 0 && of.s < kv.n_seq, grouped = of.g >= 0 && of.g < kv.n_group;
  const int s = there ? of.s : 0;
  int length = 0, q0 = t, q1 = t + 1, prefix = 0, g0 = s, g1 = s + 1;
  if (kv.n_seq > 0) {
    length = kv.length[s];
    if (kv.cu_q) {
      q0 = kv.cu_q[s];
      q1 = kv.cu_q[s + 1];
    }
  }
  if (grouped) {
    prefix = kv.prefix_len[of.g];
    g0 = kv.group_seq[of.g];
    g1 = kv.group_seq[of.g + 1];
  }
  int error = 0, place = -1;
  if (!there || q0 < 0 || q0 > t || q1 <= t || length < 0 || length > (kv.max_pages << kv.page_shift) || q1 - q0 > length || prefix < 0 ||
      prefix > (kv.max_prefix_pages << kv.page_shift) || g0 < 0 || g0 > s || g1 <= s || g1 > kv.n_seq)
    error = AT_GRPO_DATA_SEQLENS;
  else
    place = length - (q1 - t);
  if (place >= 0) {
    const int page = kv.pages[static_cast<int64_t>(s) * kv.max_pages + (place >> kv.page_shift)];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(kv.n_pages)) error |= AT_GRPO_DATA_PAGE;
    if (n_pos >= 0 && prefix + place >= n_pos) error |= AT_GRPO_DATA_POSITION;
    if (!error) {
      spot.position = prefix + place;
      spot.at = ((static_cast<int64_t>(page) * kv.Hk << kv.page_shift) + (place & ((1 << kv.page_shift) - 1))) * kv.D;
    }
  }
  if ((threadIdx.x & 63) == 0) raise_data_error(data_error, error);
  return spot;
}

// The rows of one token are its queries' heads, then its keys', then (appending) its values'; a wavefront takes every parts-th group of
// 64 / LANES of them, kBatch groups in flight at a time.  Where a row lies: element 0 of head j of its kind.
constexpr int kBatch = 4;

template <typename T>
struct Token {
  const T* src[3];
  T* dst[3];
  int64_t src_hs[3], dst_hs[3];
  int end[3];        // first row behind the kind
};

template <typename T>
__device__ __forceinline__ const T* source_of(const Token<T>& t, int j) {
  return j < t.end[0] ? t.src[0] + j * t.src_hs[0] : j < t.end[1] ? t.src[1] + (j - t.end[0]) * t.src_hs[1] : t.src[2] + (j - t.end[1]) * t.src_hs[2];
}
template <typename T>
__device__ __forceinline__ T* target_of(const Token<T>& t, int j) {
  return j < t.end[0] ? t.dst[0] + j * t.dst_hs[0] : j < t.end[1] ? t.dst[1] + (j - t.end[0]) * t.dst_hs[1] : t.dst[2] + (j - t.end[1]) * t.dst_hs[2];
}

template <typename T, int LANES, bool VEC>
struct Rotator {
  static constexpr int G = 64 / LANES;
  const Layer& L;
  const Places p;
  const int l, grp, turning;      // of the lane's pairs the first `turning` turn
  const bool mine;
  Raw<T> raw_wq{}, raw_wk{}, x[kBatch];
  Pairs wq, wk;

  __device__ __forceinline__ explicit Rotator(const Layer& layer)
      : L(layer), p(places_of<VEC>(layer, threadIdx.x & (LANES - 1))), l(threadIdx.x & (LANES - 1)), grp((threadIdx.x & 63) / LANES), turning(layer.half - 4 * l),
        mine(8 * l < layer.D) {
    if (mine && L.qw) raw_wq = load_raw<VEC>(static_cast<const T*>(L.qw), p);
    if (mine && L.kw) raw_wk = load_raw<VEC>(static_cast<const T*>(L.kw), p);
  }
  // Once the first rows are on their way; store looks at no weight that there is not.
  __device__ __forceinline__ void take_weights() {
    wq = pairs_of(raw_wq, p);
    wk = pairs_of(raw_wk, p);
  }

  __device__ __forceinline__ void load(const Token<T>& t, int j0, int step) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int j = j0 + i * step + grp;
      x[i] = Raw<T>{};
      if (mine && j < t.end[2]) x[i] = load_raw<VEC>(source_of(t, j), p);
    }
  }

  // zero: queries get zeros, and there is no place for the rest
  __device__ __forceinline__ void store(const Token<T>& t, int j0, int step, const Pairs& turn, bool zero) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int j = j0 + i * step + grp;
      if (j0 + i * step >= t.end[2]) break;
      const bool is_q = j < t.end[0], value = j >= t.end[1], norm = is_q ? L.qw != nullptr : !value && L.kw != nullptr;
      Pairs u = pairs_of(x[i], p);
      const float r = inverse_size<LANES>(u, L);
      Raw<T> y = x[i];
      if (!value) {
        Pairs v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (norm) {
            u.a[e] *= r * (is_q ? wq.a[e] : wk.a[e]);
            u.b[e] *= r * (is_q ? wq.b[e] : wk.b[e]);
          }
          v.a[e] = e < turning ? fmaf(u.a[e], turn.a[e], -u.b[e] * turn.b[e]) : u.a[e];
          v.b[e] = e < turning ? fmaf(u.b[e], turn.a[e], u.a[e] * turn.b[e]) : u.b[e];
        }
        y = raw_of<T>(v, p);
      }
      if (zero) y = Raw<T>{};
      if (mine && j < t.end[2]) store_raw<VEC>(target_of(t, j), p, y);
    }
  }
};

// 16384 tokens of 40 heads of 128, bf16: 65 to 67 us, 5.0 to 5.2 TB/s.  197 tokens of 24 heads: 3.8 us, one wait for memory behind another.
template <typename T, int LANES, bool VEC>
__global__ __launch_bounds__(256) void k_norm_rope(Layer L, int n_tok, int parts, int Hq, int Hk, Rows q, Rows k, const int32_t* __restrict__ position,
                                                   Rows q_out, Rows k_out, int32_t* data_error) {
  const uint32_t unit = flat_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t token_of = unit / static_cast<uint32_t>(parts);
  if (token_of >= static_cast<uint32_t>(n_tok)) return;
  const int t = static_cast<int>(token_of), part = static_cast<int>(unit - token_of * parts);
  const Token<T> token{{static_cast<const T*>(q.data) + t * q.ts, static_cast<const T*>(k.data) + t * k.ts, nullptr},
                       {static_cast<T*>(q_out.data) + t * q_out.ts, static_cast<T*>(k_out.data) + t * k_out.ts, nullptr},
                       {q.hs, k.hs, 0}, {q_out.hs, k_out.hs, 0}, {Hq, Hq + Hk, Hq + Hk}};
  Rotator<T, LANES, VEC> R(L);
  const int step = parts * R.G;
  int j0 = part * R.G;
  const int pos = L.half ? position[t] : 0;
  R.load(token, j0, step);
  const bool bad = L.half && static_cast<unsigned>(pos) >= static_cast<unsigned>(L.n_pos);
  if (bad && part == 0 && (threadIdx.x & 63) == 0) raise_data_error(data_error, AT_GRPO_DATA_POSITION);
  Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
  if (!bad && L.half) turn = load_turn<VEC>(L, R.l, pos);
  R.take_weights();
  for (;;) {
    R.store(token, j0, step, turn, bad);
    j0 += kBatch * step;
    if (j0 >= Hq + Hk) break;
    R.load(token, j0, step);
  }
}

// A token finds its sequence by bisection, its position and its page, while its rows are on their way.  46659 tokens of 64 prompts, 32 heads
// of 128 in and out, bf16: 150 us, 5.1 TB/s.  1339 single tokens of 48 heads: 11 us, 3.0 TB/s; four: 4.0 us, a chain of waits.
template <typename T, int LANES, bool VEC>
__global__ __launch_bounds__(256) void k_kv_append(KvView kv, Layer L, int n_tok, int parts, int Hq, Rows q, Rows k, Rows v, Rows q_out,
                                                   int32_t* data_error) {
  const uint32_t unit = flat_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t token_of = unit / static_cast<uint32_t>(parts);
  if (token_of >= static_cast<uint32_t>(n_tok)) return;
  const int t = static_cast<int>(token_of), part = static_cast<int>(unit - token_of * parts);
  const Owner owner = find_owner(kv, t);
  const int64_t hs = static_cast<int64_t>(kv.D) << kv.page_shift;
  Token<T> token{{static_cast<const T*>(q.data) + t * q.ts, static_cast<const T*>(k.data) + t * k.ts, static_cast<const T*>(v.data) + t * v.ts},
                 {static_cast<T*>(q_out.data) + t * q_out.ts, static_cast<T*>(kv.k), static_cast<T*>(kv.v)},
                 {q.hs, k.hs, v.hs}, {q_out.hs, hs, hs}, {Hq, Hq + kv.Hk, Hq + 2 * kv.Hk}};
  Rotator<T, LANES, VEC> R(L);
  const int step = parts * R.G;
  int j0 = part * R.G;
  R.load(token, j0, step);      // rows do not wait for where they go
  const Spot spot = find_spot(kv, L.half ? L.n_pos : -1, t, owner, part == 0 ? data_error : nullptr);
  const bool bad = spot.position < 0;
  Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
  if (!bad && L.half) turn = load_turn<VEC>(L, R.l, spot.position);
  R.take_weights();
  token.dst[1] += spot.at;
  token.dst[2] += spot.at;
  if (bad) token.end[1] = token.end[2] = Hq;
  for (;;) {
    R.store(token, j0, step, turn, bad);
    j0 += kBatch * step;
    if (j0 >= token.end[2]) break;
    R.load(token, j0, step);
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
constexpr int kGradBlocks = 1024;

constexpr int kGradBatch = 2;

template <typename T, int LANES, bool VEC>
__device__ __forceinline__ void rotate_rows_back(const Layer& L, const T* dy, int64_t dy_hs, const T* src, int64_t src_hs, T* dst, int64_t dst_hs, int H,
                                                 const Pairs& w, bool norm, const Pairs& turn, const Places& p, bool zero, int part, int parts, Pairs& dw) {
  constexpr int G = 64 / LANES;
  const int l = threadIdx.x & (LANES - 1), grp = (threadIdx.x & 63) / LANES;
  const int turning = L.half - 4 * l;
  const bool mine = 8 * l < L.D;
  for (int h0 = part * G; h0 < H; h0 += kGradBatch * parts * G) {
    Raw<T> rx[kGradBatch], rg[kGradBatch];
#pragma unroll
    for (int i = 0; i < kGradBatch; ++i) {
      const int h = h0 + i * parts * G + grp;
      rx[i] = rg[i] = Raw<T>{};
      if (mine && h < H) {
        rg[i] = load_raw<VEC>(dy + h * dy_hs, p);
        if (norm) rx[i] = load_raw<VEC>(src + h * src_hs, p);
      }
    }
#pragma unroll
    for (int i = 0; i < kGradBatch; ++i) {
      const int h = h0 + i * parts * G + grp;
      if (h0 + i * parts * G >= H) break;
      const bool on = mine && h < H;
      const Pairs d = pairs_of(rg[i], p);
      Pairs x = pairs_of(rx[i], p), g;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g.a[e] = e < turning ? fmaf(d.a[e], turn.a[e], d.b[e] * turn.b[e]) : d.a[e];
        g.b[e] = e < turning ? fmaf(d.b[e], turn.a[e], -d.a[e] * turn.b[e]) : d.b[e];
      }
      if (norm) {
        const float r = inverse_size<LANES>(x, L);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x.a[e] *= r;
          x.b[e] *= r;
          if (on && !zero) {      // a lane without a row would add 0 times the size of no row
            dw.a[e] = fmaf(g.a[e], x.a[e], dw.a[e]);
            dw.b[e] = fmaf(g.b[e], x.b[e], dw.b[e]);
          }
          g.a[e] *= w.a[e];
          g.b[e] *= w.b[e];
          dot = fmaf(g.a[e], x.a[e], fmaf(g.b[e], x.b[e], dot));
        }
        const float mean = row_sum<LANES>(dot) * L.inv_D;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g.a[e] = r * fmaf(-x.a[e], mean, g.a[e]);
          g.b[e] = r * fmaf(-x.b[e], mean, g.b[e]);
        }
      }
      Raw<T> y = raw_of<T>(g, p);
      if (zero) y = Raw<T>{};
      if (on) store_raw<VEC>(dst + h * dst_hs, p, y);
    }
  }
}

// The rows of one kind (0 queries, 1 keys) that a workgroup's lanes added up, as one row of partial sums.
template <int LANES, bool VEC>
__device__ void store_partial(const Layer& L, Pairs dw, float* lds, float* __restrict__ partial) {
  const int l = threadIdx.x & (LANES - 1), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1) {
      dw.a[i] += __shfl_xor(dw.a[i], o, 64);
      dw.b[i] += __shfl_xor(dw.b[i], o, 64);
    }
  __syncthreads();
  if (lane < LANES && 8 * l < L.D) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = 4 * l + i;
      const bool far = !L.interleaved && pair < L.half;
      lds[wave * kMaxHeadDim + (far ? pair : 2 * pair)] = dw.a[i];
      lds[wave * kMaxHeadDim + (far ? pair + L.half : 2 * pair + 1)] = dw.b[i];
    }
  }
  __syncthreads();
  const int d = threadIdx.x;
  if (d < L.D) partial[d] = (lds[d] + lds[kMaxHeadDim + d]) + (lds[2 * kMaxHeadDim + d] + lds[3 * kMaxHeadDim + d]);
}

// 16383 tokens of 24 heads of 128, bf16: 55 us, 5.5 TB/s; 3001 of 16 of 64, fp32: 12 us, 3.0 TB/s.  A workgroup keeps the weights'
// gradients of its rows in registers and writes them once; k_weight_grad adds up the workgroups' (5 us).
template <typename T, int LANES, bool VEC>
__global__ __launch_bounds__(256) void k_norm_rope_bwd(Layer L, int n_tok, int parts, int Hq, int Hk, Rows dq_out, Rows dk_out, Rows q, Rows k,
                                                       const int32_t* __restrict__ position, Rows dq, Rows dk, float* __restrict__ partial,
                                                       int32_t* data_error) {
  __shared__ float lds[4 * kMaxHeadDim];
  const int l = threadIdx.x & (LANES - 1);
  const Places p = places_of<VEC>(L, l);
  Pairs dwq{}, dwk{}, wq{}, wk{};
  if (8 * l < L.D && L.qw) wq = pairs_of(load_raw<VEC>(static_cast<const T*>(L.qw), p), p);
  if (8 * l < L.D && L.kw) wk = pairs_of(load_raw<VEC>(static_cast<const T*>(L.kw), p), p);
  const int64_t units = static_cast<int64_t>(n_tok) * parts;
  for (int64_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += gridDim.x * 4) {
    const int64_t t = unit / parts;
    const int part = static_cast<int>(unit - t * parts);
    const int pos = L.half ? position[t] : 0;
    const bool bad = L.half && static_cast<unsigned>(pos) >= static_cast<unsigned>(L.n_pos);
    if (bad && part == 0 && (threadIdx.x & 63) == 0) raise_data_error(data_error, AT_GRPO_DATA_POSITION);
    Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
    if (!bad && L.half) turn = load_turn<VEC>(L, l, pos);
    if (Hq)
      rotate_rows_back<T, LANES, VEC>(L, static_cast<const T*>(dq_out.data) + t * dq_out.ts, dq_out.hs, static_cast<const T*>(q.data) + t * q.ts, q.hs,
                                      static_cast<T*>(dq.data) + t * dq.ts, dq.hs, Hq, wq, L.qw != nullptr, turn, p, bad, part, parts, dwq);
    if (Hk)
      rotate_rows_back<T, LANES, VEC>(L, static_cast<const T*>(dk_out.data) + t * dk_out.ts, dk_out.hs, static_cast<const T*>(k.data) + t * k.ts, k.hs,
                                      static_cast<T*>(dk.data) + t * dk.ts, dk.hs, Hk, wk, L.kw != nullptr, turn, p, bad, part, parts, dwk);
  }
  if (L.qw) store_partial<LANES, VEC>(L, dwq, lds, partial + static_cast<int64_t>(blockIdx.x) * L.D);
  if (L.kw) store_partial<LANES, VEC>(L, dwk, lds, partial + (static_cast<int64_t>(kGradBlocks) + blockIdx.x) * L.D);
}

// d_weight[d] = sum over the workgroups' rows, eight elements a workgroup, in 64 bits
__global__ __launch_bounds__(1024) void k_weight_grad(int D, int blocks, const float* __restrict__ partial, float* dq_weight, float* dk_weight) {
  __shared__ double red[128][8];
  const int c = threadIdx.x & 7, slice = threadIdx.x >> 3, d = blockIdx.x * 8 + c;      // D is a multiple of 8
  float* out = blockIdx.y ? dk_weight : dq_weight;
  if (!out) return;
  const float* rows = partial + static_cast<int64_t>(blockIdx.y) * kGradBlocks * D + d;
  float x[kGradBlocks / 128];
#pragma unroll
  for (int i = 0; i < kGradBlocks / 128; ++i) x[i] = slice + 128 * i < blocks ? rows[static_cast<int64_t>(slice + 128 * i) * D] : 0.f;
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kGradBlocks / 128; ++i) s += static_cast<double>(x[i]);
  red[slice][c] = s;
  for (int o = 64; o > 0; o >>= 1) {
    __syncthreads();
    if (slice < o) red[slice][c] += red[slice + o][c];
  }
  if (slice == 0) out[d] = static_cast<float>(red[0][c]);
}

// ---- table ------------------------------------------------------------------------------------------
struct TableArgs {
  int n_pos, half, scaling;
  double log_base, factor, trained, slow, fast, magnitude;
};

__global__ __launch_bounds__(256) void k_rope_table(TableArgs A, float2* __restrict__ table) {
  const int64_t n = static_cast<int64_t>(A.n_pos) * A.half;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int pos = static_cast<int>(i / A.half), pair = static_cast<int>(i - static_cast<int64_t>(pos) * A.half);
    double f = exp(-A.log_base * pair / A.half);
    if (A.scaling == AT_GRPO_ROPE_LINEAR) f /= A.factor;
    if (A.scaling == AT_GRPO_ROPE_PARTS) {
      const double turns = A.trained * f / 6.283185307179586;
      const double keep = fmin(fmax((turns - A.slow) / (A.fast - A.slow), 0.0), 1.0);
      f *= keep + (1.0 - keep) / A.factor;
    }
    double s, c;
    sincos(pos * f, &s, &c);
    table[i] = make_float2(static_cast<float>(A.magnitude * c), static_cast<float>(A.magnitude * s));
  }
}

int check_layer(const at_grpo_norm_rope* a, Layer* out) {
  if (!a) return AT_GRPO_EINVAL;
  ATG_TRY(check_head_dim(a->dtype, a->D));
  if (a->rot_dim < 0 || a->rot_dim > a->D || a->rot_dim % 2 || !(a->eps >= 0.f)) return AT_GRPO_EINVAL;
  if (a->layout != AT_GRPO_ROPE_HALF && a->layout != AT_GRPO_ROPE_INTERLEAVED) return AT_GRPO_EINVAL;
  if (a->rot_dim > 0 && (!a->table || a->n_pos <= 0 || !aligned16(a->table))) return AT_GRPO_EINVAL;
  if ((a->q_weight && !aligned16(a->q_weight)) || (a->k_weight && !aligned16(a->k_weight))) return AT_GRPO_EINVAL;
  *out = Layer{a->D, a->rot_dim / 2, a->layout, a->n_pos, a->eps, 1.f / static_cast<float>(a->D), a->table, a->q_weight, a->k_weight};
  return AT_GRPO_OK;
}

// Rows of a token are counted in 32 bits, up to some 10^5 behind their last.
int check_heads(int64_t q, int64_t k) {
  if (q < 0 || k < 0) return AT_GRPO_EINVAL;
  return q + k <= 1 << 30 ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// Few tokens are shared by several wavefronts each, so that the chip has work: about 4096 wavefronts, or all groups of heads.
int parts_of(int n_tok, int rows, int lanes) {
  const int groups = static_cast<int>(ceil_div(rows, 64 / lanes));
  const int64_t want = ceil_div(4096, n_tok > 0 ? n_tok : 1);
  return static_cast<int>(want < groups ? want : groups);
}

// f(element, integral constant of the lanes of a row, whether pairs come in whole vectors)
template <typename F>
int by_shape(int32_t dtype, const Layer& L, F f) {
  const auto by_lanes = [&](auto t, auto vec) -> int {
    const int lanes = lanes_of(L.D);
    if (lanes == 8) return f(t, std::integral_constant<int, 8>{}, vec);
    return lanes == 16 ? f(t, std::integral_constant<int, 16>{}, vec) : f(t, std::integral_constant<int, 32>{}, vec);
  };
  const bool vec = L.half % 4 == 0;
  if (dtype == AT_GRPO_BF16) return vec ? by_lanes(bf16_t{}, std::true_type{}) : by_lanes(bf16_t{}, std::false_type{});
  return vec ? by_lanes(0.f, std::true_type{}) : by_lanes(0.f, std::false_type{});
}

}  // namespace

size_t qk_norm_rope_bwd_workspace() {
  WsAlloc ws(nullptr);
  ws.take<float>(2 * static_cast<size_t>(kGradBlocks) * kMaxHeadDim);
  return ws.bytes();
}

}  // namespace atg

using namespace atg;

extern "C" int at_grpo_rope_table(const at_grpo_rope* rope, int32_t n_pos, float* table, void* hip_stream) {
  if (!rope || rope->rot_dim <= 0 || rope->rot_dim % 2 || n_pos < 0) return AT_GRPO_EINVAL;
  if (rope->rot_dim > kMaxHeadDim) return AT_GRPO_EUNSUPPORTED;
  if (!(rope->base > 0) || !(rope->magnitude > 0) || !isfinite(rope->base) || !isfinite(rope->magnitude)) return AT_GRPO_EINVAL;
  if (rope->scaling < AT_GRPO_ROPE_PLAIN || rope->scaling > AT_GRPO_ROPE_PARTS) return AT_GRPO_EINVAL;
  TableArgs A{n_pos, rope->rot_dim / 2, rope->scaling, log(rope->base), 1.0, 1.0, 0.0, 1.0, rope->magnitude};
  if (rope->scaling != AT_GRPO_ROPE_PLAIN) {
    if (!(rope->factor >= 1) || !isfinite(rope->factor)) return AT_GRPO_EINVAL;
    A.factor = rope->factor;
  }
  if (rope->scaling == AT_GRPO_ROPE_BASE) {
    if (rope->rot_dim <= 2) return AT_GRPO_EINVAL;
    A.log_base += log(rope->factor) * rope->rot_dim / (rope->rot_dim - 2);
  }
  if (rope->scaling == AT_GRPO_ROPE_PARTS) {
    if (!(rope->trained > 0) || !(rope->slow < rope->fast) || !isfinite(rope->trained) || !isfinite(rope->slow) || !isfinite(rope->fast)) return AT_GRPO_EINVAL;
    A.trained = rope->trained;
    A.slow = rope->slow;
    A.fast = rope->fast;
  }
  if (n_pos == 0) return AT_GRPO_OK;
  if (!table || !aligned16(table)) return AT_GRPO_EINVAL;
  const int64_t want = ceil_div(static_cast<int64_t>(n_pos) * A.half, 256);
  hipLaunchKernelGGL(k_rope_table, dim3(static_cast<unsigned>(want < 65536 ? want : 65536)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), A,
                     reinterpret_cast<float2*>(table));
  ATG_LAUNCH_CHECK();
  return AT_GRPO_OK;
}

extern "C" int at_grpo_qk_norm_rope(const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq, int32_t Hk, const at_grpo_rows* q, const at_grpo_rows* k,
                                    const int32_t* position, const at_grpo_rows* q_out, const at_grpo_rows* k_out, int32_t* data_error,
                                    void* hip_stream) {
  Layer L;
  ATG_TRY(check_layer(layer, &L));
  if (n_tok < 0 || (Hq == 0 && Hk == 0)) return AT_GRPO_EINVAL;
  ATG_TRY(check_heads(Hq, Hk));
  if (n_tok == 0) return AT_GRPO_OK;
  if (L.half && !position) return AT_GRPO_EINVAL;
  if (Hq) ATG_TRY(check_rows(q, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q_out, layer->dtype));
  if (Hk) ATG_TRY(check_rows(k, layer->dtype));
  if (Hk) ATG_TRY(check_rows(k_out, layer->dtype));
  if (Hq) ATG_TRY(check_in_place(q, q_out, n_tok, Hq, L.D, layer->dtype));
  if (Hk) ATG_TRY(check_in_place(k, k_out, n_tok, Hk, L.D, layer->dtype));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int parts = parts_of(n_tok, Hq + Hk, lanes_of(L.D));
  if (static_cast<int64_t>(n_tok) * parts > 0x7fffffff) return AT_GRPO_EUNSUPPORTED;
  const dim3 blocks = grid_of(ceil_div(static_cast<int64_t>(n_tok) * parts, 4));
  ProfScope ps(PROF_ROPE, s);
  return by_shape(layer->dtype, L, [&](auto t, auto n, auto vec) -> int {
    hipLaunchKernelGGL((k_norm_rope<decltype(t), decltype(n)::value, decltype(vec)::value>), blocks, dim3(256), 0, s, L, n_tok, parts, Hq, Hk,
                       Hq ? rows_of(q) : Rows{}, Hk ? rows_of(k) : Rows{}, position, Hq ? rows_of(q_out) : Rows{}, Hk ? rows_of(k_out) : Rows{}, data_error);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  });
}

extern "C" int at_grpo_qk_norm_rope_bwd(const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq, int32_t Hk, const at_grpo_rows* dq_out,
                                        const at_grpo_rows* dk_out, const at_grpo_rows* q, const at_grpo_rows* k, const int32_t* position,
                                        const at_grpo_rows* dq, const at_grpo_rows* dk, float* dq_weight, float* dk_weight, int32_t* data_error,
                                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  Layer L;
  ATG_TRY(check_layer(layer, &L));
  if (n_tok < 0 || (Hq == 0 && Hk == 0)) return AT_GRPO_EINVAL;
  ATG_TRY(check_heads(Hq, Hk));
  if (!Hq) L.qw = nullptr;
  if (!Hk) L.kw = nullptr;
  if ((L.qw && !dq_weight) || (L.kw && !dk_weight)) return AT_GRPO_EINVAL;
  if (n_tok > 0) {
    if (L.half && !position) return AT_GRPO_EINVAL;
    if (Hq) {
      ATG_TRY(check_rows(dq_out, layer->dtype));
      ATG_TRY(check_rows(dq, layer->dtype));
      if (L.qw) ATG_TRY(check_rows(q, layer->dtype));
      ATG_TRY(check_in_place(dq_out, dq, n_tok, Hq, L.D, layer->dtype));
      if (L.qw) ATG_TRY(check_in_place(q, dq, n_tok, Hq, L.D, layer->dtype));
    }
    if (Hk) {
      ATG_TRY(check_rows(dk_out, layer->dtype));
      ATG_TRY(check_rows(dk, layer->dtype));
      if (L.kw) ATG_TRY(check_rows(k, layer->dtype));
      ATG_TRY(check_in_place(dk_out, dk, n_tok, Hk, L.D, layer->dtype));
      if (L.kw) ATG_TRY(check_in_place(k, dk, n_tok, Hk, L.D, layer->dtype));
    }
  }
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < qk_norm_rope_bwd_workspace()) return AT_GRPO_EWORKSPACE;
  float* partial = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int parts = parts_of(n_tok, Hq > Hk ? Hq : Hk, lanes_of(L.D));
  const int64_t want = ceil_div(static_cast<int64_t>(n_tok) * parts, 4);
  const unsigned blocks = static_cast<unsigned>(want > kGradBlocks ? kGradBlocks : want < 1 ? 1 : want);
  const bool rows = n_tok > 0;
  ProfScope ps(PROF_ROPE, s);
  ATG_TRY(by_shape(layer->dtype, L, [&](auto t, auto n, auto vec) -> int {
    hipLaunchKernelGGL((k_norm_rope_bwd<decltype(t), decltype(n)::value, decltype(vec)::value>), dim3(blocks), dim3(256), 0, s, L, n_tok, parts, Hq, Hk,
                       rows && Hq ? rows_of(dq_out) : Rows{}, rows && Hk ? rows_of(dk_out) : Rows{}, rows && L.qw ? rows_of(q) : Rows{},
                       rows && L.kw ? rows_of(k) : Rows{}, position, rows && Hq ? rows_of(dq) : Rows{}, rows && Hk ? rows_of(dk) : Rows{}, partial,
                       data_error);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  }));
  if (L.qw || L.kw) {
    hipLaunchKernelGGL(k_weight_grad, dim3(static_cast<unsigned>(L.D / 8), 2), dim3(1024), 0, s, L.D, static_cast<int>(blocks), partial,
                       L.qw ? dq_weight : nullptr, L.kw ? dk_weight : nullptr);
    ATG_LAUNCH_CHECK();
  }
  return AT_GRPO_OK;
}

extern "C" int at_grpo_kv_append(const at_grpo_kv* kv, const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq, const at_grpo_rows* q,
                                 const at_grpo_rows* k, const at_grpo_rows* v, const at_grpo_rows* q_out, int32_t* data_error, void* hip_stream) {
  Layer L;
  KvView view;
  ATG_TRY(check_layer(layer, &L));
  ATG_TRY(check_kv(kv, n_tok, &view));
  if (kv->dtype != layer->dtype || kv->D != layer->D) return AT_GRPO_EINVAL;
  ATG_TRY(check_heads(Hq, 2 * static_cast<int64_t>(kv->Hk)));
  if (n_tok == 0) return AT_GRPO_OK;
  ATG_TRY(check_rows(k, layer->dtype));
  ATG_TRY(check_rows(v, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q_out, layer->dtype));
  if (Hq) ATG_TRY(check_in_place(q, q_out, n_tok, Hq, L.D, layer->dtype));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int parts = parts_of(n_tok, Hq + 2 * kv->Hk, lanes_of(L.D));
  if (static_cast<int64_t>(n_tok) * parts > 0x7fffffff) return AT_GRPO_EUNSUPPORTED;
  const dim3 blocks = grid_of(ceil_div(static_cast<int64_t>(n_tok) * parts, 4));
  ProfScope ps(PROF_ROPE, s);
  return by_shape(layer->dtype, L, [&](auto t, auto n, auto vec) -> int {
    hipLaunchKernelGGL((k_kv_append<decltype(t), decltype(n)::value, decltype(vec)::value>), blocks, dim3(256), 0, s, view, L, n_tok, parts, Hq,
                       Hq ? rows_of(q) : Rows{}, rows_of(k), rows_of(v), Hq ? rows_of(q_out) : Rows{}, data_error);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  });
}
