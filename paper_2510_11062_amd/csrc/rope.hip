// Queries and keys of a layer: norm of every head's row, rotation by position, the gradient of both, and the same on the way into a
// paged cache (gfx950).
//
// A row of D elements x with weight w at position p:  u = x r w, r = 1 / sqrt(mean(x^2) + eps), then the pairs (a, b) of the first
// rot_dim elements turn by the table's angle: y_a = c u_a - s u_b, y_b = c u_b + s u_a.  The gradient turns back, then with n = x r and
// g' = g w:  dx = r (g' - n mean(g' n)),  dw = sum over rows of g n.  All sums are fp32.
//
// Bound by memory: two rows' bytes forward, three backward.  A row belongs to LANES neighbouring lanes with four pairs each, so that a
// pair never leaves its lane in either layout.
#include "kv_common.hpp"

#include <math.h>

namespace atg {

namespace {

struct Layer {
  int D, half, interleaved, n_pos;   // half: pairs that turn
  float eps;
  const float* table;
  const void *qw, *kw;
};

struct Pairs {
  float a[4], b[4];
};

// Where the pairs 4 l .. 4 l + 3 of a row lie.
struct Places {
  int at_a[4], at_b[4];
};

__device__ __forceinline__ Places places_of(const Layer& L, int l) {
  Places p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = 4 * l + i;
    const bool apart = !L.interleaved && pair < L.half;
    p.at_a[i] = apart ? pair : 2 * pair;
    p.at_b[i] = apart ? pair + L.half : 2 * pair + 1;
  }
  return p;
}

template <typename T>
__device__ __forceinline__ Pairs load_pairs(const T* row, const Places& p) {
  Pairs x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] = to_f32(row[p.at_a[i]]);
    x.b[i] = to_f32(row[p.at_b[i]]);
  }
  return x;
}

template <typename T>
__device__ __forceinline__ void store_pairs(T* row, const Places& p, const Pairs& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    row[p.at_a[i]] = from_f32<T>(x.a[i]);
    row[p.at_b[i]] = from_f32<T>(x.b[i]);
  }
}

// Cosines and sines of a lane's pairs; 1 and 0 behind the last that turns.
__device__ __forceinline__ Pairs load_turn(const Layer& L, int l, int position) {
  Pairs t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = 4 * l + i;
    const bool turns = pair < L.half;
    const float* e = L.table + 2 * (static_cast<int64_t>(position) * L.half + pair);
    t.a[i] = turns ? e[0] : 1.f;
    t.b[i] = turns ? e[1] : 0.f;
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
  return 1.f / sqrtf(row_sum<LANES>(ss) / static_cast<float>(L.D) + L.eps);
}

// Where a new token belongs: its position, and its place in the cache (rows between its heads are page_size * D apart).
struct Spot {
  int position;      // -1: nowhere
  int64_t at;
};

__device__ __forceinline__ Spot find_spot(const KvView& kv, int n_pos, int t, int32_t* data_error) {
  Spot spot{-1, 0};
  int error = 0, s = t, q0 = t, q1 = t + 1;
  if (kv.cu_q) {
    s = wave_upper_bound(kv.cu_q, kv.n_seq + 1, t) - 1;
    if (s >= 0 && s < kv.n_seq) {
      q0 = kv.cu_q[s];
      q1 = kv.cu_q[s + 1];
    }
  }
  int place = -1;
  if (s < 0 || s >= kv.n_seq || q0 < 0 || q0 > t || q1 <= t) {
    error = AT_GRPO_DATA_SEQLENS;
  } else {
    const int length = kv.length[s], most = kv.max_pages << kv.page_shift;
    if (length < 0 || length > most || q1 - q0 > length) error = AT_GRPO_DATA_SEQLENS;
    else place = length - (q1 - t);
  }
  int prefix = 0;
  if (place >= 0 && kv.n_group > 0) {
    const int g = wave_upper_bound(kv.group_seq, kv.n_group + 1, s) - 1;
    if (g >= 0 && g < kv.n_group) {
      prefix = kv.prefix_len[g];
      if (prefix < 0 || prefix > (kv.max_prefix_pages << kv.page_shift)) {
        error = AT_GRPO_DATA_SEQLENS;
        place = -1;
      }
    }
  }
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

// The heads of one token that a wavefront takes: part, part + parts, .. of groups of 64 / LANES heads.
template <typename T, int LANES>
__device__ void rotate_rows(const Layer& L, const T* src, int64_t src_hs, T* dst, int64_t dst_hs, int H, const void* weight, const Pairs& turn,
                            const Places& p, bool zero, int part, int parts) {
  constexpr int G = 64 / LANES;
  const int l = threadIdx.x & (LANES - 1), grp = (threadIdx.x & 63) / LANES;
  const bool mine = 8 * l < L.D;
  Pairs w{{1.f, 1.f, 1.f, 1.f}, {1.f, 1.f, 1.f, 1.f}};
  if (weight && mine) w = load_pairs(static_cast<const T*>(weight), p);
  for (int h0 = part * G; h0 < H; h0 += parts * G) {
    const int h = h0 + grp;
    const bool on = mine && h < H;
    Pairs x{};
    if (on && !zero) x = load_pairs(src + h * src_hs, p);
    if (weight) {
      const float r = inverse_size<LANES>(x, L);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x.a[i] *= r * w.a[i];
        x.b[i] *= r * w.b[i];
      }
    }
    Pairs y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y.a[i] = fmaf(x.a[i], turn.a[i], -x.b[i] * turn.b[i]);
      y.b[i] = fmaf(x.b[i], turn.a[i], x.a[i] * turn.b[i]);
    }
    if (zero) y = Pairs{};
    if (on) store_pairs(dst + h * dst_hs, p, y);
  }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_norm_rope(Layer L, int n_tok, int parts, int Hq, int Hk, Rows q, Rows k, const int32_t* __restrict__ position,
                                                   Rows q_out, Rows k_out, int32_t* data_error) {
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = unit / parts, part = unit - t * parts, l = threadIdx.x & (LANES - 1);
  if (t >= n_tok) return;
  const int pos = L.half ? position[t] : 0;
  const bool bad = L.half && static_cast<unsigned>(pos) >= static_cast<unsigned>(L.n_pos);
  if (bad && (threadIdx.x & 63) == 0) raise_data_error(data_error, AT_GRPO_DATA_POSITION);
  const Places p = places_of(L, l);
  Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
  if (!bad && L.half) turn = load_turn(L, l, pos);
  if (Hq) rotate_rows<T, LANES>(L, static_cast<const T*>(q.data) + t * q.ts, q.hs, static_cast<T*>(q_out.data) + t * q_out.ts, q_out.hs, Hq, L.qw, turn, p,
                                bad, part, parts);
  if (Hk) rotate_rows<T, LANES>(L, static_cast<const T*>(k.data) + t * k.ts, k.hs, static_cast<T*>(k_out.data) + t * k_out.ts, k_out.hs, Hk, L.kw, turn, p,
                                bad, part, parts);
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_kv_append(KvView kv, Layer L, int n_tok, int parts, int Hq, Rows q, Rows k, Rows v, Rows q_out,
                                                   int32_t* data_error) {
  constexpr int G = 64 / LANES;
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = unit / parts, part = unit - t * parts, l = threadIdx.x & (LANES - 1), grp = (threadIdx.x & 63) / LANES;
  if (t >= n_tok) return;
  const Spot spot = find_spot(kv, L.half ? L.n_pos : -1, t, part == 0 ? data_error : nullptr);
  const bool bad = spot.position < 0;
  const Places p = places_of(L, l);
  Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
  if (!bad && L.half) turn = load_turn(L, l, spot.position);
  if (Hq) rotate_rows<T, LANES>(L, static_cast<const T*>(q.data) + t * q.ts, q.hs, static_cast<T*>(q_out.data) + t * q_out.ts, q_out.hs, Hq, L.qw, turn, p,
                                bad, part, parts);
  if (bad) return;
  const int64_t hs = static_cast<int64_t>(kv.D) << kv.page_shift;
  rotate_rows<T, LANES>(L, static_cast<const T*>(k.data) + t * k.ts, k.hs, static_cast<T*>(kv.k) + spot.at, hs, kv.Hk, L.kw, turn, p, false, part, parts);
  if (8 * l >= L.D) return;
  for (int h = part * G + grp; h < kv.Hk; h += parts * G) {
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(v.data) + t * v.ts + h * v.hs + 8 * l);
    uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(kv.v) + spot.at + h * hs + 8 * l);
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) to[i] = from[i];
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
constexpr int kGradBlocks = 1024;

template <typename T, int LANES>
__device__ void rotate_rows_back(const Layer& L, const T* dy, int64_t dy_hs, const T* src, int64_t src_hs, T* dst, int64_t dst_hs, int H, const void* weight,
                                 const Pairs& turn, const Places& p, bool zero, int part, int parts, Pairs& dw) {
  constexpr int G = 64 / LANES;
  const int l = threadIdx.x & (LANES - 1), grp = (threadIdx.x & 63) / LANES;
  const bool mine = 8 * l < L.D;
  Pairs w{};
  if (weight && mine) w = load_pairs(static_cast<const T*>(weight), p);
  for (int h0 = part * G; h0 < H; h0 += parts * G) {
    const int h = h0 + grp;
    const bool on = mine && h < H;
    Pairs x{}, g{};
    if (on && !zero) {
      const Pairs d = load_pairs(dy + h * dy_hs, p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g.a[i] = fmaf(d.a[i], turn.a[i], d.b[i] * turn.b[i]);
        g.b[i] = fmaf(d.b[i], turn.a[i], -d.a[i] * turn.b[i]);
      }
      if (weight) x = load_pairs(src + h * src_hs, p);
    }
    if (weight) {
      const float r = inverse_size<LANES>(x, L);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x.a[i] *= r;
        x.b[i] *= r;
        if (on && !zero) {      // lanes without a row would add 0 times the size of no row
          dw.a[i] = fmaf(g.a[i], x.a[i], dw.a[i]);
          dw.b[i] = fmaf(g.b[i], x.b[i], dw.b[i]);
        }
        g.a[i] *= w.a[i];
        g.b[i] *= w.b[i];
        dot = fmaf(g.a[i], x.a[i], fmaf(g.b[i], x.b[i], dot));
      }
      const float mean = row_sum<LANES>(dot) / static_cast<float>(L.D);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g.a[i] = r * fmaf(-x.a[i], mean, g.a[i]);
        g.b[i] = r * fmaf(-x.b[i], mean, g.b[i]);
      }
    }
    if (zero) g = Pairs{};
    if (on) store_pairs(dst + h * dst_hs, p, g);
  }
}

// The rows of one kind (0 queries, 1 keys) that a workgroup's lanes added up, as one row of partial sums.
template <int LANES>
__device__ void store_partial(const Layer& L, Pairs dw, const Places& p, float* lds, float* __restrict__ partial) {
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
      lds[wave * kMaxHeadDim + p.at_a[i]] = dw.a[i];
      lds[wave * kMaxHeadDim + p.at_b[i]] = dw.b[i];
    }
  }
  __syncthreads();
  const int d = threadIdx.x;
  if (d < L.D) partial[d] = (lds[d] + lds[kMaxHeadDim + d]) + (lds[2 * kMaxHeadDim + d] + lds[3 * kMaxHeadDim + d]);
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_norm_rope_bwd(Layer L, int n_tok, int parts, int Hq, int Hk, Rows dq_out, Rows dk_out, Rows q, Rows k,
                                                       const int32_t* __restrict__ position, Rows dq, Rows dk, float* __restrict__ partial,
                                                       int32_t* data_error) {
  __shared__ float lds[4 * kMaxHeadDim];
  const int l = threadIdx.x & (LANES - 1);
  const Places p = places_of(L, l);
  Pairs dwq{}, dwk{};
  const int64_t units = static_cast<int64_t>(n_tok) * parts;
  for (int64_t unit = blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += gridDim.x * 4) {
    const int64_t t = unit / parts;
    const int part = static_cast<int>(unit - t * parts);
    const int pos = L.half ? position[t] : 0;
    const bool bad = L.half && static_cast<unsigned>(pos) >= static_cast<unsigned>(L.n_pos);
    if (bad && part == 0 && (threadIdx.x & 63) == 0) raise_data_error(data_error, AT_GRPO_DATA_POSITION);
    Pairs turn{{1.f, 1.f, 1.f, 1.f}, {}};
    if (!bad && L.half) turn = load_turn(L, l, pos);
    if (Hq)
      rotate_rows_back<T, LANES>(L, static_cast<const T*>(dq_out.data) + t * dq_out.ts, dq_out.hs, static_cast<const T*>(q.data) + t * q.ts, q.hs,
                                 static_cast<T*>(dq.data) + t * dq.ts, dq.hs, Hq, L.qw, turn, p, bad, part, parts, dwq);
    if (Hk)
      rotate_rows_back<T, LANES>(L, static_cast<const T*>(dk_out.data) + t * dk_out.ts, dk_out.hs, static_cast<const T*>(k.data) + t * k.ts, k.hs,
                                 static_cast<T*>(dk.data) + t * dk.ts, dk.hs, Hk, L.kw, turn, p, bad, part, parts, dwk);
  }
  if (L.qw) store_partial<LANES>(L, dwq, p, lds, partial + static_cast<int64_t>(blockIdx.x) * L.D);
  if (L.kw) store_partial<LANES>(L, dwk, p, lds, partial + (static_cast<int64_t>(kGradBlocks) + blockIdx.x) * L.D);
}

// d_weight[d] = sum over the workgroups' rows, 16 elements a workgroup, in 64 bits
__global__ __launch_bounds__(256) void k_weight_grad(int D, int blocks, const float* __restrict__ partial, float* dq_weight, float* dk_weight) {
  __shared__ double red[16][17];
  const int c = threadIdx.x & 15, slice = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
  float* out = blockIdx.y ? dk_weight : dq_weight;
  if (!out) return;
  const float* rows = partial + static_cast<int64_t>(blockIdx.y) * kGradBlocks * D;
  double s = 0.0;
  if (d < D)
    for (int b = slice; b < blocks; b += 16) s += static_cast<double>(rows[static_cast<int64_t>(b) * D + d]);
  red[slice][c] = s;
  __syncthreads();
  if (slice == 0 && d < D) {
    for (int i = 1; i < 16; ++i) s += red[i][c];
    out[d] = static_cast<float>(s);
  }
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
  *out = Layer{a->D, a->rot_dim / 2, a->layout, a->n_pos, a->eps, a->table, a->q_weight, a->k_weight};
  return AT_GRPO_OK;
}

int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// Few tokens are shared by several wavefronts each, so that the chip has work: about 4096 wavefronts, or all groups of heads.
int parts_of(int n_tok, int most_heads, int lanes) {
  const int groups = static_cast<int>(ceil_div(most_heads, 64 / lanes));
  const int64_t want = ceil_div(4096, n_tok > 0 ? n_tok : 1);
  return static_cast<int>(want < groups ? want : groups);
}

template <typename F>
int by_type_and_lanes(int32_t dtype, int lanes, F f) {
  if (dtype == AT_GRPO_BF16) return lanes == 8 ? f(bf16_t{}, std::integral_constant<int, 8>{}) : lanes == 16 ? f(bf16_t{}, std::integral_constant<int, 16>{}) : f(bf16_t{}, std::integral_constant<int, 32>{});
  return lanes == 8 ? f(0.f, std::integral_constant<int, 8>{}) : lanes == 16 ? f(0.f, std::integral_constant<int, 16>{}) : f(0.f, std::integral_constant<int, 32>{});
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
  if (n_tok < 0 || Hq < 0 || Hk < 0 || (Hq == 0 && Hk == 0)) return AT_GRPO_EINVAL;
  if (n_tok == 0) return AT_GRPO_OK;
  if (L.half && !position) return AT_GRPO_EINVAL;
  if (Hq) ATG_TRY(check_rows(q, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q_out, layer->dtype));
  if (Hk) ATG_TRY(check_rows(k, layer->dtype));
  if (Hk) ATG_TRY(check_rows(k_out, layer->dtype));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int lanes = lanes_of(L.D), parts = parts_of(n_tok, Hq > Hk ? Hq : Hk, lanes);
  const int64_t blocks = ceil_div(static_cast<int64_t>(n_tok) * parts, 4);
  if (blocks > 0x7fffffff || static_cast<int64_t>(n_tok) * parts > 0x7fffffff) return AT_GRPO_EUNSUPPORTED;
  ProfScope ps(PROF_ROPE, s);
  return by_type_and_lanes(layer->dtype, lanes, [&](auto t, auto n) -> int {
    hipLaunchKernelGGL((k_norm_rope<decltype(t), decltype(n)::value>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, L, n_tok, parts, Hq, Hk,
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
  if (n_tok < 0 || Hq < 0 || Hk < 0 || (Hq == 0 && Hk == 0)) return AT_GRPO_EINVAL;
  if (!Hq) L.qw = nullptr;
  if (!Hk) L.kw = nullptr;
  if ((L.qw && !dq_weight) || (L.kw && !dk_weight)) return AT_GRPO_EINVAL;
  if (n_tok > 0) {
    if (L.half && !position) return AT_GRPO_EINVAL;
    if (Hq) {
      ATG_TRY(check_rows(dq_out, layer->dtype));
      ATG_TRY(check_rows(dq, layer->dtype));
      if (L.qw) ATG_TRY(check_rows(q, layer->dtype));
    }
    if (Hk) {
      ATG_TRY(check_rows(dk_out, layer->dtype));
      ATG_TRY(check_rows(dk, layer->dtype));
      if (L.kw) ATG_TRY(check_rows(k, layer->dtype));
    }
  }
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < qk_norm_rope_bwd_workspace()) return AT_GRPO_EWORKSPACE;
  float* partial = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int lanes = lanes_of(L.D), parts = parts_of(n_tok, Hq > Hk ? Hq : Hk, lanes);
  const int64_t want = ceil_div(static_cast<int64_t>(n_tok) * parts, 4);
  const unsigned blocks = static_cast<unsigned>(want > kGradBlocks ? kGradBlocks : want < 1 ? 1 : want);
  const bool rows = n_tok > 0;
  ProfScope ps(PROF_ROPE, s);
  ATG_TRY(by_type_and_lanes(layer->dtype, lanes, [&](auto t, auto n) -> int {
    hipLaunchKernelGGL((k_norm_rope_bwd<decltype(t), decltype(n)::value>), dim3(blocks), dim3(256), 0, s, L, n_tok, parts, Hq, Hk,
                       rows && Hq ? rows_of(dq_out) : Rows{}, rows && Hk ? rows_of(dk_out) : Rows{}, rows && L.qw ? rows_of(q) : Rows{},
                       rows && L.kw ? rows_of(k) : Rows{}, position, rows && Hq ? rows_of(dq) : Rows{}, rows && Hk ? rows_of(dk) : Rows{}, partial,
                       data_error);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  }));
  if (L.qw || L.kw) {
    hipLaunchKernelGGL(k_weight_grad, dim3(static_cast<unsigned>(ceil_div(L.D, 16)), 2), dim3(256), 0, s, L.D, static_cast<int>(blocks), partial,
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
  if (kv->dtype != layer->dtype || kv->D != layer->D || Hq < 0) return AT_GRPO_EINVAL;
  if (n_tok == 0) return AT_GRPO_OK;
  ATG_TRY(check_rows(k, layer->dtype));
  ATG_TRY(check_rows(v, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q, layer->dtype));
  if (Hq) ATG_TRY(check_rows(q_out, layer->dtype));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int lanes = lanes_of(L.D), parts = parts_of(n_tok, Hq > kv->Hk ? Hq : kv->Hk, lanes);
  if (static_cast<int64_t>(n_tok) * parts > 0x7fffffff) return AT_GRPO_EUNSUPPORTED;
  const unsigned blocks = static_cast<unsigned>(ceil_div(static_cast<int64_t>(n_tok) * parts, 4));
  ProfScope ps(PROF_ROPE, s);
  return by_type_and_lanes(layer->dtype, lanes, [&](auto t, auto n) -> int {
    hipLaunchKernelGGL((k_kv_append<decltype(t), decltype(n)::value>), dim3(blocks), dim3(256), 0, s, view, L, n_tok, parts, Hq,
                       Hq ? rows_of(q) : Rows{}, rows_of(k), rows_of(v), Hq ? rows_of(q_out) : Rows{}, data_error);
    ATG_LAUNCH_CHECK();
    return AT_GRPO_OK;
  });
}
