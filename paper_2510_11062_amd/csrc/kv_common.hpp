// What the calls on a paged cache share: the cache and its sequences as the kernels see them, and the checks on the host.
#pragma once

#include "common.hpp"

namespace atg {

constexpr int kMaxHeadDim = 256;

// at_grpo_rows as the kernels see it
struct Rows {
  void* data;
  int64_t ts, hs;
};

inline Rows rows_of(const at_grpo_rows* r) { return r ? Rows{r->data, r->token_stride, r->head_stride} : Rows{}; }

struct KvView {
  int Hk, D, page_shift, n_pages, n_seq, max_pages, n_group, max_prefix_pages;
  void *k, *v;
  const int32_t *pages, *length, *cu_q, *group_seq, *prefix_len, *prefix_pages;
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline int elem_size(int32_t dtype) { return dtype == AT_GRPO_BF16 ? 2 : 4; }

inline int check_head_dim(int32_t dtype, int32_t D) {
  if (dtype != AT_GRPO_F32 && dtype != AT_GRPO_BF16) return AT_GRPO_EUNSUPPORTED;
  if (D <= 0) return AT_GRPO_EINVAL;
  return D % 8 == 0 && D <= kMaxHeadDim ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

// 16-byte loads of a row's elements need its address and both strides to be multiples of 16 bytes.
inline int check_rows(const at_grpo_rows* r, int32_t dtype) {
  if (!r || !r->data || !aligned16(r->data)) return AT_GRPO_EINVAL;
  const int64_t step = 16 / elem_size(dtype);
  return r->token_stride % step == 0 && r->head_stride % step == 0 ? AT_GRPO_OK : AT_GRPO_EINVAL;
}

// Whether rows [n, H, D] of `a` and `b` share memory: exact where their strides are the same (views of one buffer that lie between each
// other's rows do not); with other strides they do where their ranges meet.
inline bool rows_meet(const at_grpo_rows& a, const at_grpo_rows& b, int64_t n, int64_t H, int64_t D, int elem) {
  const int64_t width = D * elem, apart = static_cast<int64_t>(reinterpret_cast<intptr_t>(b.data) - reinterpret_cast<intptr_t>(a.data));
  const auto range = [&](const at_grpo_rows& r, int64_t* lo, int64_t* hi) {      // of the rows' first bytes
    const int64_t t = (n - 1) * r.token_stride * elem, h = (H - 1) * r.head_stride * elem;
    *lo = (t < 0 ? t : 0) + (h < 0 ? h : 0);
    *hi = (t > 0 ? t : 0) + (h > 0 ? h : 0);
  };
  int64_t lo_a, hi_a, lo_b, hi_b;
  range(a, &lo_a, &hi_a);
  range(b, &lo_b, &hi_b);
  if (apart + lo_b >= hi_a + width || lo_a >= apart + hi_b + width) return false;
  if ((n > 1 && a.token_stride != b.token_stride) || (H > 1 && a.head_stride != b.head_stride)) return true;
  // Rows (t, h) of b and (t', h') of a are apart + i * outer + j * inner bytes from each other, i and j the differences of their numbers: for
  // each of the fewer i's the j's that bring that next to 0.
  const bool by_token = n < H;
  const int64_t outer = (by_token ? a.token_stride : a.head_stride) * elem, inner = (by_token ? a.head_stride : a.token_stride) * elem;
  const int64_t most = by_token ? n : H, other = by_token ? H : n;
  for (int64_t i = 1 - most; i < most; ++i) {
    const int64_t x = apart + i * outer, j = inner ? -x / inner : 0;
    for (int64_t y = j - 1; y <= j + 1; ++y) {
      const int64_t k = y <= -other ? 1 - other : y >= other ? other - 1 : y;
      if (x + k * inner < width && x + k * inner > -width) return true;
    }
  }
  return false;
}

// An output of rows that are read once may be its input itself, or lie apart from it.
inline int check_in_place(const at_grpo_rows* in, const at_grpo_rows* out, int64_t n, int64_t H, int64_t D, int32_t dtype) {
  if (in->data == out->data && (n == 1 || in->token_stride == out->token_stride) && (H == 1 || in->head_stride == out->head_stride)) return AT_GRPO_OK;
  return rows_meet(*in, *out, n, H, D, elem_size(dtype)) ? AT_GRPO_EINVAL : AT_GRPO_OK;
}

inline int check_kv_sizes(const at_grpo_kv* kv, int32_t n_tok) {
  if (!kv) return AT_GRPO_EINVAL;
  ATG_TRY(check_head_dim(kv->dtype, kv->D));
  if (kv->Hk <= 0 || kv->n_pages <= 0 || kv->n_seq < 0 || kv->max_pages < 0 || kv->n_group < 0 || kv->max_prefix_pages < 0 || n_tok < 0)
    return AT_GRPO_EINVAL;
  if (kv->page_size < 8 || kv->page_size > 65536 || (kv->page_size & (kv->page_size - 1))) return AT_GRPO_EUNSUPPORTED;
  const int64_t most = 0x7fffff00;       // places, rows of a call and units of the schedule are counted in 32 bits
  if (static_cast<int64_t>(kv->max_pages) * kv->page_size > most / 2 || static_cast<int64_t>(kv->max_prefix_pages) * kv->page_size > most / 2 ||
      static_cast<int64_t>(kv->n_seq) + kv->n_group > most / 2)
    return AT_GRPO_EUNSUPPORTED;
  if (static_cast<int64_t>(kv->Hk) * kv->page_size > (1 << 30) / kv->D) return AT_GRPO_EUNSUPPORTED;      // bytes of a page too
  return AT_GRPO_OK;
}

// Pointers are looked at only where there is something behind them.
inline int check_kv(const at_grpo_kv* kv, int32_t n_tok, KvView* out) {
  ATG_TRY(check_kv_sizes(kv, n_tok));
  if (!kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v)) return AT_GRPO_EINVAL;
  if (kv->n_seq > 0 && (!kv->length || (kv->max_pages > 0 && !kv->pages))) return AT_GRPO_EINVAL;
  if (!kv->cu_q && n_tok != kv->n_seq) return AT_GRPO_EINVAL;
  if (kv->n_group > 0 && (!kv->group_seq || !kv->prefix_len || (kv->max_prefix_pages > 0 && !kv->prefix_pages))) return AT_GRPO_EINVAL;
  int shift = 0;
  while ((1 << shift) < kv->page_size) ++shift;
  *out = KvView{kv->Hk, kv->D, shift, kv->n_pages, kv->n_seq, kv->max_pages, kv->n_group, kv->max_prefix_pages,
                kv->k, kv->v, kv->pages, kv->length, kv->cu_q, kv->group_seq, kv->prefix_len, kv->prefix_pages};
  return AT_GRPO_OK;
}

#ifdef __HIPCC__
// A launch's threads along one dimension are counted in 32 bits: workgroups of 256 of which there may be more than 2^24 stand in rows of 2^23, and
// those behind the last of them find that they have nothing to do.
inline dim3 grid_of(int64_t blocks) {
  const int64_t x = blocks < 1 << 23 ? blocks : 1 << 23;
  return dim3(static_cast<unsigned>(x), static_cast<unsigned>(ceil_div(blocks, x)));
}
__device__ __forceinline__ uint32_t flat_block() { return blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return bf16_to_f32(x); }

// How many of the rising a[0 .. n) are <= key, found by a whole wavefront, 64 entries at a time; between 0 and n whatever a holds.
__device__ __forceinline__ int wave_upper_bound(const int32_t* __restrict__ a, int n, int key) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  while (n > 64) {
    const int step = (n + 63) >> 6, at = lane * step;
    const int c = __popcll(__ballot(at < n && a[base + (at < n ? at : 0)] <= key));
    if (c == 0) return base;
    base += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  return base + __popcll(__ballot(lane < n && a[base + (lane < n ? lane : 0)] <= key));
}

__device__ __forceinline__ void raise_data_error(int32_t* word, int bits) {
  if (word && bits) atomicOr(word, bits);
}
#endif

}  // namespace atg
