// Attention of new tokens over a paged cache, the prompts of groups of candidates among it (gfx950).
//
//   out = sum_i p_i v_i / sum_i p_i,  p_i = exp(scale <q, k_i> - m)  over the visible tokens, with the running maximum m and sum of one pass.
//
// One wavefront per query and head: a lane scores a token, then the lanes own elements of the output.
#include "kv_common.hpp"

#include <math.h>

namespace atg {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void k_attend(KvView kv, int n_tok, int Hq, Rows q, float scale, int causal, Rows out, float* __restrict__ lse,
                                                int32_t* data_error) {
  __shared__ float q_lds[4][kMaxHeadDim];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (unit >= static_cast<int64_t>(n_tok) * Hq) return;
  const int t = static_cast<int>(unit / Hq), h = static_cast<int>(unit - static_cast<int64_t>(t) * Hq), hk = h / (Hq / kv.Hk), D = kv.D;
  int error = 0, s = t, q0 = t, q1 = t + 1;
  // an index that falls anywhere leaves nothing visible anywhere
  bool falls = false;
  if (kv.cu_q)
    for (int i = lane; i < kv.n_seq; i += 64) falls |= kv.cu_q[i] < 0 || kv.cu_q[i + 1] < kv.cu_q[i] || kv.cu_q[i + 1] > n_tok;
  if (kv.n_group)
    for (int i = lane; i < kv.n_group; i += 64)
      falls |= kv.group_seq[i] < 0 || kv.group_seq[i + 1] < kv.group_seq[i] || kv.group_seq[i + 1] > kv.n_seq;
  int own = 0, prefix = 0, g = 0;
  if (__any(falls)) {
    error = AT_GRPO_DATA_SEQLENS;
  } else {
    if (kv.cu_q) {
      s = wave_upper_bound(kv.cu_q, kv.n_seq + 1, t) - 1;
      if (s >= 0 && s < kv.n_seq) {
        q0 = kv.cu_q[s];
        q1 = kv.cu_q[s + 1];
      }
    }
    if (s >= 0 && s < kv.n_seq) {
      own = kv.length[s];
      if (own < 0 || own > (kv.max_pages << kv.page_shift)) {
        own = 0;
        error |= AT_GRPO_DATA_SEQLENS;
      }
      if (causal) own = max(0, own - (q1 - 1 - t));
      if (kv.n_group) {
        g = wave_upper_bound(kv.group_seq, kv.n_group + 1, s) - 1;
        if (g >= 0 && g < kv.n_group) {
          prefix = kv.prefix_len[g];
          if (prefix < 0 || prefix > (kv.max_prefix_pages << kv.page_shift)) {
            prefix = 0;
            error |= AT_GRPO_DATA_SEQLENS;
          }
        }
      }
    }
  }
  const T* qr = static_cast<const T*>(q.data) + t * q.ts + h * q.hs;
  for (int d = lane; d < D; d += 64) q_lds[wave][d] = to_f32(qr[d]) * scale;
  __builtin_amdgcn_wave_barrier();
  float acc[kMaxHeadDim / 64] = {}, m = -INFINITY, l = 0.f;
  for (int seg = 0; seg < 2; ++seg) {
    const int n = seg ? own : prefix;
    const int32_t* table = seg ? kv.pages + static_cast<int64_t>(s) * kv.max_pages : kv.prefix_pages + static_cast<int64_t>(g) * kv.max_prefix_pages;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const int i = i0 + lane;
      int64_t row = -1;
      float z = -INFINITY;
      if (i < n) {
        const int page = table[i >> kv.page_shift];
        if (static_cast<unsigned>(page) < static_cast<unsigned>(kv.n_pages)) {
          row = (((static_cast<int64_t>(page) * kv.Hk + hk) << kv.page_shift) + (i & ((1 << kv.page_shift) - 1))) * D;
          const T* kr = static_cast<const T*>(kv.k) + row;
          z = 0.f;
          for (int d = 0; d < D; ++d) z = fmaf(q_lds[wave][d], to_f32(kr[d]), z);
        } else {
          error |= AT_GRPO_DATA_PAGE;
        }
      }
      float top = z;
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.f : now, keep = expf(m - ref), p = row >= 0 ? expf(z - ref) : 0.f;
      float sum = p;
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      l = l * keep + sum;
      m = now;
      for (int e = 0; e < kMaxHeadDim / 64; ++e) acc[e] *= keep;
      for (int j = 0; j < min(64, n - i0); ++j) {
        const int64_t r = __shfl(row, j, 64);
        const float pj = __shfl(p, j, 64);
        if (r < 0) continue;
        const T* vr = static_cast<const T*>(kv.v) + r;
        for (int e = 0; e < kMaxHeadDim / 64; ++e)
          if (e * 64 + lane < D) acc[e] = fmaf(pj, to_f32(vr[e * 64 + lane]), acc[e]);
      }
    }
  }
  raise_data_error(data_error, error);
  T* o = static_cast<T*>(out.data) + t * out.ts + h * out.hs;
  for (int e = 0; e < kMaxHeadDim / 64; ++e)
    if (e * 64 + lane < D) o[e * 64 + lane] = from_f32<T>(l == 0.f ? 0.f : acc[e] / l);
  if (lse && lane == 0) lse[unit] = l == 0.f ? -INFINITY : m + logf(l);
}

size_t workspace_of(const at_grpo_kv*, int32_t, int32_t, int32_t) {
  WsAlloc ws(nullptr);
  ws.take<int32_t>(64);
  return ws.bytes();
}

int check_sizes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  ATG_TRY(check_kv_sizes(kv, n_tok));
  if (Hq <= 0 || Hq % kv->Hk || max_q < 1) return AT_GRPO_EINVAL;
  return static_cast<int64_t>(n_tok) * Hq <= 0x7fffff00 ? AT_GRPO_OK : AT_GRPO_EUNSUPPORTED;
}

}  // namespace
}  // namespace atg

using namespace atg;

extern "C" size_t at_grpo_prefix_attention_workspace_bytes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  return check_sizes(kv, n_tok, Hq, max_q) == AT_GRPO_OK ? workspace_of(kv, n_tok, Hq, max_q) : 0;
}

extern "C" int at_grpo_prefix_attention(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, const at_grpo_rows* q, float scale, int32_t causal,
                                        int32_t max_q, const at_grpo_rows* out, float* lse, int32_t* data_error, void* workspace,
                                        size_t workspace_bytes, void* hip_stream) {
  ATG_TRY(check_sizes(kv, n_tok, Hq, max_q));
  if (!(scale > 0.f) || !isfinite(scale)) return AT_GRPO_EINVAL;
  KvView view;
  ATG_TRY(check_kv(kv, n_tok, &view));
  if (n_tok == 0) return AT_GRPO_OK;
  ATG_TRY(check_rows(q, kv->dtype));
  ATG_TRY(check_rows(out, kv->dtype));
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < workspace_of(kv, n_tok, Hq, max_q)) return AT_GRPO_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const unsigned blocks = static_cast<unsigned>(ceil_div(static_cast<int64_t>(n_tok) * Hq, 4));
  ProfScope ps(PROF_ATTENTION, s);
  auto k = kv->dtype == AT_GRPO_BF16 ? k_attend<bf16_t> : k_attend<float>;
  hipLaunchKernelGGL(k, dim3(blocks), dim3(256), 0, s, view, n_tok, Hq, rows_of(q), scale, causal, rows_of(out), lse, data_error);
  ATG_LAUNCH_CHECK();
  return AT_GRPO_OK;
}
