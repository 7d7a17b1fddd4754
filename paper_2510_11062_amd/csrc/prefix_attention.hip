// Attention of new tokens in their order: each sees those in front of it, or all.
#include "attention.hpp"

using namespace atg;

extern "C" size_t at_grpo_prefix_attention_workspace_bytes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  return attention_workspace<false>(kv, n_tok, Hq, max_q);
}

extern "C" int at_grpo_prefix_attention(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, const at_grpo_rows* q, float scale, int32_t causal,
                                        int32_t max_q, const at_grpo_rows* out, float* lse, int32_t* data_error, void* workspace,
                                        size_t workspace_bytes, void* hip_stream) {
  return attend<false>(kv, n_tok, Hq, q, nullptr, scale, causal, max_q, out, lse, data_error, workspace, workspace_bytes, hip_stream);
}
