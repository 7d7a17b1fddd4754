// Attention of trees of drafted tokens: each sees its sequence and those of the new tokens that its bits name.
#include "attention.hpp"

using namespace atg;

extern "C" size_t at_grpo_tree_attention_workspace_bytes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q) {
  return attention_workspace<true>(kv, n_tok, Hq, max_q);
}

extern "C" int at_grpo_tree_attention(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, const at_grpo_rows* q, const uint64_t* ancestors, float scale,
                                      int32_t max_q, const at_grpo_rows* out, float* lse, int32_t* data_error, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
  return attend<true>(kv, n_tok, Hq, q, ancestors, scale, 0, max_q, out, lse, data_error, workspace, workspace_bytes, hip_stream);
}
