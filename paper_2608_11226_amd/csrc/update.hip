// C entry points of the update side of a GRPO step: token log probabilities and their gradient, the clipped group
// loss, embedding lookup and its gradient.  They need no context: buffers and workspaces are the caller's, and the
// stream is an argument.
#include "update_checks.h"

#include <algorithm>

using namespace rollout;

namespace {

constexpr int32_t kMaxVocab = 1 << 30, kMaxRows = 1 << 30;

// what both directions of the log probabilities ask of a matrix of logits
rollout_status check_rows(const void* z, int32_t dtype, int64_t stride, int32_t rows, int32_t vocab, float temperature) {
  if (!is_float_type(dtype)) return fail(ROLLOUT_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
  if (rows < 1 || vocab < 1) return fail(ROLLOUT_EINVAL, "n_rows and vocab must be >= 1");
  if (rows > kMaxRows || vocab > kMaxVocab) return fail(ROLLOUT_EUNSUPPORTED, "n_rows or vocab above 2^30");
  if (stride < vocab) return fail(ROLLOUT_EINVAL, "row_stride must be at least vocab");
  if (stride > INT64_MAX / 8 / rows) return fail(ROLLOUT_EINVAL, "row_stride too large");
  if (!z) return fail(ROLLOUT_EINVAL, "logits must be non-NULL");
  if (!aligned_to(z, elem_bytes(dtype))) return fail(ROLLOUT_EINVAL, "logits are not aligned to their type");
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite((float)(2.0 / (double)temperature)))
    return fail(ROLLOUT_EINVAL, "temperature must be > 0, and its reciprocal finite");
  return ROLLOUT_OK;
}

// what lookup and gradient ask of a table and a matrix of rows
rollout_status check_table(int32_t table_dtype, int32_t row_dtype, int32_t vocab, int32_t dim, int32_t n, float scale) {
  if (!is_float_type(table_dtype) || !is_float_type(row_dtype)) return fail(ROLLOUT_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
  if (vocab < 1 || dim < 1 || n < 1) return fail(ROLLOUT_EINVAL, "vocab, dim and n_tokens must be >= 1");
  if (vocab > kMaxVocab || dim > kMaxVocab) return fail(ROLLOUT_EUNSUPPORTED, "vocab or dim above 2^30");
  if (n > kMaxEmbeddingTokens) return fail(ROLLOUT_EUNSUPPORTED, "more than 2^28 tokens");
  if (!std::isfinite(scale)) return fail(ROLLOUT_EINVAL, "scale must be finite");
  return ROLLOUT_OK;
}

}  // namespace

extern "C" {

rollout_status rollout_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  if (n_rows < 1 || vocab < 1) return fail(ROLLOUT_EINVAL, "n_rows and vocab must be >= 1");
  if (n_rows > kMaxRows || vocab > kMaxVocab) return fail(ROLLOUT_EUNSUPPORTED, "n_rows or vocab above 2^30");
  if (n_top < 0 || n_top > kMaxTop || n_top > vocab) return fail(ROLLOUT_EINVAL, "n_top must be in [0, 32] and at most vocab");
  if (n_top && vocab > kMaxTopVocab) return fail(ROLLOUT_EUNSUPPORTED, "alternatives of more than 327,680 ids");
  *h_bytes = logprobs_workspace(n_rows, vocab, n_top);
  return ROLLOUT_OK;
}

rollout_status rollout_token_logprobs(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows,
                                      int32_t vocab, float temperature, const int32_t* d_tokens, int32_t n_top,
                                      float* d_logp, float* d_entropy, float* d_stats, int32_t* d_top_ids,
                                      float* d_top_logp, void* d_workspace, uint64_t workspace_bytes,
                                      void* hip_stream) {
  Range range("rollout_token_logprobs");
  rollout_status st = check_rows(d_logits, dtype, row_stride, n_rows, vocab, temperature);
  if (st != ROLLOUT_OK) return st;
  uint64_t need = 0;
  st = rollout_token_logprobs_workspace(n_rows, vocab, n_top, &need);
  if (st != ROLLOUT_OK) return st;
  if (n_top && (!d_top_ids || !d_top_logp)) return fail(ROLLOUT_EINVAL, "alternatives asked for without their outputs");
  if (!d_tokens && d_logp) return fail(ROLLOUT_EINVAL, "log probabilities asked for without tokens");
  if (!d_logp && !d_entropy && !d_stats && !n_top) return fail(ROLLOUT_EINVAL, "no output asked for");
  st = check_workspace(d_workspace, workspace_bytes, need);
  if (st != ROLLOUT_OK) return st;
  st = check_words({d_tokens, d_logp, d_entropy, d_stats, n_top ? d_top_ids : nullptr, n_top ? d_top_logp : nullptr});
  if (st != ROLLOUT_OK) return st;
  const size_t es = elem_bytes(dtype), n = n_rows;
  st = check_apart({{"d_logp", d_logp, 4 * n}, {"d_entropy", d_entropy, 4 * n}, {"d_stats", d_stats, 8 * n},
                    {"d_top_ids", d_top_ids, 4 * n * n_top}, {"d_top_logp", d_top_logp, 4 * n * n_top},
                    {"the workspace", d_workspace, need}},
                   {{"the logits", d_logits, vocab * es, n, row_stride * es}, {"d_tokens", d_tokens, 4 * n}});
  if (st != ROLLOUT_OK) return st;
  st = check_stream(hip_stream);
  if (st != ROLLOUT_OK) return st;
  const LogprobArgs a = {d_logits, row_stride, n_rows, vocab, temperature, d_tokens, n_top,
                         d_logp, d_entropy, d_stats, d_top_ids, d_top_logp};
  return launched(launch_logprobs((hipStream_t)hip_stream, dtype, a, d_workspace), "token logprobs");
}

rollout_status rollout_token_logprobs_backward(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows,
                                               int32_t vocab, float temperature, const int32_t* d_tokens,
                                               const float* d_stats, const float* d_entropy, const float* d_grad_logp,
                                               const float* d_grad_entropy, void* d_grad_logits, int64_t grad_stride,
                                               void* hip_stream) {
  Range range("rollout_token_logprobs_backward");
  rollout_status st = check_rows(d_logits, dtype, row_stride, n_rows, vocab, temperature);
  if (st != ROLLOUT_OK) return st;
  if (!d_tokens || !d_stats || !d_grad_logp || !d_grad_logits) return fail(ROLLOUT_EINVAL, "NULL buffer");
  if (d_grad_entropy && !d_entropy) return fail(ROLLOUT_EINVAL, "a gradient of the entropies needs the entropies");
  if (grad_stride < vocab) return fail(ROLLOUT_EINVAL, "grad_stride must be at least vocab");
  if (grad_stride > INT64_MAX / 8 / n_rows) return fail(ROLLOUT_EINVAL, "grad_stride too large");
  const size_t es = elem_bytes(dtype);
  if (!aligned_to(d_grad_logits, es)) return fail(ROLLOUT_EINVAL, "gradients are not aligned to their type");
  const bool in_place = d_grad_logits == d_logits && grad_stride == row_stride;
  if (!in_place && overlap(d_logits, ((size_t)(n_rows - 1) * row_stride + vocab) * es, d_grad_logits,
                           ((size_t)(n_rows - 1) * grad_stride + vocab) * es))
    return fail(ROLLOUT_EINVAL, "the gradients overlap the logits without being in their place");
  const size_t n = n_rows;
  const float* entropy = d_grad_entropy ? d_entropy : nullptr;  // not read otherwise
  st = check_words({d_tokens, d_stats, entropy, d_grad_logp, d_grad_entropy});
  if (st != ROLLOUT_OK) return st;
  st = check_apart({{"d_grad_logits", d_grad_logits, vocab * es, n, grad_stride * es}},
                   {{"d_tokens", d_tokens, 4 * n}, {"d_stats", d_stats, 8 * n}, {"d_entropy", entropy, 4 * n},
                    {"d_grad_logp", d_grad_logp, 4 * n}, {"d_grad_entropy", d_grad_entropy, 4 * n}});
  if (st != ROLLOUT_OK) return st;
  st = check_stream(hip_stream);
  if (st != ROLLOUT_OK) return st;
  const LogprobGradArgs a = {d_logits, row_stride, n_rows, vocab, temperature, d_tokens, d_stats,
                             d_entropy, d_grad_logp, d_grad_entropy, d_grad_logits, grad_stride};
  return launched(launch_logprobs_backward((hipStream_t)hip_stream, dtype, a), "token logprobs backward");
}

rollout_status grpo_policy_loss_workspace(int32_t n_seqs, int32_t max_len, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  if (n_seqs < 1 || max_len < 1) return fail(ROLLOUT_EINVAL, "n_seqs and max_len must be >= 1");
  if ((int64_t)n_seqs * max_len > INT32_MAX) return fail(ROLLOUT_EUNSUPPORTED, "more than 2^31 - 1 tokens");
  *h_bytes = policy_loss_workspace(n_seqs, max_len);
  return ROLLOUT_OK;
}

rollout_status grpo_policy_loss(const float* d_logp, const float* d_old_logp, const float* d_ref_logp,
                                const float* d_entropy, const float* d_adv, const int32_t* d_lengths, int32_t n_seqs,
                                int32_t max_len, float clip_low, float clip_high, float kl_coef, float entropy_coef,
                                int32_t mean, float* d_loss, float* d_stats, float* d_grad_logp, float* d_grad_entropy,
                                void* d_workspace, uint64_t workspace_bytes, void* hip_stream) {
  Range range("grpo_policy_loss");
  uint64_t need = 0;
  rollout_status st = grpo_policy_loss_workspace(n_seqs, max_len, &need);
  if (st != ROLLOUT_OK) return st;
  if (!d_logp || !d_adv) return fail(ROLLOUT_EINVAL, "log probabilities and advantages must be non-NULL");
  if (!(clip_low >= 0.f && clip_low <= 1.f)) return fail(ROLLOUT_EINVAL, "clip_low must be in [0, 1]");
  if (!(clip_high >= 0.f) || !std::isfinite(clip_high)) return fail(ROLLOUT_EINVAL, "clip_high must be >= 0");
  if (!std::isfinite(kl_coef) || !std::isfinite(entropy_coef)) return fail(ROLLOUT_EINVAL, "coefficients must be finite");
  if (kl_coef != 0.f && !d_ref_logp) return fail(ROLLOUT_EINVAL, "kl_coef without reference log probabilities");
  if ((entropy_coef != 0.f || d_grad_entropy) && !d_entropy) return fail(ROLLOUT_EINVAL, "an entropy term without entropies");
  if (mean != ROLLOUT_MEAN_SEQUENCE && mean != ROLLOUT_MEAN_TOKEN && mean != ROLLOUT_MEAN_FIXED)
    return fail(ROLLOUT_EINVAL, "mean must be 0 (sequence), 1 (token) or 2 (fixed)");
  if (!d_loss && !d_stats && !d_grad_logp && !d_grad_entropy) return fail(ROLLOUT_EINVAL, "no output asked for");
  const size_t whole = (size_t)n_seqs * max_len * 4;
  if (d_grad_logp && d_grad_entropy && overlap(d_grad_logp, whole, d_grad_entropy, whole))
    return fail(ROLLOUT_EINVAL, "the gradients overlap");
  st = check_workspace(d_workspace, workspace_bytes, need);
  if (st != ROLLOUT_OK) return st;
  st = check_words({d_logp, d_old_logp, d_ref_logp, d_entropy, d_adv, d_lengths, d_loss, d_stats, d_grad_logp, d_grad_entropy});
  if (st != ROLLOUT_OK) return st;
  const size_t n = n_seqs;
  st = check_apart({{"d_loss", d_loss, 4}, {"d_stats", d_stats, 20}, {"d_grad_logp", d_grad_logp, whole},
                    {"d_grad_entropy", d_grad_entropy, whole}, {"the workspace", d_workspace, need}},
                   {{"d_logp", d_logp, whole}, {"d_old_logp", d_old_logp, whole}, {"d_ref_logp", d_ref_logp, whole},
                    {"d_entropy", d_entropy, whole}, {"d_adv", d_adv, 4 * n}, {"d_lengths", d_lengths, 4 * n}});
  if (st != ROLLOUT_OK) return st;
  st = check_stream(hip_stream);
  if (st != ROLLOUT_OK) return st;
  const PolicyLossArgs a = {d_logp, d_old_logp, d_ref_logp, d_entropy, d_adv, d_lengths, n_seqs, max_len, clip_low,
                            clip_high, kl_coef, entropy_coef, mean, d_loss, d_stats, d_grad_logp, d_grad_entropy};
  return launched(launch_policy_loss((hipStream_t)hip_stream, a, d_workspace), "policy loss");
}

rollout_status rollout_embedding(const void* d_table, int32_t table_dtype, int32_t vocab, int32_t dim,
                                 const int32_t* d_tokens, int32_t n_tokens, float scale, void* d_out, int32_t out_dtype,
                                 void* hip_stream) {
  Range range("rollout_embedding");
  rollout_status st = check_table(table_dtype, out_dtype, vocab, dim, n_tokens, scale);
  if (st != ROLLOUT_OK) return st;
  if (!d_table || !d_tokens || !d_out) return fail(ROLLOUT_EINVAL, "NULL buffer");
  if (!aligned_to(d_table, elem_bytes(table_dtype)) || !aligned_to(d_out, elem_bytes(out_dtype)))
    return fail(ROLLOUT_EINVAL, "a matrix is not aligned to its type");
  st = check_words({d_tokens});
  if (st != ROLLOUT_OK) return st;
  st = check_apart({{"d_out", d_out, (size_t)n_tokens * dim * elem_bytes(out_dtype)}},
                   {{"d_table", d_table, (size_t)vocab * dim * elem_bytes(table_dtype)}, {"d_tokens", d_tokens, 4 * (size_t)n_tokens}});
  if (st != ROLLOUT_OK) return st;
  st = check_stream(hip_stream);
  if (st != ROLLOUT_OK) return st;
  const EmbeddingArgs a = {d_table, vocab, dim, d_tokens, n_tokens, scale, d_out};
  return launched(launch_embedding((hipStream_t)hip_stream, table_dtype, out_dtype, a), "embedding");
}

rollout_status rollout_embedding_backward_workspace(int32_t n_tokens, int32_t vocab, int32_t dim, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  const rollout_status st = check_table(ROLLOUT_DTYPE_FP32, ROLLOUT_DTYPE_FP32, vocab, dim, n_tokens, 1.f);
  if (st != ROLLOUT_OK) return st;
  if (!embedding_backward_fits(n_tokens, dim))
    return fail(ROLLOUT_EUNSUPPORTED, "n_tokens times ceil(dim / 1024) above 2^25");
  *h_bytes = embedding_backward_workspace(n_tokens, vocab, dim);
  return ROLLOUT_OK;
}

rollout_status rollout_embedding_backward(const void* d_grad, int32_t grad_dtype, const int32_t* d_tokens, int32_t n_tokens,
                                          int32_t vocab, int32_t dim, float scale, int32_t accumulate, void* d_grad_table,
                                          int32_t table_dtype, void* d_workspace, uint64_t workspace_bytes,
                                          void* hip_stream) {
  Range range("rollout_embedding_backward");
  rollout_status st = check_table(table_dtype, grad_dtype, vocab, dim, n_tokens, scale);
  if (st != ROLLOUT_OK) return st;
  uint64_t need = 0;
  st = rollout_embedding_backward_workspace(n_tokens, vocab, dim, &need);
  if (st != ROLLOUT_OK) return st;
  if (accumulate != 0 && accumulate != 1) return fail(ROLLOUT_EINVAL, "accumulate must be 0 or 1");
  if (!d_grad || !d_tokens || !d_grad_table) return fail(ROLLOUT_EINVAL, "NULL buffer");
  if (!aligned_to(d_grad, elem_bytes(grad_dtype)) || !aligned_to(d_grad_table, elem_bytes(table_dtype)))
    return fail(ROLLOUT_EINVAL, "a matrix is not aligned to its type");
  st = check_workspace(d_workspace, workspace_bytes, need);
  if (st != ROLLOUT_OK) return st;
  st = check_words({d_tokens});
  if (st != ROLLOUT_OK) return st;
  st = check_apart({{"d_grad_table", d_grad_table, (size_t)vocab * dim * elem_bytes(table_dtype)}, {"the workspace", d_workspace, need}},
                   {{"d_grad", d_grad, (size_t)n_tokens * dim * elem_bytes(grad_dtype)}, {"d_tokens", d_tokens, 4 * (size_t)n_tokens}});
  if (st != ROLLOUT_OK) return st;
  st = check_stream(hip_stream);
  if (st != ROLLOUT_OK) return st;
  const EmbeddingGradArgs a = {d_grad, d_tokens, n_tokens, vocab, dim, scale, accumulate != 0, d_grad_table};
  return launched(launch_embedding_backward((hipStream_t)hip_stream, grad_dtype, table_dtype, a, d_workspace),
                  "embedding backward");
}

}  // extern "C"
