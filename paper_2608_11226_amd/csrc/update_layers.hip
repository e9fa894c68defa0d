// C entry points that carry an update through the layers: packed attention and its gradient, the residual norm and its
// gradient, the optimiser's step.  As in update.hip they need no context.
#include "update_checks.h"

#include <algorithm>
#include <vector>

using namespace rollout;

namespace {

// A launch has less than 2^32 threads, in workgroups of 256.  Attention has one for some 32 rows of a head at least, and one more
// for a head and sequence.
constexpr int64_t kMaxGroups = (1 << 24) - 8, kMaxHeadRows = 1 << 26, kMaxHeadSeqs = 1 << 23;
static_assert(kMaxHeadRows / 32 + kMaxHeadSeqs < kMaxGroups, "a launch of attention");
constexpr int64_t kMaxRowBytes = 1 << 25;

rollout_status check_shape(const rollout_attention_shape* s) {
  if (!s) return fail(ROLLOUT_EINVAL, "the shape is NULL");
  if (!is_float_type(s->dtype)) return fail(ROLLOUT_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
  if (s->n_heads < 1 || s->n_kv_heads < 1 || s->n_heads % s->n_kv_heads)
    return fail(ROLLOUT_EINVAL, "n_heads must be a multiple of n_kv_heads, both >= 1");
  if (s->n_heads / s->n_kv_heads > kMaxHeadsPerKey) return fail(ROLLOUT_EUNSUPPORTED, "more than 64 query heads for a key's");
  if (s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128)
    return fail(ROLLOUT_EUNSUPPORTED, "head_dim must be 32, 64 or 128");
  if (s->n_seqs < 1 || s->n_q < 1 || s->n_k < 1) return fail(ROLLOUT_EINVAL, "n_seqs, n_q and n_k must be >= 1");
  if (s->causal != 0 && s->causal != 1) return fail(ROLLOUT_EINVAL, "causal must be 0 or 1");
  // (the gradient forms lse / scale)
  if (!(s->scale >= 0x1p-100f && s->scale <= 0x1p100f)) return fail(ROLLOUT_EINVAL, "scale must be in [2^-100, 2^100]");
  if ((int64_t)s->n_heads * std::max(s->n_q, s->n_k) > kMaxHeadRows)
    return fail(ROLLOUT_EUNSUPPORTED, "n_heads times tokens above 2^26");
  if ((int64_t)s->n_heads * s->n_seqs > kMaxHeadSeqs) return fail(ROLLOUT_EUNSUPPORTED, "n_heads times sequences above 2^23");
  return ROLLOUT_OK;
}

AttentionArgs args_of(const rollout_attention_shape& s) {
  AttentionArgs a = {};
  a.heads = s.n_heads, a.kv_heads = s.n_kv_heads, a.head_dim = s.head_dim;
  a.n_seqs = s.n_seqs, a.n_q = s.n_q, a.n_k = s.n_k;
  a.causal = s.causal != 0;
  a.scale = s.scale;
  return a;
}

// a matrix of tokens
rollout_status check_tokens(const char* name, const void* p, int64_t stride, int64_t width, int dtype) {
  const int64_t es = (int64_t)elem_bytes(dtype);
  if (!p) return fail(ROLLOUT_EINVAL, std::string(name) + " is NULL");
  if (!aligned_to(p, 16)) return fail(ROLLOUT_EINVAL, std::string(name) + " must be aligned to 16 bytes");
  if (stride < width) return fail(ROLLOUT_EINVAL, std::string(name) + ": the stride must be at least the row's width");
  if (stride > kMaxRowBytes / es) return fail(ROLLOUT_EUNSUPPORTED, std::string(name) + ": rows more than 2^25 bytes apart");
  if (stride * es % 16) return fail(ROLLOUT_EINVAL, std::string(name) + ": the stride must be a multiple of 16 bytes");
  return ROLLOUT_OK;
}

// places of the sequences; the keys' are the queries' where they are not given
rollout_status check_places(const rollout_attention_shape& s, const int32_t* q_starts, const int32_t* q_lens,
                            const int32_t* k_starts, const int32_t* k_lens, AttentionArgs* a) {
  if (!q_starts) return fail(ROLLOUT_EINVAL, "d_q_starts is NULL");
  if (!k_starts && k_lens) return fail(ROLLOUT_EINVAL, "d_k_lens without d_k_starts");
  if (!k_starts && s.n_k != s.n_q) return fail(ROLLOUT_EINVAL, "without d_k_starts there are as many keys as queries");
  a->q_starts = q_starts, a->q_lens = q_lens;
  a->k_starts = k_starts ? k_starts : q_starts, a->k_lens = k_starts ? k_lens : q_lens;
  return check_words({q_starts, q_lens, k_starts, k_lens});
}

// rows of the norm
rollout_status check_norm(int32_t rows, int32_t dim) {
  if (rows < 1 || dim < 1) return fail(ROLLOUT_EINVAL, "n_rows and dim must be >= 1");
  if (dim > kMaxNormDim) return fail(ROLLOUT_EUNSUPPORTED, "dim above 32,768");
  if (!norm_fits(rows, dim)) return fail(ROLLOUT_EUNSUPPORTED, "too many rows for one launch");
  return ROLLOUT_OK;
}

size_t type_bytes(int32_t dtype) { return dtype == ROLLOUT_DTYPE_E4M3 ? 1 : elem_bytes(dtype); }

// Where a call of AdamW reads or writes.
struct Place {
  uintptr_t lo, hi;
  int tensor;
  bool written;
};

}  // namespace

extern "C" {

rollout_status rollout_attention_workspace(const rollout_attention_shape* shape, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  const rollout_status st = check_shape(shape);
  if (st != ROLLOUT_OK) return st;
  *h_bytes = packed_attention_workspace(args_of(*shape));
  return ROLLOUT_OK;
}

rollout_status rollout_attention(const rollout_attention_shape* shape, const void* d_q, int64_t q_stride, const void* d_k,
                                 int64_t k_stride, const void* d_v, int64_t v_stride, const int32_t* d_q_starts,
                                 const int32_t* d_q_lens, const int32_t* d_k_starts, const int32_t* d_k_lens, void* d_out,
                                 int64_t out_stride, float* d_lse, void* d_workspace, uint64_t workspace_bytes,
                                 void* hip_stream) {
  Range range("rollout_attention");
  uint64_t need = 0;
  rollout_status st = rollout_attention_workspace(shape, &need);
  if (st != ROLLOUT_OK) return st;
  const rollout_attention_shape& s = *shape;
  const int64_t wq = (int64_t)s.n_heads * s.head_dim, wk = (int64_t)s.n_kv_heads * s.head_dim;
  if ((st = check_tokens("d_q", d_q, q_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_k", d_k, k_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_v", d_v, v_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_out", d_out, out_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if (!d_lse) return fail(ROLLOUT_EINVAL, "d_lse is NULL");
  AttentionArgs a = args_of(s);
  if ((st = check_places(s, d_q_starts, d_q_lens, d_k_starts, d_k_lens, &a)) != ROLLOUT_OK) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, need)) != ROLLOUT_OK) return st;
  if ((st = check_words({d_lse})) != ROLLOUT_OK) return st;
  const size_t es = elem_bytes(s.dtype), nq = s.n_q, nk = s.n_k, starts = 4 * ((size_t)s.n_seqs + 1), lens = 4 * (size_t)s.n_seqs;
  st = check_apart({{"d_out", d_out, wq * es, nq, out_stride * es}, {"d_lse", d_lse, 4 * nq * s.n_heads}, {"the workspace", d_workspace, need}},
                   {{"d_q", d_q, wq * es, nq, q_stride * es}, {"d_k", d_k, wk * es, nk, k_stride * es},
                    {"d_v", d_v, wk * es, nk, v_stride * es}, {"d_q_starts", d_q_starts, starts}, {"d_q_lens", d_q_lens, lens},
                    {"d_k_starts", d_k_starts, starts}, {"d_k_lens", d_k_lens, lens}});
  if (st != ROLLOUT_OK) return st;
  if ((st = check_stream(hip_stream)) != ROLLOUT_OK) return st;
  a.q = d_q, a.k = d_k, a.v = d_v, a.out = d_out, a.lse = d_lse;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.out_stride = out_stride;
  return launched(launch_packed_attention((hipStream_t)hip_stream, s.dtype, a, d_workspace), "attention");
}

rollout_status rollout_attention_backward_workspace(const rollout_attention_shape* shape, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  const rollout_status st = check_shape(shape);
  if (st != ROLLOUT_OK) return st;
  *h_bytes = packed_attention_backward_workspace(args_of(*shape));
  return ROLLOUT_OK;
}

rollout_status rollout_attention_backward(const rollout_attention_shape* shape, const void* d_q, int64_t q_stride,
                                          const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                                          const int32_t* d_q_starts, const int32_t* d_q_lens, const int32_t* d_k_starts,
                                          const int32_t* d_k_lens, const void* d_out, int64_t out_stride, const float* d_lse,
                                          const void* d_grad_out, int64_t grad_out_stride, void* d_grad_q,
                                          int64_t grad_q_stride, void* d_grad_k, int64_t grad_k_stride, void* d_grad_v,
                                          int64_t grad_v_stride, void* d_workspace, uint64_t workspace_bytes,
                                          void* hip_stream) {
  Range range("rollout_attention_backward");
  uint64_t need = 0;
  rollout_status st = rollout_attention_backward_workspace(shape, &need);
  if (st != ROLLOUT_OK) return st;
  const rollout_attention_shape& s = *shape;
  const int64_t wq = (int64_t)s.n_heads * s.head_dim, wk = (int64_t)s.n_kv_heads * s.head_dim;
  if ((st = check_tokens("d_q", d_q, q_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_k", d_k, k_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_v", d_v, v_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_out", d_out, out_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_grad_out", d_grad_out, grad_out_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_grad_q", d_grad_q, grad_q_stride, wq, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_grad_k", d_grad_k, grad_k_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if ((st = check_tokens("d_grad_v", d_grad_v, grad_v_stride, wk, s.dtype)) != ROLLOUT_OK) return st;
  if (!d_lse) return fail(ROLLOUT_EINVAL, "d_lse is NULL");
  AttentionGradArgs a;
  static_cast<AttentionArgs&>(a) = args_of(s);
  if ((st = check_places(s, d_q_starts, d_q_lens, d_k_starts, d_k_lens, &a)) != ROLLOUT_OK) return st;
  if ((st = check_workspace(d_workspace, workspace_bytes, need)) != ROLLOUT_OK) return st;
  if ((st = check_words({d_lse})) != ROLLOUT_OK) return st;
  const size_t es = elem_bytes(s.dtype), nq = s.n_q, nk = s.n_k, starts = 4 * ((size_t)s.n_seqs + 1), lens = 4 * (size_t)s.n_seqs;
  st = check_apart({{"d_grad_q", d_grad_q, wq * es, nq, grad_q_stride * es}, {"d_grad_k", d_grad_k, wk * es, nk, grad_k_stride * es},
                    {"d_grad_v", d_grad_v, wk * es, nk, grad_v_stride * es}, {"the workspace", d_workspace, need}},
                   {{"d_q", d_q, wq * es, nq, q_stride * es}, {"d_k", d_k, wk * es, nk, k_stride * es},
                    {"d_v", d_v, wk * es, nk, v_stride * es}, {"d_out", d_out, wq * es, nq, out_stride * es},
                    {"d_grad_out", d_grad_out, wq * es, nq, grad_out_stride * es}, {"d_lse", d_lse, 4 * nq * s.n_heads},
                    {"d_q_starts", d_q_starts, starts}, {"d_q_lens", d_q_lens, lens},
                    {"d_k_starts", d_k_starts, starts}, {"d_k_lens", d_k_lens, lens}});
  if (st != ROLLOUT_OK) return st;
  if ((st = check_stream(hip_stream)) != ROLLOUT_OK) return st;
  a.q = d_q, a.k = d_k, a.v = d_v, a.out = const_cast<void*>(d_out), a.lse = const_cast<float*>(d_lse);
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.out_stride = out_stride;
  a.dout = d_grad_out, a.dq = d_grad_q, a.dk = d_grad_k, a.dv = d_grad_v;
  a.dout_stride = grad_out_stride, a.dq_stride = grad_q_stride, a.dk_stride = grad_k_stride, a.dv_stride = grad_v_stride;
  return launched(launch_packed_attention_backward((hipStream_t)hip_stream, s.dtype, a, d_workspace), "attention backward");
}

rollout_status rollout_rms_norm(const void* d_x, int32_t x_dtype, const void* d_delta, int32_t delta_dtype,
                                const float* d_gain, int32_t n_rows, int32_t dim, float eps, void* d_h, void* d_y,
                                int32_t y_dtype, float* d_scales, float* d_rstd, void* hip_stream) {
  Range range("rollout_rms_norm");
  rollout_status st = check_norm(n_rows, dim);
  if (st != ROLLOUT_OK) return st;
  if (!is_float_type(x_dtype)) return fail(ROLLOUT_EINVAL, "x_dtype must be 0 (fp32) or 1 (bf16)");
  if (d_delta && !is_float_type(delta_dtype)) return fail(ROLLOUT_EINVAL, "delta_dtype must be 0 (fp32) or 1 (bf16)");
  if (!is_float_type(y_dtype) && y_dtype != ROLLOUT_DTYPE_E4M3)
    return fail(ROLLOUT_EINVAL, "y_dtype must be 0 (fp32), 1 (bf16) or 3 (e4m3)");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(ROLLOUT_EINVAL, "eps must be >= 0 and finite");
  if (!d_x || !d_y) return fail(ROLLOUT_EINVAL, "NULL buffer");
  if (!d_delta != !d_h) return fail(ROLLOUT_EINVAL, "d_delta and d_h come together");
  if ((y_dtype == ROLLOUT_DTYPE_E4M3) != (d_scales != nullptr)) return fail(ROLLOUT_EINVAL, "d_scales belongs to an e4m3 output, which needs it");
  if (!aligned_to(d_x, type_bytes(x_dtype)) || !aligned_to(d_y, type_bytes(y_dtype)) || !aligned_to(d_h, type_bytes(x_dtype)) ||
      (d_delta && !aligned_to(d_delta, type_bytes(delta_dtype))))
    return fail(ROLLOUT_EINVAL, "a matrix is not aligned to its type");
  if ((st = check_words({d_gain, d_scales, d_rstd})) != ROLLOUT_OK) return st;
  const size_t n = (size_t)n_rows * dim, rows = n_rows;
  st = check_apart({{"d_h", d_h == d_x ? nullptr : d_h, n * type_bytes(x_dtype)}, {"d_y", d_y, n * type_bytes(y_dtype)},
                    {"d_scales", d_scales, 4 * rows}, {"d_rstd", d_rstd, 4 * rows}},
                   {{"d_x", d_x, n * type_bytes(x_dtype)}, {"d_delta", d_delta, d_delta ? n * type_bytes(delta_dtype) : 0},
                    {"d_gain", d_gain, 4 * (size_t)dim}});
  if (st != ROLLOUT_OK) return st;
  // in place: x is an output too
  st = check_apart({{"d_h", d_h == d_x ? d_h : nullptr, n * type_bytes(x_dtype)}},
                   {{"d_delta", d_delta, d_delta ? n * type_bytes(delta_dtype) : 0}, {"d_gain", d_gain, 4 * (size_t)dim}});
  if (st != ROLLOUT_OK) return st;
  if ((st = check_stream(hip_stream)) != ROLLOUT_OK) return st;
  const NormArgs a = {d_x, d_delta, d_gain, n_rows, dim, eps, d_h, d_y, d_scales, d_rstd, 1.0 / dim};
  return launched(launch_rms_norm((hipStream_t)hip_stream, x_dtype, delta_dtype, y_dtype, a), "rms norm");
}

rollout_status rollout_rms_norm_backward_workspace(int32_t n_rows, int32_t dim, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  const rollout_status st = check_norm(n_rows, dim);
  if (st != ROLLOUT_OK) return st;
  *h_bytes = rms_norm_backward_workspace(n_rows, dim);
  return ROLLOUT_OK;
}

rollout_status rollout_rms_norm_backward(const void* d_grad_y, int32_t grad_y_dtype, const void* d_h, int32_t h_dtype,
                                         const float* d_gain, const float* d_rstd, int32_t n_rows, int32_t dim,
                                         const void* d_grad_h, void* d_grad_x, int32_t grad_x_dtype, float* d_grad_gain,
                                         int32_t accumulate, void* d_workspace, uint64_t workspace_bytes,
                                         void* hip_stream) {
  Range range("rollout_rms_norm_backward");
  uint64_t need = 0;
  rollout_status st = rollout_rms_norm_backward_workspace(n_rows, dim, &need);
  if (st != ROLLOUT_OK) return st;
  if (!is_float_type(grad_y_dtype) || !is_float_type(h_dtype) || !is_float_type(grad_x_dtype))
    return fail(ROLLOUT_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
  if (accumulate != 0 && accumulate != 1) return fail(ROLLOUT_EINVAL, "accumulate must be 0 or 1");
  if (!d_grad_y || !d_h || !d_rstd || !d_grad_x) return fail(ROLLOUT_EINVAL, "NULL buffer");
  if (!aligned_to(d_grad_y, elem_bytes(grad_y_dtype)) || !aligned_to(d_h, elem_bytes(h_dtype)) ||
      !aligned_to(d_grad_x, elem_bytes(grad_x_dtype)) || !aligned_to(d_grad_h, elem_bytes(grad_x_dtype)))
    return fail(ROLLOUT_EINVAL, "a matrix is not aligned to its type");
  if ((st = check_words({d_gain, d_rstd, d_grad_gain})) != ROLLOUT_OK) return st;
  if (!d_grad_gain) need = 0;
  if ((st = check_workspace(d_workspace, workspace_bytes, need)) != ROLLOUT_OK) return st;
  const size_t n = (size_t)n_rows * dim, x_bytes = n * elem_bytes(grad_x_dtype);
  st = check_apart({{"d_grad_x", d_grad_x, x_bytes}, {"d_grad_gain", d_grad_gain, 4 * (size_t)dim}, {"the workspace", d_workspace, need}},
                   {{"d_grad_y", d_grad_y, n * elem_bytes(grad_y_dtype)}, {"d_h", d_h, n * elem_bytes(h_dtype)},
                    {"d_gain", d_gain, 4 * (size_t)dim}, {"d_rstd", d_rstd, 4 * (size_t)n_rows},
                    {"d_grad_h", d_grad_h == d_grad_x ? nullptr : d_grad_h, x_bytes}});
  if (st != ROLLOUT_OK) return st;
  if ((st = check_stream(hip_stream)) != ROLLOUT_OK) return st;
  const NormGradArgs a = {d_grad_y, d_h, d_gain, d_rstd, n_rows, dim, d_grad_h, d_grad_x, d_grad_gain, accumulate};
  return launched(launch_rms_norm_backward((hipStream_t)hip_stream, h_dtype, grad_y_dtype, grad_x_dtype, a, d_workspace),
                  "rms norm backward");
}

rollout_status rollout_adamw_table_bytes(int32_t n_tensors, uint64_t* h_bytes) {
  if (!h_bytes) return fail(ROLLOUT_EINVAL, "the result pointer is NULL");
  if (n_tensors < 1) return fail(ROLLOUT_EINVAL, "n_tensors must be >= 1");
  if (n_tensors > kMaxAdamwTensors) return fail(ROLLOUT_EUNSUPPORTED, "more than 2^20 tensors");
  *h_bytes = (uint64_t)n_tensors * sizeof(AdamwEntry);
  return ROLLOUT_OK;
}

rollout_status rollout_adamw_table(const rollout_adamw_tensor* h_tensors, int32_t n_tensors, void* h_table,
                                   uint64_t table_bytes, int64_t* h_chunks) {
  uint64_t need = 0;
  rollout_status st = rollout_adamw_table_bytes(n_tensors, &need);
  if (st != ROLLOUT_OK) return st;
  if (!h_tensors || !h_table || !h_chunks) return fail(ROLLOUT_EINVAL, "NULL argument");
  if (table_bytes < need)
    return fail(ROLLOUT_ENOMEM, "table of " + std::to_string(table_bytes) + " bytes; these tensors need " + std::to_string(need));
  try {
    std::vector<Place> places;
    int64_t all = 0;
    for (int i = 0; i < n_tensors; ++i) {
      const rollout_adamw_tensor& t = h_tensors[i];
      const std::string at = "tensor " + std::to_string(i) + ": ";
      if (t.n < 0) return fail(ROLLOUT_EINVAL, at + "n must be >= 0");
      if (t.n > kMaxAdamwElements - all) return fail(ROLLOUT_EUNSUPPORTED, "more than 2^36 elements");
      if (!is_float_type(t.param_dtype) || !is_float_type(t.grad_dtype)) return fail(ROLLOUT_EINVAL, at + "dtype must be 0 (fp32) or 1 (bf16)");
      const bool eight = t.state_dtype == ROLLOUT_DTYPE_E4M3;
      if (!eight && t.state_dtype != ROLLOUT_DTYPE_FP32) return fail(ROLLOUT_EINVAL, at + "state_dtype must be 0 (fp32) or 3 (e4m3)");
      if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.f) return fail(ROLLOUT_EINVAL, at + "weight_decay must be >= 0 and finite");
      if (t.d_copy && t.param_dtype != ROLLOUT_DTYPE_FP32) return fail(ROLLOUT_EINVAL, at + "a bf16 copy is one of fp32 weights");
      if (!t.n) continue;
      all += t.n;
      if (!t.d_param || !t.d_grad || !t.d_m || !t.d_v || (eight && (!t.d_m_scales || !t.d_v_scales)))
        return fail(ROLLOUT_EINVAL, at + "NULL buffer");
      if (!eight && (t.d_m_scales || t.d_v_scales)) return fail(ROLLOUT_EINVAL, at + "scales belong to states in 8 bits");
      const size_t n = t.n, p = elem_bytes(t.param_dtype), g = elem_bytes(t.grad_dtype), s = eight ? 1 : 4;
      if (!aligned_to(t.d_param, p) || !aligned_to(t.d_grad, g) || !aligned_to(t.d_m, s) || !aligned_to(t.d_v, s) ||
          !aligned_to(t.d_m_scales, 4) || !aligned_to(t.d_v_scales, 4) || !aligned_to(t.d_copy, 2))
        return fail(ROLLOUT_EINVAL, at + "a buffer is not aligned to its type");
      const size_t blocks = 4 * ((n + 127) / 128);
      auto put = [&](const void* at, size_t bytes, bool written) {
        if (at) places.push_back({(uintptr_t)at, (uintptr_t)at + bytes, i, written});
      };
      put(t.d_param, n * p, true), put(t.d_grad, n * g, false), put(t.d_m, n * s, true), put(t.d_v, n * s, true);
      put(t.d_m_scales, blocks, true), put(t.d_v_scales, blocks, true), put(t.d_copy, n * 2, true);
    }
    // no place that is written shares a byte with another
    std::sort(places.begin(), places.end(), [](const Place& a, const Place& b) { return a.lo < b.lo; });
    uintptr_t read_to = 0, written_to = 0;
    for (const Place& p : places) {
      if (p.lo < written_to || (p.written && p.lo < read_to))
        return fail(ROLLOUT_EINVAL, "tensor " + std::to_string(p.tensor) + ": a buffer overlaps another one of the table");
      (p.written ? written_to : read_to) = std::max(p.written ? written_to : read_to, p.hi);
    }
    int64_t chunks = 0;
    AdamwEntry* out = static_cast<AdamwEntry*>(h_table);
    for (int i = 0; i < n_tensors; ++i) {
      const rollout_adamw_tensor& t = h_tensors[i];
      const int32_t kind = (t.param_dtype == ROLLOUT_DTYPE_BF16 ? 1 : 0) | (t.grad_dtype == ROLLOUT_DTYPE_BF16 ? 2 : 0) |
                           (t.state_dtype == ROLLOUT_DTYPE_E4M3 ? 4 : 0);
      const int64_t chunk = adamw_chunk(all, kind);
      const AdamwEntry e = {t.d_param, t.d_grad, t.d_m, t.d_v, t.d_m_scales, t.d_v_scales, t.d_copy, t.n, chunks, chunk, t.weight_decay, kind};
      std::copy_n(reinterpret_cast<const char*>(&e), sizeof e, reinterpret_cast<char*>(out + i));
      chunks += (t.n + chunk - 1) / chunk;
    }
    if (chunks > kMaxGroups) return fail(ROLLOUT_EUNSUPPORTED, "too many tensors and elements for one launch");
    *h_chunks = chunks;
  } catch (const std::exception& e) {
    return fail(ROLLOUT_ENOMEM, std::string("adamw table: ") + e.what());
  }
  return ROLLOUT_OK;
}

rollout_status rollout_adamw(const void* d_table, int32_t n_tensors, int64_t n_chunks, double lr, double beta1, double beta2,
                             double eps, int64_t step, uint64_t seed, const float* d_grad_scale, const float* d_lr,
                             const int64_t* d_step, void* hip_stream) {
  Range range("rollout_adamw");
  uint64_t bytes = 0;
  rollout_status st = rollout_adamw_table_bytes(n_tensors, &bytes);
  if (st != ROLLOUT_OK) return st;
  if (n_chunks < 0 || n_chunks > kMaxGroups) return fail(ROLLOUT_EINVAL, "n_chunks is not what the table's making gave");
  if (!d_table) return fail(ROLLOUT_EINVAL, "the table is NULL");
  if (!aligned_to(d_table, 8)) return fail(ROLLOUT_EINVAL, "the table must be aligned to 8 bytes");
  if (!std::isfinite((float)lr)) return fail(ROLLOUT_EINVAL, "lr must be finite in fp32");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return fail(ROLLOUT_EINVAL, "beta1 and beta2 must be in [0, 1)");
  // (the reciprocal of a smaller one is not finite, and 0 times that no number)
  if (!(eps == 0.0 || eps >= 0x1p-126) || !std::isfinite((float)eps))
    return fail(ROLLOUT_EINVAL, "eps must be 0 or at least 2^-126, and finite in fp32");
  if (!d_step && step < 1) return fail(ROLLOUT_EINVAL, "step must be >= 1");
  if ((st = check_words({d_grad_scale, d_lr})) != ROLLOUT_OK) return st;
  if (!aligned_to(d_step, 8)) return fail(ROLLOUT_EINVAL, "d_step must be aligned to 8 bytes");
  if ((st = check_stream(hip_stream)) != ROLLOUT_OK) return st;
  if (!n_chunks) return ROLLOUT_OK;
  AdamwArgs a = {};
  a.b1 = (float)beta1, a.c1 = (float)(1.0 - beta1), a.b2 = (float)beta2, a.c2 = (float)(1.0 - beta2);
  a.eps = (float)eps, a.lr = (float)lr;
  a.log_b1 = std::log(beta1), a.log_b2 = std::log(beta2);
  a.unbias1 = 1.0 / -std::expm1((double)step * a.log_b1);
  a.unbias2 = (float)(1.0 / std::sqrt(-std::expm1((double)step * a.log_b2)));
  a.step = step, a.seed = seed;
  a.grad_scale = d_grad_scale, a.d_lr = d_lr, a.d_step = d_step;
  return launched(launch_adamw((hipStream_t)hip_stream, d_table, n_tensors, n_chunks, a), "adamw");
}

}  // extern "C"
