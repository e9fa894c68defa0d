// The operators of a GRPO step's update side: token log probabilities and their gradient (logprobs.hip), the clipped
// group loss (policy_loss.hip), embedding lookup and its gradient (embedding.hip).  Launchers called by the C entry points in
// update.hip, and device helpers that these kernels share.
#pragma once

#include "internal.h"

#include <algorithm>
#include <type_traits>

namespace rollout {

constexpr int kMaxTop = 32;            // alternatives of a row
constexpr int kMaxTopVocab = 5 << 16;  // widest row that alternatives are taken from

struct LogprobArgs {
  const void* z;
  int64_t stride;
  int rows, vocab;
  float temperature;
  const int32_t* tokens;
  int top;
  float* logp;
  float* entropy;
  float* stats;
  int32_t* top_ids;
  float* top_logp;
};
size_t logprobs_workspace(int rows, int vocab, int top);
hipError_t launch_logprobs(hipStream_t s, int dtype, const LogprobArgs& a, void* ws);

struct LogprobGradArgs {
  const void* z;
  int64_t stride;
  int rows, vocab;
  float temperature;
  const int32_t* tokens;
  const float* stats;
  const float* entropy;
  const float* g;
  const float* h;
  void* dz;
  int64_t dz_stride;
};
hipError_t launch_logprobs_backward(hipStream_t s, int dtype, const LogprobGradArgs& a);

struct PolicyLossArgs {
  const float *logp, *old, *ref, *entropy, *adv;
  const int32_t* lengths;
  int seqs, max_len;
  float clip_low, clip_high, kl_coef, entropy_coef;
  int mean;  // ROLLOUT_MEAN_*
  float *loss, *stats, *grad_logp, *grad_entropy;
};
size_t policy_loss_workspace(int seqs, int max_len);
hipError_t launch_policy_loss(hipStream_t s, const PolicyLossArgs& a, void* ws);

struct EmbeddingArgs {
  const void* table;
  int vocab, dim;
  const int32_t* tokens;
  int n;
  float scale;
  void* out;
};
hipError_t launch_embedding(hipStream_t s, int table_dtype, int out_dtype, const EmbeddingArgs& a);

struct EmbeddingGradArgs {
  const void* g;
  const int32_t* tokens;
  int n, vocab, dim;
  float scale;
  bool accumulate;
  void* table;
};
constexpr int kMaxEmbeddingTokens = 1 << 28;
// its launches have few enough workgroups
inline bool embedding_backward_fits(int n, int dim) { return (int64_t)n * (((int64_t)dim + 1023) / 1024) <= (1 << 25); }
size_t embedding_backward_workspace(int n, int vocab, int dim);
hipError_t launch_embedding_backward(hipStream_t s, int grad_dtype, int table_dtype, const EmbeddingGradArgs& a, void* ws);

constexpr int kMaxHeadsPerKey = 64;
// Strides are in elements.  k_starts and k_lens are never NULL: the queries' where the sequences' keys are their own.
struct AttentionArgs {
  int heads, kv_heads, head_dim, n_seqs, n_q, n_k;
  bool causal;
  float scale;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *q_starts, *q_lens, *k_starts, *k_lens;  // lens may be NULL: whole
  void* out;
  int64_t out_stride;
  float* lse;  // [heads][n_q]
};
size_t packed_attention_workspace(const AttentionArgs& a);
hipError_t launch_packed_attention(hipStream_t s, int dtype, const AttentionArgs& a, void* ws);

struct AttentionGradArgs : AttentionArgs {
  const void* dout;
  int64_t dout_stride;
  void *dq, *dk, *dv;
  int64_t dq_stride, dk_stride, dv_stride;
};
size_t packed_attention_backward_workspace(const AttentionArgs& a);
hipError_t launch_packed_attention_backward(hipStream_t s, int dtype, const AttentionGradArgs& a, void* ws);

constexpr int kMaxNormDim = 32768;
int norm_threads(int dim);  // of a row
inline bool norm_fits(int rows, int dim) {
  const int64_t t = norm_threads(dim), each = t < 256 ? 256 / t : 1;  // rows of a workgroup
  return (rows + each - 1) / each * each * t < (int64_t)1 << 32;
}
struct NormArgs {
  const void *x, *delta;  // delta may be NULL
  const float* gain;      // may be NULL
  int rows, dim;
  float eps;
  void *h, *y;
  float *scales, *rstd;
  double per_value;  // 1 / dim
};
hipError_t launch_rms_norm(hipStream_t s, int x_dtype, int delta_dtype, int y_dtype, const NormArgs& a);

struct NormGradArgs {
  const void *dy, *h;
  const float *gain, *rstd;
  int rows, dim;
  const void* inner;  // of dx's type; may be NULL, or dx
  void* dx;
  float* dgain;  // may be NULL
  int accumulate;
};
size_t rms_norm_backward_workspace(int rows, int dim);
hipError_t launch_rms_norm_backward(hipStream_t s, int h_dtype, int dy_dtype, int dx_dtype, const NormGradArgs& a, void* ws);

// A tensor in the table that the kernel reads; its chunks are first, first + 1, ...
struct AdamwEntry {
  void* param;
  const void* grad;
  void *m, *v;
  float *m_scales, *v_scales;
  void* copy;
  int64_t n, first, chunk;
  float decay;
  int32_t kind;  // 1: bf16 weights, 2: bf16 gradients, 4: states in 8 bits
};
constexpr int kMaxAdamwTensors = 1 << 20;
constexpr int64_t kMaxAdamwElements = (int64_t)1 << 36;
// elements that a workgroup takes of a tensor of a kind, by the number of all tensors' elements
int64_t adamw_chunk(int64_t all, int kind);
struct AdamwArgs {
  float b1, c1, b2, c2, eps, lr;
  double log_b1, log_b2, unbias1;  // 1 / (1 - b1^step)
  float unbias2;                   // 1 / sqrt(1 - b2^step)
  int64_t step;
  uint64_t seed;
  const float *grad_scale, *d_lr;
  const int64_t* d_step;
};
hipError_t launch_adamw(hipStream_t s, const void* table, int tensors, int64_t chunks, const AdamwArgs& a);

}  // namespace rollout

#ifdef __HIPCC__
namespace rollout {

// 16 bytes of a row that starts at any element: rows of an odd width begin anywhere, and the hardware takes such
// loads and stores whole.
template <typename T>
struct Chunk16;
template <>
struct Chunk16<float> {
  static constexpr int N = 4;
  typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(4), may_alias));
};
template <>
struct Chunk16<uint16_t> {
  static constexpr int N = 8;
  typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(2), may_alias));
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p) {
  return *reinterpret_cast<const typename Chunk16<T>::Raw*>(p);
}
// the same for data that is read or written once: it does not push other lines out of the caches (log probabilities of
// 3,584 rows of 152,064 bf16 logits 206 -> 184 us)
template <typename T>
__device__ __forceinline__ u32x4 stream16(const T* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const typename Chunk16<T>::Raw*>(p));
}
template <typename T>
__device__ __forceinline__ void stream16(T* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<typename Chunk16<T>::Raw*>(p));
}
template <typename T>
__device__ __forceinline__ void store16(T* p, u32x4 v) {
  *reinterpret_cast<typename Chunk16<T>::Raw*>(p) = v;
}

__device__ __forceinline__ void unpack16(u32x4 r, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void unpack16(u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
}
// round to nearest, ties to even; a NaN stays one
__device__ __forceinline__ uint16_t round_bf16(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ u32x4 pack16(const float (&v)[4]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
  return r;
}
__device__ __forceinline__ u32x4 pack16(const float (&v)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)round_bf16(v[2 * i]) | ((uint32_t)round_bf16(v[2 * i + 1]) << 16);
  return r;
}
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = round_bf16(v); }

// max(a, b) where b is a number: one infinite value shall not make its neighbours' codes 0
__device__ __forceinline__ float larger(float a, float b) { return b > a && b < INFINITY ? b : a; }

// Smallest power of two that brings `most` (>= 0, finite) to at most 448, the largest e4m3 value; 2^-126 at least.  448 is 1.75 2^8.
__device__ __forceinline__ float e4m3_scale(float most) {
  const uint32_t u = __float_as_uint(most);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// Reductions of one value per lane by lane moves, without LDS, the result the same in every lane: shifts of 1, 2, 4 and 8
// lanes within each row of 16, then row 0's result into row 1 and row 2's into row 3, then the first two rows' into the
// others; a lane with no source takes `none`.  Lane 63 then has all of them.
template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t none, F f) {
#define ROLLOUT_STEP(ctrl, rows) \
  v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, ctrl, rows, 0xf, false))
  ROLLOUT_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8
  ROLLOUT_STEP(0x112, 0xf);
  ROLLOUT_STEP(0x114, 0xf);
  ROLLOUT_STEP(0x118, 0xf);
  ROLLOUT_STEP(0x142, 0xa);  // row_bcast:15 into rows 1 and 3
  ROLLOUT_STEP(0x143, 0xc);  // row_bcast:31 into rows 2 and 3
#undef ROLLOUT_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float wave_max_f32(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), 0xFF800000u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

}  // namespace rollout
#endif
