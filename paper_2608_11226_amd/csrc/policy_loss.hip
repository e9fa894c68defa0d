// The clipped policy loss over groups of completions, and its gradient with respect to log probabilities and entropies.
//
//   d = lp - old, r = e^d;   surr = min(r A, clip(r, 1 - el, 1 + eh) A);   x = ref - lp, kl = e^x - 1 - x
//   tok = -surr + b kl - c H;   loss = sum_s w_s sum_{t < len_s} tok
//   dlp = w_s (-A r [not clipped] - b (e^x - 1));   dH = -c w_s
//
// Which side of a clipping border a token is on is decided on the exact difference in 64 bits, against the border's
// logarithm, so that it does not hang on the rounding of an exponential.  Terms are fp32; their sums are fp64, added up
// per thread, per workgroup, and over the workgroups by a second kernel, always in the same order.
#include "update.h"

namespace rollout {
namespace {

constexpr int LB = 256;
constexpr int kTile = LB * 4;     // tokens of a workgroup's step
constexpr int kMaxBlocks = 1024;  // as many as the join has threads
constexpr int kSums = 6;          // loss, r, kl, clipped low, clipped high, H
constexpr int kCountSeqs = 8192;  // up to here every workgroup counts the tokens itself

struct Borders {
  double low, high;  // ln(1 - el), ln(1 + eh)
};

// Sums of K values per thread over the workgroup, in a fixed order, for the threads 0 .. K - 1 (one each).
template <int K>
__device__ __forceinline__ double block_sums(const double (&v)[K], double* red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  double s[K];
#pragma unroll
  for (int k = 0; k < K; ++k) s[k] = v[k];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] += __shfl_xor(s[k], o, 64);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) red[w * K + k] = s[k];
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x < K)
    for (int i = 0; i < nw; ++i) t += red[i * K + threadIdx.x];
  return t;
}

__device__ __forceinline__ int length_of(const int32_t* lengths, int s, int N) {
  return lengths ? max(0, min(lengths[s], N)) : N;
}

// Number of counted tokens, in every thread (whole numbers below 2^53: exact in any order).
__device__ __forceinline__ double count_tokens(const int32_t* lengths, int S, int N, double* red) {
  if (!lengths) return (double)S * N;
  double v = 0.0;
  for (int s = threadIdx.x; s < S; s += blockDim.x) v += length_of(lengths, s, N);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) v += red[i];
  return v;
}

__global__ __launch_bounds__(1024) void k_policy_count(const int32_t* __restrict__ lengths, int S, int N,
                                                       double* __restrict__ count) {
  __shared__ double red[16];
  const double c = count_tokens(lengths, S, N, red);
  if (threadIdx.x == 0) *count = c;
}

__device__ __forceinline__ void load4(const float* p, int n, float (&v)[4]) {
  if (n >= 4) {
    unpack16(load16(p), v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < n ? p[j] : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int n, const float (&v)[4]) {
  if (n >= 4) {
    store16(p, pack16(v));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = v[j];
  }
}

__global__ __launch_bounds__(LB) void k_policy_loss(PolicyLossArgs a, Borders border, const double* __restrict__ count,
                                                    double* __restrict__ part) {
  __shared__ double red[LB / 64], sums[LB / 64 * kSums];
  const int S = a.seqs, N = a.max_len;
  const int64_t total = (int64_t)S * N;
  double all = (double)S * N;
  if (a.mean == ROLLOUT_MEAN_TOKEN) all = fmax(count ? *count : count_tokens(a.lengths, S, N, red), 1.0);
  const float w_all = (float)(1.0 / all);
  double sum[kSums] = {};
  for (int64_t i0 = (int64_t)blockIdx.x * kTile + threadIdx.x * 4; i0 < total; i0 += (int64_t)gridDim.x * kTile) {
    const int n = (int)min((int64_t)4, total - i0);
    int s = (int)((uint32_t)i0 / (uint32_t)N), t = (int)((uint32_t)i0 - (uint32_t)s * (uint32_t)N);
    int len = length_of(a.lengths, s, N);
    float A = a.adv[s];
    float ws = a.mean == ROLLOUT_MEAN_SEQUENCE ? (float)(1.0 / ((double)S * max(len, 1))) : w_all;
    bool live[4];
    float adv[4], w[4];
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      live[j] = j < n && t < len;
      adv[j] = A;
      w[j] = ws;
      any |= live[j];
      if (++t == N && j + 1 < n) {  // the next sequence begins
        t = 0;
        ++s;
        len = length_of(a.lengths, s, N);
        A = a.adv[s];
        if (a.mean == ROLLOUT_MEAN_SEQUENCE) ws = (float)(1.0 / ((double)S * max(len, 1)));
      }
    }
    float gl[4] = {}, gh[4] = {};
    if (any) {
      float lp[4], old[4], ref[4], H[4];
      load4(a.logp + i0, n, lp);
      if (a.old) load4(a.old + i0, n, old);
      if (a.ref) load4(a.ref + i0, n, ref);
      if (a.entropy) load4(a.entropy + i0, n, H);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!live[j]) continue;
        const double d = a.old ? (double)lp[j] - (double)old[j] : 0.0;
        const float r = expf((float)d), Aj = adv[j];
        const bool high = Aj > 0.f && d > border.high, low = Aj < 0.f && d < border.low;
        // no advantage, no term, whatever the ratio
        const float rA = Aj == 0.f ? 0.f : r * Aj;
        float tok = high ? -(1.f + a.clip_high) * Aj : low ? -(1.f - a.clip_low) * Aj : -rA;
        float g = high || low ? 0.f : -rA;
        float kl = 0.f;
        if (a.ref) {
          const float x = ref[j] - lp[j], ex = expm1f(x);
          kl = ex - x;
          tok = fmaf(a.kl_coef, kl, tok);
          g = fmaf(-a.kl_coef, ex, g);
        }
        if (a.entropy) tok = fmaf(-a.entropy_coef, H[j], tok);
        sum[0] += (double)(tok * w[j]);
        sum[1] += (double)r;
        sum[2] += (double)kl;
        sum[3] += low ? 1.0 : 0.0;
        sum[4] += high ? 1.0 : 0.0;
        sum[5] += a.entropy ? (double)H[j] : 0.0;
        gl[j] = g * w[j];
        gh[j] = -a.entropy_coef * w[j];
      }
    }
    if (a.grad_logp) store4(a.grad_logp + i0, n, gl);
    if (a.grad_entropy) store4(a.grad_entropy + i0, n, gh);
  }
  const double v = block_sums(sum, sums);
  if (threadIdx.x < kSums) part[(size_t)blockIdx.x * kSums + threadIdx.x] = v;
}

__global__ __launch_bounds__(kMaxBlocks) void k_policy_join(const double* __restrict__ part, int blocks,
                                                    const int32_t* __restrict__ lengths, int S, int N,
                                                    float* __restrict__ loss, float* __restrict__ stats) {
  __shared__ double red[kMaxBlocks / 64], sums[kMaxBlocks / 64 * kSums];
  double v[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) v[k] = threadIdx.x < blocks ? part[(size_t)threadIdx.x * kSums + k] : 0.0;
  const double c = fmax(count_tokens(lengths, S, N, red), 1.0);
  const double t = block_sums(v, sums);
  if (threadIdx.x == 0 && loss) *loss = (float)t;
  if (threadIdx.x > 0 && threadIdx.x < kSums && stats) stats[threadIdx.x - 1] = (float)(t / c);
}

int blocks_of(int seqs, int max_len) {
  return (int)std::min(((int64_t)seqs * max_len + kTile - 1) / kTile, (int64_t)kMaxBlocks);
}

}  // namespace

size_t policy_loss_workspace(int seqs, int max_len) { return 16 + (size_t)blocks_of(seqs, max_len) * kSums * 8; }

hipError_t launch_policy_loss(hipStream_t s, const PolicyLossArgs& a, void* ws) {
  double* count = (double*)ws;
  double* part = count + 2;
  const int blocks = blocks_of(a.seqs, a.max_len);
  const Borders b = {std::log1p(-(double)a.clip_low), std::log1p((double)a.clip_high)};
  const bool counted = a.mean == ROLLOUT_MEAN_TOKEN && a.lengths && a.seqs > kCountSeqs;
  if (counted) hipLaunchKernelGGL(k_policy_count, dim3(1), dim3(1024), 0, s, a.lengths, a.seqs, a.max_len, count);
  hipLaunchKernelGGL(k_policy_loss, dim3(blocks), dim3(LB), 0, s, a, b, counted ? count : nullptr, part);
  // the join has a thread for every workgroup's sums, and no more waves than they and the lengths need
  const int threads = (std::max(blocks, std::min(a.seqs, kMaxBlocks)) + 63) / 64 * 64;
  hipLaunchKernelGGL(k_policy_join, dim3(1), dim3(threads), 0, s, part, blocks, a.lengths, a.seqs, a.max_len, a.loss, a.stats);
  return hipGetLastError();
}

}  // namespace rollout
