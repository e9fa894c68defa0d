// The clipped policy loss over groups of completions, and its gradient with respect to log probabilities and entropies.
//
//   d = lp - old, r = e^d;   surr = min(r A, clip(r, 1 - el, 1 + eh) A);   x = ref - lp, kl = e^x - 1 - x
//   tok = -surr + b kl - c H;   loss = sum_s w_s sum_{t < len_s} tok
//   dlp = w_s (-A r [not clipped] - b (e^x - 1));   dH = -c w_s
//
// Which side of a clipping border a token is on is decided on the exact difference in 64 bits, against the border's
// logarithm, so that it does not hang on the rounding of an exponential.  Terms are fp32; their sums are fp64, added up
// per thread, per workgroup, and over the workgroups by a second kernel, always in the same order.
//
// Bound by HBM where there are many tokens (2,048 sequences of 4,096 places, half of them tokens, with reference and
// entropies: 67 MB read and 67 written in 30.7 us, 4.4 TB/s, and 4 us for the join), by its two launches where there are few
// (64 of 512: 5.4 and 1.9 us).
#include "update.h"

namespace rollout {
namespace {

constexpr int LB = 256;
constexpr int kTile = LB * 4;     // tokens of a workgroup's step
// Odd: the steps of a workgroup are kMaxBlocks tiles apart and shall not all fall on the same part of completions, whose ends
// have nothing to do (of 8.4 M tokens, before the penalty's series: 28.7 us, 30.2 with
// 1,536; 29.1 and 32.2 with 1,023 and 1,791).
constexpr int kMaxBlocks = 1279;
// Up to one step of as many threads one workgroup does all, and there is no join (8 sequences of 256 in a graph and eager 6.7
// and 10.7 us, in four workgroups and a join 7.8 and 13.3; two steps, 16 of 512, 9.8 and 10.7, 8.1 and 13.3).
constexpr int kOneThreads = 1024;
constexpr int kJoin = 512;         // threads that join their sums, at most (256 to 512 4.0 us, 1,024 5.5)
constexpr int kSums = 7;          // loss, r, kl, clipped low, clipped high, H, tokens
// Every workgroup adds up to this many lengths itself to know how many tokens there are; more are first added up in
// kCountBlocks sums by a kernel before it (4,096 sequences of 64: 10.5 us by itself, 12 with the kernel; 16,384 of 16: 15.6 and
// 12).
constexpr int kCountSeqs = 8192, kCountBlocks = 256;

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

// Sum of n lengths, in every one of T threads (less than 2^31: exact in any order).
template <int T>
__device__ __forceinline__ int add_lengths(const int32_t* lengths, int lo, int hi, int N, int32_t* red) {
  int v = 0;
#pragma unroll 4
  for (int s = lo + threadIdx.x; s < hi; s += T) v += length_of(lengths, s, N);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) v += red[i];
  return v;
}

__global__ __launch_bounds__(LB) void k_policy_count(const int32_t* __restrict__ lengths, int S, int N, int each,
                                                     int32_t* __restrict__ counts) {
  __shared__ int32_t red[LB / 64];
  const int lo = min((int64_t)blockIdx.x * each, (int64_t)S), hi = (int)min((int64_t)lo + each, (int64_t)S);
  const int v = add_lengths<LB>(lengths, lo, hi, N, red);
  if (threadIdx.x == 0) counts[blockIdx.x] = v;
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
    stream16(p, pack16(v));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = v[j];
  }
}

// Four tokens of a thread: where they stand, and what is read for them.
struct Step {
  int64_t i0;
  int n, s, t, len;  // tokens that exist; sequence and place of the first, that sequence's length and advantage
  float A;
  float lp[4], old[4], ref[4], H[4];
};

__device__ __forceinline__ float seq_weight(int S, int len) { return (float)(1.0 / ((double)S * max(len, 1))); }

// Tokens behind their completions are not read, unless one of the four is not.
__device__ __forceinline__ Step load_step(const PolicyLossArgs& a, int64_t i0, int64_t total) {
  const int N = a.max_len;
  Step q;
  q.i0 = i0;
  q.n = (int)min((int64_t)4, total - i0);
  q.s = (int)((uint32_t)i0 / (uint32_t)N);
  q.t = (int)((uint32_t)i0 - (uint32_t)q.s * (uint32_t)N);
  q.len = length_of(a.lengths, q.s, N);
  q.A = a.adv[q.s];
  if (q.t < q.len || q.t + q.n > N) {
    load4(a.logp + i0, q.n, q.lp);
    if (a.old) load4(a.old + i0, q.n, q.old);
    if (a.ref) load4(a.ref + i0, q.n, q.ref);
    if (a.entropy) load4(a.entropy + i0, q.n, q.H);
  }
  return q;
}

// e^x - 1 - x from x and e^x - 1; infinite at both ends.  It is about x^2 / 2 near zero, where the difference would keep only
// e^x - 1's last bits (1% off at |x| = 1e-5, which is where a run starts): below a half its series, x^2 (1/2! + x/3! + ... +
// x^7/9!), whose next term is 2^-28 of it and which six roundings bring to 6 x 2^-24 of itself; from a half on the
// difference's terms are at most 4.4 times its size.
__device__ __forceinline__ float penalty(float x, float ex) {
  float p = 1.f / 362880.f;
  p = fmaf(p, x, 1.f / 40320.f);
  p = fmaf(p, x, 1.f / 5040.f);
  p = fmaf(p, x, 1.f / 720.f);
  p = fmaf(p, x, 1.f / 120.f);
  p = fmaf(p, x, 1.f / 24.f);
  p = fmaf(p, x, 1.f / 6.f);
  p = fmaf(p, x, 0.5f);
  return fabsf(x) < 0.5f ? p * (x * x) : ex == INFINITY ? ex : ex - x;
}

struct Sums {
  double loss = 0.0, r = 0.0, kl = 0.0, H = 0.0;
  int low = 0, high = 0, tokens = 0;
};

__device__ __forceinline__ void use_step(const PolicyLossArgs& a, const Borders& border, float w_all, const Step& q, Sums& sum) {
  const int S = a.seqs, N = a.max_len;
  int t = q.t, len = q.len;
  float A = q.A, w = a.mean == ROLLOUT_MEAN_SEQUENCE ? seq_weight(S, len) : w_all;
  float gl[4] = {}, gh[4] = {};
  if (q.t < q.len || q.t + q.n > N) {
    int s = q.s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < q.n && t < len) {
        const double d = a.old ? (double)q.lp[j] - (double)q.old[j] : 0.0;
        const float r = expf((float)d);
        const bool high = A > 0.f && d > border.high, low = A < 0.f && d < border.low;
        // no advantage, no term, whatever the ratio
        const float rA = A == 0.f ? 0.f : r * A;
        float tok = high ? -(1.f + a.clip_high) * A : low ? -(1.f - a.clip_low) * A : -rA;
        float g = high || low ? 0.f : -rA;
        if (a.ref) {
          const float x = q.ref[j] - q.lp[j], ex = expm1f(x), kl = penalty(x, ex);
          // no coefficient, no term: 0 times an overflowed exponential is not a number
          if (a.kl_coef != 0.f) {
            tok = fmaf(a.kl_coef, kl, tok);
            g = fmaf(-a.kl_coef, ex, g);
          }
          sum.kl += (double)kl;
        }
        if (a.entropy) {
          if (a.entropy_coef != 0.f) tok = fmaf(-a.entropy_coef, q.H[j], tok);
          sum.H += (double)q.H[j];
        }
        sum.loss += (double)(tok * w);
        sum.r += (double)r;
        sum.low += low;
        sum.high += high;
        sum.tokens += 1;
        gl[j] = g * w;
        gh[j] = -a.entropy_coef * w;
      }
      if (++t == N && j + 1 < q.n) {  // the next sequence begins
        t = 0;
        ++s;
        len = length_of(a.lengths, s, N);
        A = a.adv[s];
        if (a.mean == ROLLOUT_MEAN_SEQUENCE) w = seq_weight(S, len);
      }
    }
  }
  if (a.grad_logp) store4(a.grad_logp + q.i0, q.n, gl);
  if (a.grad_entropy) store4(a.grad_entropy + q.i0, q.n, gh);
}

// Loss and statistics from the whole sums, which the first kSums threads hold.
__device__ __forceinline__ void write_sums(double v, float* loss, float* stats) {
  const double tokens = fmax(__shfl(v, kSums - 1, 64), 1.0);
  if (threadIdx.x == 0 && loss) *loss = (float)v;
  if (threadIdx.x > 0 && threadIdx.x < kSums - 1 && stats) stats[threadIdx.x - 1] = (float)(v / tokens);
}

// A thread does four tokens at a time.  counts: n_counts numbers that add up to the tokens (the lengths, or sums of them).
template <int T>
__global__ __launch_bounds__(T) void k_policy_loss(PolicyLossArgs a, Borders border, const int32_t* __restrict__ counts,
                                                   int n_counts, double* __restrict__ part) {
  __shared__ int32_t red[T / 64];
  __shared__ double sums[T / 64 * kSums];
  const int S = a.seqs, N = a.max_len;
  const int64_t total = (int64_t)S * N, stride = (int64_t)gridDim.x * T * 4;
  Sums sum;
  double all = (double)total;
  if (a.mean == ROLLOUT_MEAN_TOKEN && a.lengths)
    all = max(add_lengths<T>(counts, 0, n_counts, counts == a.lengths ? N : 0x7FFFFFFF, red), 1);
  const float w_all = (float)(1.0 / all);
  for (int64_t i0 = (int64_t)blockIdx.x * T * 4 + threadIdx.x * 4; i0 < total; i0 += stride)
    use_step(a, border, w_all, load_step(a, i0, total), sum);
  const double each[kSums] = {sum.loss, sum.r, sum.kl, (double)sum.low, (double)sum.high, sum.H, (double)sum.tokens};
  const double v = block_sums(each, sums);
  if (gridDim.x > 1) {
    if (threadIdx.x < kSums) part[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = v;
  } else {
    write_sums(v, a.loss, a.stats);  // the only workgroup
  }
}

__global__ __launch_bounds__(kJoin) void k_policy_join(const double* __restrict__ part, int blocks, float* __restrict__ loss,
                                                       float* __restrict__ stats) {
  __shared__ double sums[kJoin / 64 * kSums];
  double v[kSums] = {};
  for (int b = threadIdx.x; b < blocks; b += blockDim.x)
#pragma unroll
    for (int k = 0; k < kSums; ++k) v[k] += part[(size_t)k * blocks + b];
  write_sums(block_sums(v, sums), loss, stats);
}

int blocks_of(int seqs, int max_len) {
  return (int)std::min(((int64_t)seqs * max_len + kTile - 1) / kTile, (int64_t)kMaxBlocks);
}

}  // namespace

size_t policy_loss_workspace(int seqs, int max_len) {
  return kCountBlocks * 4 + (size_t)blocks_of(seqs, max_len) * kSums * 8;
}

hipError_t launch_policy_loss(hipStream_t s, const PolicyLossArgs& a, void* ws) {
  int32_t* sums = (int32_t*)ws;
  double* part = (double*)(sums + kCountBlocks);
  const int blocks = blocks_of(a.seqs, a.max_len);
  const Borders b = {std::log1p(-(double)a.clip_low), std::log1p((double)a.clip_high)};
  const int32_t* counts = a.lengths;
  int n_counts = a.seqs;
  if (a.mean == ROLLOUT_MEAN_TOKEN && a.lengths && a.seqs > kCountSeqs) {
    const int each = std::max(2048, (a.seqs + kCountBlocks - 1) / kCountBlocks);
    n_counts = (a.seqs + each - 1) / each;
    hipLaunchKernelGGL(k_policy_count, dim3(n_counts), dim3(LB), 0, s, a.lengths, a.seqs, a.max_len, each, sums);
    counts = sums;
  }
  const int64_t total = (int64_t)a.seqs * a.max_len;
  if (total > kTile && total <= 4 * kOneThreads) {
    hipLaunchKernelGGL(k_policy_loss<kOneThreads>, dim3(1), dim3(kOneThreads), 0, s, a, b, counts, n_counts, part);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_policy_loss<LB>, dim3(blocks), dim3(LB), 0, s, a, b, counts, n_counts, part);
  if (blocks > 1 && (a.loss || a.stats))
    hipLaunchKernelGGL(k_policy_join, dim3(1), dim3((std::min(blocks, kJoin) + 63) / 64 * 64), 0, s, part, blocks, a.loss,
                       a.stats);
  return hipGetLastError();
}

}  // namespace rollout
