// Root-mean-square norm of the residual stream, with the addition that comes before it, and its gradient.
//
//   h = x + delta (rounded to x's type),  r = 1 / sqrt(mean h^2 + eps),  y = h r gain
//   dx_i = r (t_i - xhat_i mean_k(t_k xhat_k)) + inner_i,  t = dy gain, xhat = h r;   dgain_i = sum over rows of dy_i xhat_i
//
// A row is read once and stays in registers, 8 neighbours of it per thread and step: of one wave up to 1,024 values, above that
// of as many waves as make it one step, up to sixteen.  An output in 8 bits (e4m3) takes a second reduction, the largest |y|, and has the
// smallest power of two as scale that brings it to at most 448: a power of two takes nothing from the 4 bits of a value.
//
// Bound by HBM: 16,384 x 8,192 fp32 with a bf16 addition to 8 bits 252 us (5.9 TB/s), 12,288 x 3,584 backward 109 (5.6 TB/s) and 4.8
// for the gain's join, 8,192 x 3,584 in bf16 37 (6.4 TB/s, much of it from the last cache).  Few rows are a launch: 64 x 3,584
// 3.5 us, 259 x 1,003 backward 5.4 and 2.9.  A row over more threads of one step each beats fewer of several (7B backward 113 us with
// 512 threads, 123 with 256 and two steps; 8,192 wide forward 252 with 1,024, 268 with 512 and two).
#include "update.h"

namespace rollout {
namespace {

struct None {};

// Eight neighbours of a row from p on, of which n are the row's.  A row's last ones are read with those before them, in the same
// 16-byte loads as all others, and moved to their places by `settle` once everything is on the way: read one by one they would
// be a chain of trips to memory.  Rows of fewer than eight (`narrow`) have none before them.
template <typename T>
__device__ __forceinline__ void read8(const T* p, int n, bool narrow, float (&v)[8]) {
  if (narrow) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? ldf(p, i) : 0.f;
    return;
  }
  p += min(0, n - 8);
  if constexpr (sizeof(T) == 2) {
    unpack16(load16(p), v);
  } else {
    float a[4], b[4];
    unpack16(load16(p), a);
    unpack16(load16(p + 4), b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
}
__device__ __forceinline__ void settle(int n, bool narrow, float (&v)[8]) {
  if (n >= 8 || narrow) return;
#pragma unroll
  for (int by = 4; by > 0; by /= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((8 - n) & by) v[i] = i + by < 8 ? v[i + by < 8 ? i + by : 0] : 0.f;
}
template <typename T>
__device__ __forceinline__ void write8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 2) {
      store16(p, pack16(v));
    } else {
      const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
      store16(p, pack16(a));
      store16(p + 4, pack16(b));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) put(p + i, v[i]);
  }
}
// e4m3, to nearest, ties to even; what is not a number, or infinite, becomes NaN
__device__ __forceinline__ void write8(uint8_t* p, int n, const float (&v)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], t, true);
  }
  typedef uint32_t Raw __attribute__((ext_vector_type(2), aligned(1), may_alias));
  if (n >= 8) {
    *reinterpret_cast<Raw*>(p) = Raw{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

// Sum (or maximum) over the W threads of a row, of which v is a wave's, the same in all of them; red: W / 64 values.
template <int W, typename A = float, typename F>
__device__ __forceinline__ A row_reduce(float v, float* red, F f) {
  A all = v;
  if constexpr (W > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    all = red[0];
#pragma unroll
    for (int i = 1; i < W / 64; ++i) all = f(all, (A)red[i]);
  }
  return all;
}

// 1 / sqrt(x), rounded once: a step of Newton's from the instruction's result, where that is within a unit (fp32's three
// roundings, of the mean, the root and its reciprocal, moved 1.4 times as many e4m3 codes over a border)
__device__ __forceinline__ float inverse_root(double x) {
  const float f = (float)x;
  if (!(f >= 0x1p-126f && f < INFINITY)) return 1.f / sqrtf(f);
  const double r = __builtin_amdgcn_rsqf(f);
  return (float)fma(0.5 * r, fma(-x * r, r, 1.0), r);
}

// W threads a row (64: four rows in a workgroup), S steps of 8 values each.  D: type of what is added, or None.
template <typename X, typename D, typename Y, int W, int S>
__global__ __launch_bounds__(W < 256 ? 256 : W) void k_rms_norm(NormArgs A) {
  constexpr bool kAdds = !std::is_same<D, None>::value;
  __shared__ float red[2][W / 64];
  const int t = threadIdx.x % W;
  const int64_t row = (int64_t)blockIdx.x * (W < 256 ? 256 / W : 1) + threadIdx.x / W;
  if (row >= A.rows) return;  // (a whole wave)
  const X* x = (const X*)A.x + row * A.dim;
  const D* d = (const D*)A.delta + row * A.dim;
  X* to = (X*)A.h + row * A.dim;
  const bool narrow = A.dim < 8;
  float h[S][8], g[S][8];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int i = 8 * (t + s * W), n = A.dim - i;
    if (n <= 0) continue;
    float v[8];
    read8(x + i, n, narrow, h[s]);
    if constexpr (kAdds) read8(d + i, n, narrow, v);
    if (A.gain) read8(A.gain + i, n, narrow, g[s]);  // (in flight with the others)
    settle(n, narrow, h[s]);
    if constexpr (kAdds) {
      settle(n, narrow, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[s][e] += v[e];
        if constexpr (sizeof(X) == 2) h[s][e] = bf16_to_f32(round_bf16(h[s][e]));  // the norm is of what is stored
      }
      write8(to + i, n, h[s]);
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (8 * (t + s * W) < A.dim)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(h[s][e], h[s][e], sum);
  const double all = row_reduce<W, double>(wave_sum_f32(sum), red[0], [](double a, double b) { return a + b; });
  const float r = inverse_root(all * A.per_value + (double)A.eps);
  if (A.rstd && t == 0) A.rstd[row] = r;
  float most = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int i = 8 * (t + s * W);
    if (i >= A.dim) continue;
    if (A.gain) settle(A.dim - i, narrow, g[s]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[s][e] *= r;
      if (A.gain) h[s][e] *= g[s][e];
      if constexpr (sizeof(Y) == 1) most = larger(most, fabsf(h[s][e]));
    }
  }
  float by = 1.f;
  if constexpr (sizeof(Y) == 1) {
    most = row_reduce<W>(wave_max_f32(most), red[1], [](float a, float b) { return fmaxf(a, b); });
    const float scale = e4m3_scale(most);
    by = 1.f / scale;  // exact
    if (t == 0) A.scales[row] = scale;
  }
  Y* y = (Y*)A.y + row * A.dim;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int i = 8 * (t + s * W);
    if (i >= A.dim) continue;
    if constexpr (sizeof(Y) == 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[s][e] *= by;
    write8(y + i, A.dim - i, h[s]);
  }
}

// Rows `worker`, `worker` + workers, ... of the gradient; the worker's sum of dy xhat stays in registers, and the workgroup's (of
// four workers where a row is a wave's) ends in partial[workgroup].
template <typename X, typename G, typename O, int W, int S>
__global__ __launch_bounds__(W < 256 ? 256 : W) void k_rms_norm_backward(NormGradArgs A, int workers, float* __restrict__ partial) {
  __shared__ float red[2][W / 64];
  const int t = threadIdx.x % W;
  const int worker = (int)blockIdx.x * (W < 256 ? 256 / W : 1) + threadIdx.x / W;
  float sum[S][8] = {};
  float* turn = red[0];
  float* other = red[1];
  const bool narrow = A.dim < 8;
  constexpr bool kEarly = S < 4;  // the inner gradient is in flight with the others, where registers allow
  for (int64_t row = worker; row < A.rows; row += workers) {
    const X* hp = (const X*)A.h + row * A.dim;
    const G* dyp = (const G*)A.dy + row * A.dim;
    const float r = A.rstd[row];
    float xhat[S][8], g[S][8], v[S][8] = {};
    float dot = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int i = 8 * (t + s * W);
      if (i >= A.dim) continue;
      read8(hp + i, A.dim - i, narrow, xhat[s]);
      read8(dyp + i, A.dim - i, narrow, g[s]);
      if (kEarly && A.inner) read8((const O*)A.inner + row * A.dim + i, A.dim - i, narrow, v[s]);
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int i = 8 * (t + s * W);
      if (i >= A.dim) continue;
      float gain[8];
      if (A.gain) read8(A.gain + i, A.dim - i, narrow, gain);
      settle(A.dim - i, narrow, xhat[s]);
      settle(A.dim - i, narrow, g[s]);
      if (kEarly) settle(A.dim - i, narrow, v[s]);
      if (A.gain) settle(A.dim - i, narrow, gain);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xhat[s][e] *= r;
        sum[s][e] = fmaf(g[s][e], xhat[s][e], sum[s][e]);
        if (A.gain) g[s][e] *= gain[e];
        dot = fmaf(g[s][e], xhat[s][e], dot);
      }
    }
    dot = row_reduce<W>(wave_sum_f32(dot), turn, [](float a, float b) { return a + b; }) / (float)A.dim;
    float* swap = turn;
    turn = other;
    other = swap;
    O* to = (O*)A.dx + row * A.dim;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int i = 8 * (t + s * W);
      if (i >= A.dim) continue;
      if (!kEarly && A.inner) {
        read8((const O*)A.inner + row * A.dim + i, A.dim - i, narrow, v[s]);
        settle(A.dim - i, narrow, v[s]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[s][e] = fmaf(r, g[s][e] - xhat[s][e] * dot, v[s][e]);
      write8(to + i, A.dim - i, v[s]);
    }
  }
  if (!partial) return;
  if constexpr (W == 64) {
    __shared__ float all[3][S][8][64];
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (wave) all[wave - 1][s][e][t] = sum[s][e];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[s][e] = ((sum[s][e] + all[0][s][e][t]) + all[1][s][e][t]) + all[2][s][e][t];
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int i = 8 * (t + s * W);
    if (i < A.dim) write8(partial + (int64_t)blockIdx.x * A.dim + i, A.dim - i, sum[s]);
  }
}

// Sums of the workgroups' columns in a fixed order: 32 columns a workgroup here, four of them a thread, every 64th row of them a
// row of threads, of which a wave holds eight.
constexpr int kJoinRows = 64;
__global__ __launch_bounds__(8 * kJoinRows) void k_norm_join(const float* __restrict__ partial, int rows, int dim, int accumulate,
                                                            float* __restrict__ dgain) {
  __shared__ float red[kJoinRows / 8][32];
  const int c = threadIdx.x & 7, k = threadIdx.x >> 3, col = (int)blockIdx.x * 32 + 4 * c;
  const int mine = (int)blockIdx.x * 32 + threadIdx.x;
  const bool ends = threadIdx.x < 32 && mine < dim;
  const float before = ends && accumulate ? dgain[mine] : 0.f;
  float sum[4] = {};
#pragma unroll 4
  for (int w = k; w < rows; w += kJoinRows) {
    const float* p = partial + (int64_t)w * dim + col;
    float v[4] = {};
    if (col + 4 <= dim)
      unpack16(load16(p), v);
    else
      for (int e = 0; e < dim - col; ++e) v[e] = p[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int apart = 8; apart < 64; apart *= 2) sum[e] += __shfl_xor(sum[e], apart, 64);
    if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][4 * c + e] = sum[e];
  }
  __syncthreads();
  if (!ends) return;
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < kJoinRows / 8; ++i) total += red[i][threadIdx.x];
  dgain[mine] = accumulate ? before + total : total;
}

}  // namespace

int norm_threads(int dim) { return dim <= 1024 ? 64 : dim <= 2048 ? 256 : dim <= 4096 ? 512 : 1024; }

namespace {

// f(W, S) with the threads of a row and the steps of 8 values that they take, as constants
template <typename F>
void by_dim(int dim, F f) {
  using std::integral_constant;
  if (dim <= 512)
    f(integral_constant<int, 64>(), integral_constant<int, 1>());
  else if (dim <= 1024)
    f(integral_constant<int, 64>(), integral_constant<int, 2>());
  else if (dim <= 2048)
    f(integral_constant<int, 256>(), integral_constant<int, 1>());
  else if (dim <= 4096)
    f(integral_constant<int, 512>(), integral_constant<int, 1>());
  else if (dim <= 8192)
    f(integral_constant<int, 1024>(), integral_constant<int, 1>());
  else if (dim <= 16384)
    f(integral_constant<int, 1024>(), integral_constant<int, 2>());
  else
    f(integral_constant<int, 1024>(), integral_constant<int, 4>());
}

template <typename X, typename D, typename Y>
hipError_t forward(hipStream_t s, const NormArgs& a) {
  by_dim(a.dim, [&](auto W, auto S) {
    constexpr int kRows = W < 256 ? 256 / W : 1;
    k_rms_norm<X, D, Y, W, S><<<(a.rows + kRows - 1) / kRows, kRows * W, 0, s>>>(a);
  });
  return hipGetLastError();
}
template <typename X, typename D>
hipError_t forward_to(hipStream_t s, int y_dtype, const NormArgs& a) {
  return y_dtype == ROLLOUT_DTYPE_FP32   ? forward<X, D, float>(s, a)
         : y_dtype == ROLLOUT_DTYPE_BF16 ? forward<X, D, uint16_t>(s, a)
                                         : forward<X, D, uint8_t>(s, a);
}
template <typename X>
hipError_t forward_from(hipStream_t s, int delta_dtype, int y_dtype, const NormArgs& a) {
  return !a.delta                            ? forward_to<X, None>(s, y_dtype, a)
         : delta_dtype == ROLLOUT_DTYPE_FP32 ? forward_to<X, float>(s, y_dtype, a)
                                             : forward_to<X, uint16_t>(s, y_dtype, a);
}

// As many as the card holds at a time, by the registers that they take: more would wait for the others' places, and each has as
// many rows as they (12,288 x 3,584 114 us with 512, 120 with 768, 131 with 1,024; 8,192 x 8,192 172 with 256, 177 with 512;
// 65,536 x 640 124 with 4,096, 146 with 6,144; 60,000 x 300 83 with 6,144, 88 with 4,096, 107 with 8,192).
int workers_of(int rows, int dim) {
  return std::min(rows, dim <= 512 ? 6144 : dim <= 1024 ? 4096 : dim <= 2048 ? 1536 : dim <= 4096 ? 512 : 256);
}
int groups_of(int rows, int dim) {
  const int each = norm_threads(dim) == 64 ? 4 : 1;
  return (workers_of(rows, dim) + each - 1) / each;
}

template <typename X, typename G, typename O>
hipError_t backward(hipStream_t s, const NormGradArgs& a, float* partial) {
  const int n = workers_of(a.rows, a.dim), groups = groups_of(a.rows, a.dim);
  by_dim(a.dim, [&](auto W, auto S) {
    constexpr int kRows = W < 256 ? 256 / W : 1;
    k_rms_norm_backward<X, G, O, W, S><<<groups, kRows * W, 0, s>>>(a, n, a.dgain ? partial : nullptr);
    if (a.dgain) k_norm_join<<<(a.dim + 31) / 32, 8 * kJoinRows, 0, s>>>(partial, groups, a.dim, a.accumulate, a.dgain);
  });
  return hipGetLastError();
}
template <typename X, typename G>
hipError_t backward_to(hipStream_t s, int dx_dtype, const NormGradArgs& a, float* p) {
  return dx_dtype == ROLLOUT_DTYPE_FP32 ? backward<X, G, float>(s, a, p) : backward<X, G, uint16_t>(s, a, p);
}
template <typename X>
hipError_t backward_from(hipStream_t s, int dy_dtype, int dx_dtype, const NormGradArgs& a, float* p) {
  return dy_dtype == ROLLOUT_DTYPE_FP32 ? backward_to<X, float>(s, dx_dtype, a, p) : backward_to<X, uint16_t>(s, dx_dtype, a, p);
}

}  // namespace

hipError_t launch_rms_norm(hipStream_t s, int x_dtype, int delta_dtype, int y_dtype, const NormArgs& a) {
  return x_dtype == ROLLOUT_DTYPE_FP32 ? forward_from<float>(s, delta_dtype, y_dtype, a)
                                       : forward_from<uint16_t>(s, delta_dtype, y_dtype, a);
}

// (that of a large call does for small ones, which may have more workers)
size_t rms_norm_backward_workspace(int rows, int dim) {
  size_t most = 0;
  for (int d : {512, 1024, 2048, 4096, kMaxNormDim}) most = std::max(most, (size_t)groups_of(rows, std::min(d, dim)) * std::min(d, dim));
  return 4 * most;
}

hipError_t launch_rms_norm_backward(hipStream_t s, int h_dtype, int dy_dtype, int dx_dtype, const NormGradArgs& a, void* ws) {
  return h_dtype == ROLLOUT_DTYPE_FP32 ? backward_from<float>(s, dy_dtype, dx_dtype, a, (float*)ws)
                                       : backward_from<uint16_t>(s, dy_dtype, dx_dtype, a, (float*)ws);
}

}  // namespace rollout
