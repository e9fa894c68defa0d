// Log probabilities of given tokens with the entropy and the most likely alternatives of their rows, and the gradient
// of log probability and entropy with respect to the logits.
//
//   c = log2(e) / T,  m = max z,  t_i = (z_i - m) c,  e_i = 2^t_i,  s = sum e_i,  w = sum e_i t_i  (t_i <= 0)
//   log p_i = (z_i - m) / T - ln s,   H = ln s - ln 2 w / s
//   dz_i = (1/T) [ g (1[i = token] - p_i) - h p_i (log p_i + H) ]
//
// One pass over the row with the running maximum, sum and weighted sum of every lane, each corrected when its maximum
// moves (2^((m_old - m_new) c)), joined at the end in a fixed order.  z - m is taken before the scaling: it is exact
// near the maximum and cannot overflow where a mask holds the type's lowest value.
#include "update.h"

namespace rollout {
namespace {

constexpr int RB = 256;  // threads of a row's workgroup
constexpr int RW = RB / 64;
constexpr int kUnits = 4;  // 16-byte loads in flight a lane
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// exponents are taken at least this low: the weighted sum multiplies them with a 0, which an infinity would spoil
constexpr float kLow = -160.f;

struct Soft {
  float m, s, w;
};

__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// a's sums as they stand for maximum m (at least a.m)
__device__ __forceinline__ Soft moved(Soft a, float m, float c) {
  const float mm = finite_or_zero(m);
  const float t = (a.m - mm) * c, f = __builtin_amdgcn_exp2f(t);
  return {m, a.s * f, f * fmaf(a.s, fmaxf(t, kLow), a.w)};
}

// The 16 bytes at element i of a row of V; what lies behind the row reads -inf.
template <typename T>
__device__ __forceinline__ u32x4 load_row(const T* row, int i, int V) {
  constexpr int N = Chunk16<T>::N;
  if (i + N <= V) return load16(row + i);
  float v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = i + j < V ? ldf(row, (size_t)(i + j)) : -INFINITY;
  if constexpr (N == 4) return pack16(v);
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j)  // widened bf16 values: their upper halves are the values
    r[j] = (__float_as_uint(v[(2 * j) % N]) >> 16) | (__float_as_uint(v[(2 * j + 1) % N]) & 0xFFFF0000u);
  return r;
}

// Order of floats as unsigned integers, 0 below all of them; -0 and +0 are equal.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

// The row's top values by (value descending, id ascending), by one wave.  seg holds the keys of the maxima of the row's
// units (64 x N consecutive ids) and is used up; buf holds kMaxTop units.  The top values lie in the top units by
// (maximum, position): a unit that is not among them has as many values before its own as there are alternatives.
// Each of these units then offers its best value not yet taken, and the best offer is taken, top times.
template <typename T>
__device__ void take_top(const T* row, int V, int top, uint32_t* seg, int nseg, u32x4* buf, float m, float inv_t,
                         float ln_s, int32_t* ids, float* logp) {
  constexpr int N = Chunk16<T>::N;
  const int lane = threadIdx.x & 63;
  const int per = (nseg + 63) >> 6, first = lane * per;
  const int n = min(top, nseg);
  uint32_t key = 0;  // lane j: key of the unit it offers, and the unit
  int unit = 0x7FFFFFFF;
  for (int r = 0; r < n; ++r) {
    uint32_t best = 0;
    int at = 0;
    for (int i = 0; i < per && first + i < nseg; ++i) {
      const uint32_t k = seg[first + i];
      if (k > best) best = k, at = first + i;
    }
    const uint32_t top_key = wave_max_u32(best);
    const int owner = __ffsll((unsigned long long)__ballot(best == top_key)) - 1;
    const int chosen = __builtin_amdgcn_readlane(at, owner);
    if (lane == owner) seg[chosen] = 0;
    if (lane == r) key = top_key, unit = chosen;
  }
  // in the order of their ids, so that the first of equal offers is the lowest id
  int rank = 0;
  for (int r = 0; r < n; ++r) rank += __builtin_amdgcn_readlane(unit, r) < unit;
  key = (uint32_t)__builtin_amdgcn_ds_permute(4 * (lane < n ? rank : lane), (int)key);
  unit = __builtin_amdgcn_ds_permute(4 * (lane < n ? rank : lane), unit);
  for (int r = 0; r < n; ++r) {
    const int u = __builtin_amdgcn_readlane(unit, r);
    buf[r * 64 + lane] = load_row(row, (u * 64 + lane) * N, V);
  }
  int last = -1;  // lane j: id of the last of its unit's values that were taken and equal its offer
  for (int r = 0; r < top; ++r) {
    const uint32_t best = wave_max_u32(lane < n ? key : 0);
    const int j = __ffsll((unsigned long long)__ballot(lane < n && key == best)) - 1;
    const int u = __builtin_amdgcn_readlane(unit, j), taken = __builtin_amdgcn_readlane(last, j);
    float v[N];
    unpack16(buf[j * 64 + lane], v);
    const int id0 = (u * 64 + lane) * N;
    int found = 0x7FFFFFFF;
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
      if (key_of(v[i]) == best && id0 + i > taken && id0 + i < V) found = id0 + i;
    const int who = __ffsll((unsigned long long)__ballot(found != 0x7FFFFFFF)) - 1;
    const int id = __builtin_amdgcn_readlane(found, who);
    uint32_t next = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t k = key_of(v[i]);
      if (id0 + i < V && (k < best || (k == best && id0 + i > id))) next = max(next, k);
    }
    next = wave_max_u32(next);
    if (lane == j) key = next, last = next == best ? id : -1;
    if (lane == 0) {
      ids[r] = id;
      logp[r] = (of_key(best) - m) * inv_t - ln_s;
    }
  }
}

// One workgroup a row.
template <typename T, bool TOP>
__global__ __launch_bounds__(RB) void k_logprobs(const T* __restrict__ z, int64_t stride, int rows, int V, float inv_t,
                                                 float c, const int32_t* __restrict__ tokens, int top,
                                                 float* __restrict__ logp, float* __restrict__ entropy,
                                                 float* __restrict__ stats, int32_t* __restrict__ top_ids,
                                                 float* __restrict__ top_logp) {
  constexpr int N = Chunk16<T>::N;
  extern __shared__ u32x4 dyn[];  // TOP: kMaxTop units, then the keys of the units' maxima
  __shared__ Soft part[RW];
  u32x4* buf = dyn;
  uint32_t* seg = reinterpret_cast<uint32_t*>(dyn + top * 64);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nseg = (int)(((int64_t)V + 64 * N - 1) / (64 * N));
  for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const int token = tokens ? tokens[row] : 0;
    if (token < 0) {
      if (threadIdx.x == 0) {
        if (logp) logp[row] = 0.f;
        if (entropy) entropy[row] = 0.f;
        if (stats) stats[2 * (size_t)row] = 0.f, stats[2 * (size_t)row + 1] = 0.f;
      }
      if (TOP && threadIdx.x < top) {
        top_ids[(size_t)row * top + threadIdx.x] = -1;
        top_logp[(size_t)row * top + threadIdx.x] = 0.f;
      }
      continue;
    }
    const T* zr = z + (int64_t)row * stride;
    Soft a = {-INFINITY, 0.f, 0.f};
    for (int u0 = wave * kUnits; u0 < nseg; u0 += RW * kUnits) {
      u32x4 raw[kUnits];
#pragma unroll
      for (int j = 0; j < kUnits; ++j) raw[j] = load_row(zr, min(u0 + j, nseg - 1) * 64 * N + lane * N, V);
      float bm = -INFINITY;
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        float v[N];
        unpack16(raw[j], v);
        float um = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) um = fmaxf(um, v[i]);
        if (u0 + j < nseg) {
          bm = fmaxf(bm, um);
          if (TOP) {
            const uint32_t k = wave_max_u32(key_of(um));
            if (lane == 0) seg[u0 + j] = k;
          }
        }
      }
      const float mm = finite_or_zero(fmaxf(a.m, bm));
      a = moved(a, fmaxf(a.m, bm), c);
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        if (u0 + j >= nseg) break;
        float v[N];
        unpack16(raw[j], v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = (v[i] - mm) * c, e = __builtin_amdgcn_exp2f(t);
          a.s += e;
          a.w = fmaf(e, fmaxf(t, kLow), a.w);
        }
      }
    }
    a = moved(a, wave_max(a.m), c);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    __syncthreads();
    if (lane == 0) part[wave] = a;
    __syncthreads();
    if (wave == 0) {
    float m = part[0].m;
    for (int i = 1; i < RW; ++i) m = fmaxf(m, part[i].m);
    Soft r = {m, 0.f, 0.f};
    for (int i = 0; i < RW; ++i) {
      const Soft q = moved(part[i], m, c);
      r.s += q.s;
      r.w += q.w;
    }
    const bool bad = !(r.s == r.s);
    const float ln_s = logf(r.s);
    if (lane == 0) {
      const float x = token < V ? ldf(zr, (size_t)token) : NAN;
      if (logp) logp[row] = bad || token >= V ? NAN : x == -INFINITY ? -INFINITY : (x - m) * inv_t - ln_s;
      if (entropy) entropy[row] = bad ? NAN : m == -INFINITY ? 0.f : ln_s - kLn2 * r.w / r.s;
      if (stats) stats[2 * (size_t)row] = bad ? NAN : m, stats[2 * (size_t)row + 1] = bad ? NAN : ln_s;
    }
    if (TOP) {
      if (bad) {
        if (lane < top) top_ids[(size_t)row * top + lane] = -1, top_logp[(size_t)row * top + lane] = NAN;
      } else {
        // a row of -inf alone: every difference to the maximum is taken as -inf
        take_top(zr, V, top, seg, nseg, buf, finite_or_zero(m), inv_t, m == -INFINITY ? 0.f : ln_s,
                 top_ids + (size_t)row * top, top_logp + (size_t)row * top);
      }
    }
    }
    if (TOP) __syncthreads();  // the next row's keys
  }
}

// z and dz may be the same matrix: a thread reads its values before it writes them.
template <typename T>
__global__ __launch_bounds__(RB) void k_logprobs_backward(const T* z, int64_t stride, int rows, int V,
                                                          float inv_t, const int32_t* __restrict__ tokens,
                                                          const float* __restrict__ stats,
                                                          const float* __restrict__ entropy,
                                                          const float* __restrict__ gp, const float* __restrict__ hp,
                                                          T* dz, int64_t dz_stride) {
  constexpr int N = Chunk16<T>::N;
  for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* zr = z + (int64_t)row * stride;
    T* dr = dz + (int64_t)row * dz_stride;
    const int token = tokens[row];
    const float m = stats[2 * (size_t)row], ln_s = stats[2 * (size_t)row + 1];
    const float g = gp[row], h = hp ? hp[row] : 0.f, H = hp ? entropy[row] : 0.f;
    const bool dead = token < 0 || (g == 0.f && h == 0.f) || m == -INFINITY;
    const float c = inv_t * kLog2e, l2 = ln_s * kLog2e;
    for (int i = threadIdx.x * N; i < V; i += RB * N) {
      float v[N], d[N];
      if (!dead) unpack16(load_row(zr, i, V), v);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (dead) {
          d[j] = 0.f;
        } else if (token >= V) {
          d[j] = NAN;
        } else {
          const float t = fmaf(v[j] - m, c, -l2), p = __builtin_amdgcn_exp2f(t);
          const float k = fmaf(h, fmaf(fmaxf(t, kLow), kLn2, H), g);
          d[j] = (i + j == token ? fmaf(-p, k, g) : -p * k) * inv_t;
        }
      }
      if (i + N <= V) {
        store16(dr + i, pack16(d));
      } else {
        for (int j = 0; i + j < V; ++j) put(dr + i + j, d[j]);
      }
    }
  }
}

template <typename T>
void forward(hipStream_t s, const LogprobArgs& a) {
  constexpr int N = Chunk16<T>::N;
  const float inv_t = 1.f / a.temperature, c = (float)(1.4426950408889634 / (double)a.temperature);
  const unsigned grid = (unsigned)std::min(a.rows, 1 << 20);
  if (a.top) {
    const size_t lds = (size_t)a.top * 1024 + ((size_t)a.vocab + 64 * N - 1) / (64 * N) * 4;
    hipLaunchKernelGGL((k_logprobs<T, true>), dim3(grid), dim3(RB), lds, s, (const T*)a.z, a.stride, a.rows, a.vocab, inv_t,
                       c, a.tokens, a.top, a.logp, a.entropy, a.stats, a.top_ids, a.top_logp);
  } else {
    hipLaunchKernelGGL((k_logprobs<T, false>), dim3(grid), dim3(RB), 0, s, (const T*)a.z, a.stride, a.rows, a.vocab, inv_t, c,
                       a.tokens, 0, a.logp, a.entropy, a.stats, a.top_ids, a.top_logp);
  }
}

template <typename T>
void backward(hipStream_t s, const LogprobGradArgs& a) {
  hipLaunchKernelGGL(k_logprobs_backward<T>, dim3((unsigned)std::min(a.rows, 1 << 20)), dim3(RB), 0, s, (const T*)a.z,
                     a.stride, a.rows, a.vocab, 1.f / a.temperature, a.tokens, a.stats, a.entropy, a.g, a.h, (T*)a.dz,
                     a.dz_stride);
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) { return 0; }

hipError_t launch_logprobs(hipStream_t s, int dtype, const LogprobArgs& a, void* ws) {
  dtype == ROLLOUT_DTYPE_BF16 ? forward<uint16_t>(s, a) : forward<float>(s, a);
  return hipGetLastError();
}

hipError_t launch_logprobs_backward(hipStream_t s, int dtype, const LogprobGradArgs& a) {
  dtype == ROLLOUT_DTYPE_BF16 ? backward<uint16_t>(s, a) : backward<float>(s, a);
  return hipGetLastError();
}

}  // namespace rollout
