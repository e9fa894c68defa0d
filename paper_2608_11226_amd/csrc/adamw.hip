// An AdamW step over many tensors in one launch.
//
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by HBM: every tensor is read and written once.  A table in device memory names the tensors; a workgroup takes a chunk
// of one of them, which it finds in the table by probing 64 entries at a time.  A 7B layer, 233 million elements: fp32 weights with
// a bf16 copy and bf16 gradients 748 us with states in 8 bits (5.0 TB/s), 1,206 with fp32 states (5.4); bf16 weights with states in
// 8 bits 614 (3.8 TB/s), where two hashes and the rounding of three values an element keep the vector ALU busy.
//
// States in 8 bits are e4m3 with a power of two as scale for each run of 128 elements (16 lanes of 8): the first moment, and
// the root of the second, whose range is half as wide.  To nearest, a state would not move at all where a step changes it by
// less than half the distance of two values (1/16 of it; a second moment with b2 = 0.999 changes by a thousandth), so it is
// rounded up or down with the probability that keeps its expectation, by the bits of a counter hash.  So are weights held in
// bf16 alone.
#include "update.h"

namespace rollout {
namespace {

constexpr int kThreads = 256, kStep = kThreads * 8;

// A published finaliser of 32 bits (MurmurHash3's).
__device__ __forceinline__ uint32_t finish32(uint32_t h) {
  h ^= h >> 16;
  h *= 0x85EBCA6Bu;
  h ^= h >> 13;
  h *= 0xC2B2AE35u;
  return h ^ (h >> 16);
}
// SplitMix64's.
__device__ __forceinline__ uint64_t finish64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}
constexpr uint64_t kGold = 0x9E3779B97F4A7C15ull;

typedef uint32_t u32x2_1 __attribute__((ext_vector_type(2), aligned(1), may_alias));

template <typename T>
__device__ __forceinline__ void read8(const T* p, int64_t n, float (&v)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 1) {
      const u32x2_1 w = *reinterpret_cast<const u32x2_1*>(p);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        v[4 * i] = a[0], v[4 * i + 1] = a[1], v[4 * i + 2] = b[0], v[4 * i + 3] = b[1];
      }
    } else if constexpr (sizeof(T) == 2) {
      unpack16(load16(p), v);
    } else {
      float a[4], b[4];
      unpack16(load16(p), a);
      unpack16(load16(p + 4), b);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (i < n) {
      if constexpr (sizeof(T) == 1)
        v[i] = __builtin_amdgcn_cvt_pk_f32_fp8((int)p[i], false)[0];
      else
        v[i] = ldf(p, i);
    }
  }
}
template <typename T>
__device__ __forceinline__ void write8(T* p, int64_t n, const float (&v)[8]) {
  if constexpr (sizeof(T) == 1) {
    // (values of the format already: nothing is rounded here)
    u32x2_1 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], t, true);
    }
    if (n >= 8) {
      *reinterpret_cast<u32x2_1*>(p) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
  } else if (n >= 8) {
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

// maximum over a row of 16 lanes, the same in all of them
__device__ __forceinline__ float row_max(float v) {
#define ROLLOUT_TURN(ctrl) \
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false)))
  ROLLOUT_TURN(0x128);  // row_ror:8, 4, 2, 1
  ROLLOUT_TURN(0x124);
  ROLLOUT_TURN(0x122);
  ROLLOUT_TURN(0x121);
#undef ROLLOUT_TURN
  return v;
}

// x, |x| <= 448, to one of the two e4m3 values beside it: the upper one with the probability that x is on the way there, by 16
// random bits.  (Below 2^-6 the values are 2^-9 apart, as they are between 2^-6 and 2^-5, where the sum is rounded.)
__device__ __forceinline__ float towards(float x, uint32_t bits) {
  const float a = fabsf(x);
  const bool small = a < 0x1p-6f;
  const float z = small ? a + 0x1p-6f : a;
  const float q = __uint_as_float((__float_as_uint(z) + (bits << 4) + 8u) & 0xFFF00000u);
  return copysignf(small ? q - 0x1p-6f : q, x);
}

// b m + c x, each product and the sum rounded: a unit's difference in a moment is enough to send it to the other one of two states
// that are an eighth apart, and the next step with it, and no formula in fp32 says where a compiler fuses
__device__ __forceinline__ float moment(float b, float m, float c, float x) {
#pragma clang fp contract(off)
  const float p = b * m, q = c * x;
  return p + q;
}

// The instruction's root is within a unit.  It is one too large if x <= r (r - unit), and one too small if x > r (r + unit): the
// border between two neighbours, squared, lies within a quarter of a unit squared of their product (Tuckerman's test).  x is 0, or so
// large that fp32 holds the sign of the differences: they are multiples of a unit squared, some 2^-47 of x, and some 2^-24 of it in
// size.  (0 and infinity stay: their neighbours' products are 0 or no numbers.)
__device__ __forceinline__ float nearest_root(float x) {
  const float r = __builtin_amdgcn_sqrtf(x);
  const float below = __uint_as_float(__float_as_uint(r) - 1u), above = __uint_as_float(__float_as_uint(r) + 1u);
  const float lower = fmaf(-below, r, x), upper = fmaf(-above, r, x);
  return lower <= 0.f ? below : upper > 0.f ? above : r;
}
// Where x is smaller than 2^-100 the differences are rounded to multiples of 2^-149, and x is scaled first.
constexpr float kSmallRoot = 0x1p-50f;
__device__ __forceinline__ float nearest_small_root(float x) { return nearest_root(x * 0x1p64f) * 0x1p-32f; }

// A NaN of any pattern as the one that `towards` carries nowhere: added to, those with high bits would be 0.
__device__ __forceinline__ float one_nan(float x) { return x == x ? x : __builtin_nanf(""); }

struct Factors {
  float b1, c1, b2, c2, eps, lr, step, root;  // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float grad;
  uint64_t key;
};

// P, G, S: types of the weights, gradients and states.
template <typename P, typename G, typename S>
__device__ __forceinline__ void update(const AdamwEntry& E, const Factors& F, int64_t lo, int64_t hi) {
  constexpr bool kEight = sizeof(S) == 1, kCoarse = sizeof(P) == 2;
  const float keep = 1.f - F.lr * E.decay;
  // a chunk lies in one run of 2^32 elements
  const uint64_t key = finish64(F.key + kGold * (uint64_t)((lo >> 32 << 20) + 1));
  for (int64_t i = lo + 8 * (int64_t)threadIdx.x; i - 8 * (int64_t)(threadIdx.x) < hi; i += kStep) {
    const int64_t n = hi - i;  // (none left for some lanes of the last step, which still take part in the maxima)
    float p[8], g[8], m[8], v[8];
    const int64_t block = i / 128;
    read8((const P*)E.param + i, n, p);
    read8((const G*)E.grad + i, n, g);
    read8((const S*)E.m + i, n, m);
    read8((const S*)E.v + i, n, v);
    if constexpr (kEight) {
      const float ms = n > 0 ? E.m_scales[block] : 0.f, vs = n > 0 ? E.v_scales[block] : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] *= ms;
        v[e] *= vs;
        v[e] *= v[e];
      }
    }
    float root[8];
    float most_m = 0.f, most_v = 0.f;
    uint32_t most = 0u, least = ~0u;  // of the roots' patterns, 0 apart: as numbers in order, behind them what is none
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = g[e] * F.grad;
      m[e] = moment(F.b1, m[e], F.c1, d);
      v[e] = moment(F.b2, v[e], F.c2, d * d);
      // what a weight's step is divided by may be off by a unit, and a root that becomes a state may not
      root[e] = kEight ? nearest_root(v[e]) : __builtin_amdgcn_sqrtf(v[e]);
      if constexpr (kEight) {
        most_m = fmaxf(most_m, fabsf(m[e]));
        most = max(most, __float_as_uint(root[e]));
        least = min(least, __float_as_uint(root[e]) - 1u);
      }
    }
    if constexpr (kEight) {
      most_v = __uint_as_float(most);
      // rare, and looked for in all eight at once (7B layer 748 us, bf16 weights 614; each scaled, left out or given a pattern by itself
      // 761 and 639)
      if (!(most_m < INFINITY) || !(most_v < INFINITY) || least < __float_as_uint(kSmallRoot)) {
        most_m = 0.f, most_v = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (root[e] > 0.f && root[e] < 2.f * kSmallRoot) root[e] = nearest_small_root(v[e]);
          m[e] = one_nan(m[e]), root[e] = one_nan(root[e]);
          most_m = larger(most_m, fabsf(m[e])), most_v = larger(most_v, root[e]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = p[e] * keep - F.step * m[e] * __builtin_amdgcn_rcpf(root[e] * F.root + F.eps);
    if constexpr (kEight || kCoarse) {
      uint32_t h[8];
      const uint32_t start = (uint32_t)i * 0x9E3779B1u + (uint32_t)key;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = finish32(start + (uint32_t)e * 0x9E3779B1u);
      if constexpr (kEight) {
        const float ms = e4m3_scale(row_max(most_m)), vs = e4m3_scale(row_max(most_v));
        const float mb = 1.f / ms, vb = 1.f / vs;  // exact
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          m[e] = towards(m[e] * mb, h[e] & 0xFFFFu);
          // a second moment that is not 0 stays so, or the next step would divide by eps alone
          const float q = towards(root[e] * vb, h[e] >> 16);
          v[e] = q == 0.f && root[e] > 0.f ? 0x1p-9f : q;
        }
        if (n > 0 && (i & 127) == 0) E.m_scales[block] = ms, E.v_scales[block] = vs;
      }
      if constexpr (kCoarse) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t u = __float_as_uint(p[e]);
          // what is not finite is left to the store's rounding
          if ((u & 0x7F800000u) != 0x7F800000u)
            p[e] = __uint_as_float((u + (finish32(h[e] + (uint32_t)(key >> 32)) & 0xFFFFu)) & 0xFFFF0000u);
        }
      }
    }
    write8((P*)E.param + i, n, p);
    write8((S*)E.m + i, n, m);
    write8((S*)E.v + i, n, v);
    if constexpr (!kCoarse) {
      if (E.copy) write8((uint16_t*)E.copy + i, n, p);
    }
  }
}

__global__ __launch_bounds__(kThreads) void k_adamw(const AdamwEntry* __restrict__ table, int tensors, AdamwArgs A) {
  const int64_t chunk = blockIdx.x;
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = tensors;
  do {  // the last tensor whose first chunk is not behind this one
    const int each = (hi - lo + 63) >> 6, t = lo + lane * each;
    const int k = __popcll(__ballot(t < hi && table[t].first <= chunk)) - 1;
    if (k < 0) return;
    lo += k * each;
    hi = min(lo + each, hi);
  } while (hi - lo > 1);
  const int tensor = __builtin_amdgcn_readfirstlane(lo);
  const AdamwEntry E = table[tensor];
  const int64_t first = (chunk - E.first) * E.chunk, last = min(first + E.chunk, E.n);
  if (first >= last) return;
  Factors F = {A.b1, A.c1, A.b2, A.c2, A.eps, A.lr, 0.f, 0.f, 1.f, 0};
  if (A.grad_scale) F.grad = *A.grad_scale;
  if (!(fabsf(F.grad) < INFINITY)) return;  // gradients that have overflowed: nothing changes
  if (A.d_lr) F.lr = *A.d_lr;
  const int64_t step = A.d_step ? max(*A.d_step, (int64_t)1) : A.step;
  if (A.d_step) {
    F.step = (float)((double)F.lr / -expm1((double)step * A.log_b1));
    F.root = (float)(1.0 / sqrt(-expm1((double)step * A.log_b2)));
  } else {
    F.step = (float)((double)F.lr * A.unbias1);
    F.root = A.unbias2;
  }
  F.key = finish64(A.seed + kGold * (uint64_t)step) + kGold * (uint64_t)tensor;
  const bool p16 = E.kind & 1, g16 = E.kind & 2, s8 = E.kind & 4;
  if (s8) {
    if (p16)
      g16 ? update<uint16_t, uint16_t, uint8_t>(E, F, first, last) : update<uint16_t, float, uint8_t>(E, F, first, last);
    else
      g16 ? update<float, uint16_t, uint8_t>(E, F, first, last) : update<float, float, uint8_t>(E, F, first, last);
  } else {
    if (p16)
      g16 ? update<uint16_t, uint16_t, float>(E, F, first, last) : update<uint16_t, float, float>(E, F, first, last);
    else
      g16 ? update<float, uint16_t, float>(E, F, first, last) : update<float, float, float>(E, F, first, last);
  }
}

}  // namespace

// What a workgroup finds out before its first element (its tensor, factors, the hash's keys) costs nothing where memory is the
// bound, and short chunks spread the load: a 7B layer with fp32 states 1,197 us with one step a workgroup, 1,228 with two and
// 1,249 with four, its bf16 weights with fp32 states 911, 948 and 967.  Rounding by hashes makes arithmetic the bound: bf16 weights
// with states in 8 bits 719, 672 and 614, fp32 weights with them 749, 747 and 747.  A table of few elements needs every workgroup (300 x 1,200 in two
// layers 12.7 us with one step, 16.5 with four), and one of more than 2^34 takes four, for a launch of less than 2^32 threads.
int64_t adamw_chunk(int64_t all, int kind) {
  if (all > (int64_t)1 << 34) return 4 * kStep;
  if (all <= (int64_t)1 << 24 || !(kind & 4)) return kStep;
  return kind & 1 ? 4 * kStep : 2 * kStep;
}

hipError_t launch_adamw(hipStream_t s, const void* table, int tensors, int64_t chunks, const AdamwArgs& a) {
  k_adamw<<<(unsigned)chunks, kThreads, 0, s>>>((const AdamwEntry*)table, tensors, a);
  return hipGetLastError();
}

}  // namespace rollout
