// The gradient of packed attention.
//
//   p_ij = e^(s_ij - lse_i),  D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i)
//   dv_j = sum_i p_ij do_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
//
// (sums over the queries of all heads that share a key's head).  Probabilities are formed again from the scores.  Two kernels
// do so, one for the keys' gradients and one for the queries': seven products of the size of q k^T where one that adds up
// queries' gradients atomically has five, but every sum has an order of its own that does not depend on scheduling.
//
// Probabilities and ds enter the second products as bf16 where the inputs are bf16: each is off by at most 2^-9 of itself, as
// far as the result's own rounding moves it.
#include "packed_attention.h"

namespace rollout {
namespace {

constexpr int kWaves = 4;

// lse in units of log 2 (+inf where a query has no keys: its probabilities are then 0) and D of every row and head.  A wave
// takes 64 * 16 bytes of rows at a time.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_attention_delta(AttentionGradArgs A, float* __restrict__ lse2, float* __restrict__ delta) {
  constexpr int kLanes = HD / Chunk16<T>::N;  // of a row of a head
  const int64_t total = (int64_t)A.n_q * A.heads;
  const int64_t at = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (at >= total) return;
  const int64_t row = at / A.heads;
  const int head = (int)(at - row * A.heads);
  const int c = head * HD + (int)(threadIdx.x % kLanes) * Chunk16<T>::N;
  float o[Chunk16<T>::N], d[Chunk16<T>::N];
  unpack16(load16((const T*)A.out + row * A.out_stride + c), o);
  unpack16(load16((const T*)A.dout + row * A.dout_stride + c), d);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < Chunk16<T>::N; ++i) sum = fmaf(o[i], d[i], sum);
#pragma unroll
  for (int i = kLanes / 2; i > 0; i >>= 1) sum += __shfl_xor(sum, i, 64);
  if (threadIdx.x % kLanes == 0) {
    const float l = A.lse[(size_t)head * A.n_q + row];
    lse2[(size_t)head * A.n_q + row] = l == -INFINITY ? INFINITY : l * kLog2e;
    delta[(size_t)head * A.n_q + row] = sum;
  }
}

// Keys' gradients.  A workgroup takes 128 keys, a wave 32 of them, whose k and v stay in registers, and walks over tiles of 32
// queries of every head that shares them.  Scores have queries as rows and keys as columns, so that a lane holds one key's.
constexpr int kBackKeys = 32 * kWaves, kBackQueries = 32;

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_attention_dkv(AttentionGradArgs A, int slots, int parts,
                                                                                  const float* __restrict__ lse2,
                                                                                  const float* __restrict__ delta,
                                                                                  float* __restrict__ partial) {
  typedef Rows<T, HD> R;
  __shared__ __align__(16) char s_q[2][kBackQueries * R::kBytes];
  __shared__ __align__(16) char s_do[2][kBackQueries * R::kBytes];
  __shared__ __align__(16) float s_stat[2][2][kBackQueries];
  const int w = neighbours_on_die(slots * A.kv_heads * parts);
  if (w < 0) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = A.heads / A.kv_heads, kvh = w / slots / parts, part = w / slots % parts;
  int seq, t0;
  Sequence sk;
  if (!find_tile<kBackKeys>(A.k_starts, A.k_lens, A.n_seqs, A.n_k, w % slots, lane, &seq, &sk, &t0)) return;
  const Sequence sq = sequence_at(A.q_starts, A.q_lens, seq, A.n_q);
  const int behind = sk.len - sq.len;
  const int head0 = kvh * group + group * part / parts, heads = kvh * group + group * (part + 1) / parts - head0;

  const int w_first = t0 + 32 * wave, kj = w_first + a;
  const size_t row = (size_t)sk.start + min(kj, sk.len - 1);
  typename R::Frag kf[HD / 16], vf[HD / 16];
  {
    const T* kp = (const T*)A.k + row * A.k_stride + (size_t)kvh * HD + 8 * half;
    const T* vp = (const T*)A.v + row * A.v_stride + (size_t)kvh * HD + 8 * half;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) kf[c] = load_operand(kp + 16 * c), vf[c] = load_operand(vp + 16 * c);
  }
  // causal: key j is attended from query j - behind on
  auto from = [&](int j) { return A.causal ? max(0, j - behind) : 0; };
  const int first = min(from(t0), sq.len) / kBackQueries;
  const int tiles = (sq.len + kBackQueries - 1) / kBackQueries - first;  // of a head
  const int total = tiles * heads;

  const uint32_t q_stride = (uint32_t)(A.q_stride * sizeof(T)), do_stride = (uint32_t)(A.dout_stride * sizeof(T));
  const char* qb = (const char*)((const T*)A.q + (size_t)sq.start * A.q_stride);
  const char* dob = (const char*)((const T*)A.dout + (size_t)sq.start * A.dout_stride);
  int l_head = head0, l_tile = first;  // what is loaded next
  auto load = [&](int buf) {
    const int i0 = l_tile * kBackQueries, last = sq.len - 1 - i0;
    R::template load<kBackQueries, kWaves>(s_q[buf], qb + (size_t)i0 * q_stride + (size_t)l_head * R::kBytes, q_stride, last, wave, lane);
    R::template load<kBackQueries, kWaves>(s_do[buf], dob + (size_t)i0 * do_stride + (size_t)l_head * R::kBytes, do_stride, last, wave, lane);
    float x = half ? 0.f : INFINITY;  // behind the last query: no probability
    if (wave == 0 && a <= last) x = (half ? delta : lse2)[(size_t)l_head * A.n_q + sq.start + i0 + a];
    if (++l_tile == first + tiles) l_tile = first, ++l_head;
    return x;
  };
  const RowReader<T, HD> rows(lane);
  const ColReader<T, HD> cols(lane);

  f32x16 dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(dk[d]), clear(dv[d]);
  const float c2 = A.scale * kLog2e;
  if (total > 0) {
    const float x = load(0);
    if (wave == 0) s_stat[0][half][a] = x;
  }
  int tile = first;
  for (int it = 0; it < total; ++it) {
    const int buf = it & 1, i0 = tile * kBackQueries;
    if (++tile == first + tiles) tile = first;
    dma_wait_barrier();
    float next = 0.f;
    if (it + 1 < total) next = load(buf ^ 1);
    if (i0 + kBackQueries > from(w_first)) {  // (the same for the whole wave)
      f32x16 s, dp;
      clear(s);
      clear(dp);
#pragma unroll
      for (int c = 0; c < HD / 16; ++c) mma(rows(s_q[buf], 0, c), kf[c], s);
#pragma unroll
      for (int c = 0; c < HD / 16; ++c) mma(rows(s_do[buf], 0, c), vf[c], dp);
      const bool edge = i0 < from(w_first + 31);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = 16 * (e >> 3) + 8 * half + (e & 7);
        s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c2, -s_stat[buf][0][i]));
        if (edge && i0 + i < from(kj)) s[e] = 0.f;
        dp[e] = s[e] * (dp[e] - s_stat[buf][1][i]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        typename R::Frag p, ds;
        operand_of(s, i, p);
        operand_of(dp, i, ds);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          mma(cols(s_do[buf], 16 * i, d), p, dv[d]);
          mma(cols(s_q[buf], 16 * i, d), ds, dk[d]);
        }
      }
    }
    if (wave == 0) s_stat[buf ^ 1][half][a] = next;
  }
  if (kj >= sk.len) return;
  if (parts > 1) {
    const size_t width = (size_t)A.kv_heads * HD, all = (size_t)A.n_k * width;
    float* p = partial + 2 * part * all + row * width + (size_t)kvh * HD + 8 * half;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) store8(p + 32 * d + 16 * i, dk[d], i, A.scale), store8(p + all + 32 * d + 16 * i, dv[d], i, 1.f);
    return;
  }
  T* dkp = (T*)A.dk + row * A.dk_stride + (size_t)kvh * HD + 8 * half;
  T* dvp = (T*)A.dv + row * A.dv_stride + (size_t)kvh * HD + 8 * half;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i) store8(dkp + 32 * d + 16 * i, dk[d], i, A.scale), store8(dvp + 32 * d + 16 * i, dv[d], i, 1.f);
}

// The parts' sums of a tile of keys, in order.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join(AttentionGradArgs A, int slots, int parts, const float* __restrict__ partial) {
  int seq, t0;
  Sequence sk;
  if (!find_tile<kBackKeys>(A.k_starts, A.k_lens, A.n_seqs, A.n_k, (int)blockIdx.x, threadIdx.x & 63, &seq, &sk, &t0)) return;
  const int width = A.kv_heads * A.head_dim, chunks = width / 8, rows = min(kBackKeys, sk.len - t0);
  const size_t all = (size_t)A.n_k * width;
  const bool v = blockIdx.y & 1;
  T* out = (T*)(v ? A.dv : A.dk);
  const int64_t stride = v ? A.dv_stride : A.dk_stride;
  for (int i = (int)(blockIdx.y >> 1) * 256 + threadIdx.x; i < rows * chunks; i += (int)(gridDim.y >> 1) * 256) {
    const size_t row = (size_t)sk.start + t0 + i / chunks;
    const int c = i % chunks * 8;
    const float* p = partial + (v ? all : 0) + row * width + c;
    float t[8], x[8];
    ld8(p, 0, t);
    for (int k = 1; k < parts; ++k) {
      ld8(p + 2 * k * all, 0, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] += x[e];
    }
    T* q = out + row * stride + c;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4*>(q) = pack16(t);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = t[e];
    }
  }
}

// Queries' gradients.  A workgroup takes 128 queries of a head, a wave 32 of them, whose q and do stay in registers, and walks
// over tiles of 32 keys.  Scores have keys as rows and queries as columns, as in the forward pass.
constexpr int kDqQueries = 32 * kWaves, kDqKeys = 32;

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_attention_dq(AttentionGradArgs A, int slots,
                                                                                 const float* __restrict__ lse2,
                                                                                 const float* __restrict__ delta) {
  typedef Rows<T, HD> R;
  __shared__ __align__(16) char s_k[2][kDqKeys * R::kBytes];
  __shared__ __align__(16) char s_v[2][kDqKeys * R::kBytes];
  const int w = neighbours_on_die(slots * A.heads);
  if (w < 0) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = w / slots, kvh = head / (A.heads / A.kv_heads);
  int seq, t0;
  Sequence sq;
  if (!find_tile<kDqQueries>(A.q_starts, A.q_lens, A.n_seqs, A.n_q, slots - 1 - w % slots, lane, &seq, &sq, &t0)) return;
  const Sequence sk = sequence_at(A.k_starts, A.k_lens, seq, A.n_k);
  const int behind = sk.len - sq.len;
  const int w_first = t0 + 32 * wave, qi = w_first + a;
  const size_t row = (size_t)sq.start + min(qi, sq.len - 1);
  typename R::Frag qf[HD / 16], df[HD / 16];
  {
    const T* qp = (const T*)A.q + row * A.q_stride + (size_t)head * HD + 8 * half;
    const T* dp = (const T*)A.dout + row * A.dout_stride + (size_t)head * HD + 8 * half;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) qf[c] = load_operand(qp + 16 * c), df[c] = load_operand(dp + 16 * c);
  }
  const float my_lse = lse2[(size_t)head * A.n_q + row], my_delta = delta[(size_t)head * A.n_q + row];
  auto keys_to = [&](int i) { return A.causal ? max(0, min(sk.len, min(i, sq.len - 1) + behind + 1)) : sk.len; };
  const int mine = keys_to(qi);
  const int w_least = keys_to(w_first), w_most = keys_to(w_first + 31);
  const int tiles = (keys_to(t0 + kDqQueries - 1) + kDqKeys - 1) / kDqKeys;

  const uint32_t k_stride = (uint32_t)(A.k_stride * sizeof(T)), v_stride = (uint32_t)(A.v_stride * sizeof(T));
  const char* kb = (const char*)((const T*)A.k + (size_t)sk.start * A.k_stride + (size_t)kvh * HD);
  const char* vb = (const char*)((const T*)A.v + (size_t)sk.start * A.v_stride + (size_t)kvh * HD);
  auto load = [&](int buf, int it) {
    const int last = sk.len - 1 - it * kDqKeys;
    R::template load<kDqKeys, kWaves>(s_k[buf], kb + (size_t)it * kDqKeys * k_stride, k_stride, last, wave, lane);
    R::template load<kDqKeys, kWaves>(s_v[buf], vb + (size_t)it * kDqKeys * v_stride, v_stride, last, wave, lane);
  };
  const RowReader<T, HD> rows(lane);
  const ColReader<T, HD> cols(lane);

  f32x16 dq[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(dq[d]);
  const float c2 = A.scale * kLog2e;
  if (tiles) load(0, 0);
  for (int it = 0; it < tiles; ++it) {
    const int buf = it & 1, k0 = it * kDqKeys;
    dma_wait_barrier();
    if (it + 1 < tiles) load(buf ^ 1, it + 1);
    if (k0 >= w_most) continue;  // (the same for the whole wave)
    f32x16 s, dp;
    clear(s);
    clear(dp);
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) mma(rows(s_k[buf], 0, c), qf[c], s);
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) mma(rows(s_v[buf], 0, c), df[c], dp);
    const bool edge = k0 + kDqKeys > w_least;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c2, -my_lse));
      if (edge && k0 + 16 * (e >> 3) + 8 * half + (e & 7) >= mine) s[e] = 0.f;
      dp[e] = s[e] * (dp[e] - my_delta);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      typename R::Frag ds;
      operand_of(dp, i, ds);
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) mma(cols(s_k[buf], 16 * i, d), ds, dq[d]);
    }
  }
  if (qi >= sq.len) return;
  T* out = (T*)A.dq + row * A.dq_stride + (size_t)head * HD + 8 * half;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i) store8(out + 32 * d + 16 * i, dq[d], i, A.scale);
}

// The heads that share a key's are dealt out to this many workgroups, whose sums are joined afterwards, where there are few
// tiles of keys.
int head_parts(const AttentionArgs& a) {
  const int group = a.heads / a.kv_heads;
  const int64_t tiles = (int64_t)tile_slots(a.n_k, a.n_seqs, kBackKeys) * a.kv_heads;
  return (int)std::min<int64_t>(group, (1024 + tiles - 1) / tiles);
}

size_t stats_bytes(const AttentionArgs& a) { return ((size_t)a.n_q * a.heads * 4 + 15) / 16 * 16; }

template <typename T, int HD>
hipError_t launch(hipStream_t s, const AttentionGradArgs& a, char* ws) {
  float* lse2 = (float*)ws;
  float* delta = (float*)(ws + stats_bytes(a));
  float* partial = (float*)(ws + 2 * stats_bytes(a));
  const int per = 256 / (HD / Chunk16<T>::N);
  k_attention_delta<T, HD><<<(unsigned)(((int64_t)a.n_q * a.heads + per - 1) / per), 256, 0, s>>>(a, lse2, delta);
  const int slots = tile_slots(a.n_k, a.n_seqs, kBackKeys), parts = head_parts(a);
  k_attention_dkv<T, HD><<<die_grid(slots * a.kv_heads * parts), 64 * kWaves, 0, s>>>(a, slots, parts, lse2, delta, partial);
  if (parts > 1) k_attention_join<T><<<dim3(slots, 2 * 8), 256, 0, s>>>(a, slots, parts, partial);
  const int q_slots = tile_slots(a.n_q, a.n_seqs, kDqQueries);
  k_attention_dq<T, HD><<<die_grid(q_slots * a.heads), 64 * kWaves, 0, s>>>(a, q_slots, lse2, delta);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_of(hipStream_t s, const AttentionGradArgs& a, char* ws) {
  return a.head_dim == 32 ? launch<T, 32>(s, a, ws) : a.head_dim == 64 ? launch<T, 64>(s, a, ws) : launch<T, 128>(s, a, ws);
}

}  // namespace

size_t packed_attention_backward_workspace(const AttentionArgs& a) {
  const int parts = head_parts(a);
  return 2 * stats_bytes(a) + (parts > 1 ? (size_t)parts * 2 * a.n_k * a.kv_heads * a.head_dim * 4 : 0);
}

hipError_t launch_packed_attention_backward(hipStream_t s, int dtype, const AttentionGradArgs& a, void* ws) {
  return dtype == ROLLOUT_DTYPE_BF16 ? launch_of<uint16_t>(s, a, (char*)ws) : launch_of<float>(s, a, (char*)ws);
}

}  // namespace rollout
