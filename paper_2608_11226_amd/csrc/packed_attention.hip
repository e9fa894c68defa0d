// Attention of packed sequences, with the log-sum-exp that its gradient needs.
//
//   s_ij = scale q_i k_j  (keys j <= i + len_k - len_q if causal);  lse_i = log sum_j e^s_ij;  o_i = sum_j e^(s_ij - lse_i) v_j
//
// A workgroup takes 128 queries of a head, a wave 32 of them, and walks over tiles of 64 keys once, with the running maximum
// and sum of each query in 32 bits.  Scores are formed transposed (keys as rows, queries as columns), so that a lane holds one
// query's: maximum and sum are the lane's own but for one exchange with the lane 32 away, and the probabilities' registers are
// the operand of the product with the values.
#include "packed_attention.h"

namespace rollout {
namespace {

constexpr int kWaves = 4;
constexpr int kQueries = 32 * kWaves;  // of a workgroup
constexpr int kKeys = 64;              // of a tile
// the running maximum follows only when a query outgrows it by 2^kGrow: until then its probabilities are that much above 1,
// which costs no precision, and the output need not be scaled
constexpr float kGrow = 8.f;

// maximum over a lane and the lane 32 away
__device__ __forceinline__ float pair_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename T, int HD>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_packed_attention(AttentionArgs A, int slots) {
  typedef Rows<T, HD> R;
  __shared__ __align__(16) char s_k[2][kKeys * R::kBytes];
  __shared__ __align__(16) char s_v[2][kKeys * R::kBytes];
  const int w = neighbours_on_die(slots * A.heads);
  if (w < 0) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = w / slots, kvh = head / (A.heads / A.kv_heads);
  int seq, t0;
  Sequence sq;
  // a sequence's last queries, which have the most keys, first
  if (!find_tile<kQueries>(A.q_starts, A.q_lens, A.n_seqs, A.n_q, slots - 1 - w % slots, lane, &seq, &sq, &t0)) return;
  const Sequence sk = sequence_at(A.k_starts, A.k_lens, seq, A.n_k);

  const int behind = sk.len - sq.len;  // causal: query i attends keys 0 .. i + behind
  const int w_first = t0 + 32 * wave, qi = w_first + a;
  const size_t row = (size_t)sq.start + min(qi, sq.len - 1);
  typename R::Frag qf[HD / 16];
  const T* qp = (const T*)A.q + row * A.q_stride + (size_t)head * HD + 8 * half;
#pragma unroll
  for (int c = 0; c < HD / 16; ++c) qf[c] = load_operand(qp + 16 * c);
  auto keys_to = [&](int i) { return A.causal ? max(0, min(sk.len, min(i, sq.len - 1) + behind + 1)) : sk.len; };
  const int mine = keys_to(qi);                                    // of this lane's query
  const int w_least = keys_to(w_first), w_most = keys_to(w_first + 31);  // of the wave's
  const int tiles = (keys_to(t0 + kQueries - 1) + kKeys - 1) / kKeys;

  const uint32_t k_stride = (uint32_t)(A.k_stride * sizeof(T)), v_stride = (uint32_t)(A.v_stride * sizeof(T));
  const char* kb = (const char*)((const T*)A.k + (size_t)sk.start * A.k_stride + (size_t)kvh * HD);
  const char* vb = (const char*)((const T*)A.v + (size_t)sk.start * A.v_stride + (size_t)kvh * HD);
  auto load = [&](int buf, int it) {
    const int last = sk.len - 1 - it * kKeys;
    R::template load<kKeys, kWaves>(s_k[buf], kb + (size_t)it * kKeys * k_stride, k_stride, last, wave, lane);
    R::template load<kKeys, kWaves>(s_v[buf], vb + (size_t)it * kKeys * v_stride, v_stride, last, wave, lane);
  };
  const RowReader<T, HD> rows(lane);
  const ColReader<T, HD> cols(lane);

  f32x16 o[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(o[d]);
  const float c2 = A.scale * kLog2e;  // scores are kept in units of log 2
  float m_run = -3.4e38f, l_run = 0.f;
  if (tiles) load(0, 0);
  for (int it = 0; it < tiles; ++it) {
    dma_wait_barrier();  // tile `it` is there for every wave, and nobody reads the other buffer any more
    if (it + 1 < tiles) load((it + 1) & 1, it + 1);
    const int k0 = it * kKeys;
    if (k0 >= w_most) continue;  // (the same for the whole wave)
    f32x16 s[kKeys / 32];
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b) {
      clear(s[b]);
#pragma unroll
      for (int c = 0; c < HD / 16; ++c) mma(rows(s_k[it & 1], 32 * b, c), qf[c], s[b]);
    }
    if (k0 + kKeys > w_least) {
#pragma unroll
      for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 32 * b + 16 * (e >> 3) + 8 * half + (e & 7) >= mine) s[b][e] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
    mx = pair_max(mx) * c2;
    if (__any(mx > m_run + kGrow)) {
      const float m_new = fmaxf(m_run, mx);
      const float shrink = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= shrink;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= shrink;
    }
#pragma unroll
    for (int b = 0; b < kKeys / 32; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], c2, -m_run));
        l_run += s[b][e];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // bf16 probabilities: each is off by at most 2^-9 of itself, as far as the output's own rounding moves it, and the
        // errors of many keys largely cancel; their sum is that of the unrounded ones
        typename R::Frag p;
        operand_of(s[b], i, p);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) mma(cols(s_v[it & 1], 32 * b + 16 * i, d), p, o[d]);
      }
    }
  }
  if (qi >= sq.len) return;
  const float l = l_run + __shfl_xor(l_run, 32, 64);
  // a query without keys: nothing, and the logarithm of nothing
  const float by = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  T* op = (T*)A.out + row * A.out_stride + (size_t)head * HD + 8 * half;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i) store8(op + 32 * d + 16 * i, o[d], i, by);
  if (half == 0) A.lse[(size_t)head * A.n_q + row] = l == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l)) * kLn2;
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const AttentionArgs& a) {
  const int slots = tile_slots(a.n_q, a.n_seqs, kQueries);
  k_packed_attention<T, HD><<<die_grid(slots * a.heads), 64 * kWaves, 0, s>>>(a, slots);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_of(hipStream_t s, const AttentionArgs& a) {
  return a.head_dim == 32 ? launch<T, 32>(s, a) : a.head_dim == 64 ? launch<T, 64>(s, a) : launch<T, 128>(s, a);
}

}  // namespace

size_t packed_attention_workspace(const AttentionArgs&) { return 0; }

hipError_t launch_packed_attention(hipStream_t s, int dtype, const AttentionArgs& a, void*) {
  return dtype == ROLLOUT_DTYPE_BF16 ? launch_of<uint16_t>(s, a) : launch_of<float>(s, a);
}

}  // namespace rollout
