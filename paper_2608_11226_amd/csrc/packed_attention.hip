// Attention of packed sequences, with the log-sum-exp that its gradient needs.
//
//   s_ij = scale q_i k_j  (keys j <= i + len_k - len_q if causal);  lse_i = log sum_j e^s_ij;  o_i = sum_j e^(s_ij - lse_i) v_j
//
// A workgroup takes 128 rows, a row being a token's query of one of the heads that share a key's, a wave 32 of them, and walks
// over tiles of 64 keys once, with the running maximum and sum of each row in 32 bits.  Scores are formed transposed (keys as
// rows, queries as columns), so that a lane holds one query's: maximum and sum are the lane's own but for one exchange with the
// lane 32 away, and the probabilities' registers are the operand of the product with the values.
//
// Where there are few rows for the card, the keys of each are dealt out to several workgroups, whose sums a second kernel joins.
//
// Heads that share a key's are taken together, which reads keys once for all of them: one token of 16 sequences over 1,024 to
// 8,192 keys at 64 on 8 heads of 128 takes 61 us and the join 5 (302 MB read at 5.0 TB/s, memory the bound; 428 us with a head
// a workgroup and without parts).  Long sequences are bound by the matrix products: 8,192 tokens at 40 on 8 heads 655 us, 1,050
// TFLOP/s in bf16 (products are at work in 0.61 of the compute units' cycles; exponentials and maxima fill much of the rest), at 64
// dimensions 680; fp32 102 of the 154 that fp32 products reach.  Short ones, 16 of 257 to 768 tokens at 28 on 4 heads, 60 us, 545
// TFLOP/s: walks of some five tiles, whose beginning (its place, rows and first tile, a trip to memory after the other) and end are
// hidden by the compute unit's other workgroup alone (464 sequences of 18 tokens, a tile each, 40 us).  Exponentials issued
// between the products of the tile before them took the long case from 655 to 694 us, a
// higher priority of waves at their products changed nothing, and half tiles with four on the way took few tokens' from 29 to 32.
#include "packed_attention.h"

namespace rollout {
namespace {

constexpr int kWaves = 4;
constexpr int kQueries = 32 * kWaves;  // of a workgroup
constexpr int kKeys = 64;              // of a tile
// the running maximum follows only when a query outgrows it by 2^kGrow: until then its probabilities are that much above 1,
// which costs no precision, and the output need not be scaled (8,192 tokens 655 us, with 0 691; 7B update 61, with 0 65)
constexpr float kGrow = 8.f;

// maximum over a lane and the lane 32 away
__device__ __forceinline__ float pair_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// partial: HD sums, then the maximum and the sum, of every part, token and head.
template <int HD>
__device__ __forceinline__ size_t partial_at(int part, const AttentionArgs& A, size_t row, int head) {
  return (((size_t)part * A.n_q + row) * A.heads + head) * (HD + 4);
}

template <typename T, int HD, bool kTwice>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_packed_attention(AttentionArgs A, Group group, int slots, int parts,
                                                                                     float* __restrict__ partial) {
  typedef Rows<T, HD> R;
  typedef typename R::Frag Frag;
  __shared__ __align__(16) char s_kv[2][2][kKeys * R::kBytes];
  static_assert(2 * kKeys == kQueries, "a tile's place holds the workgroup's rows");
  Walk walk;
  if (!find_walk<true>(slots, parts, A.kv_heads, &walk)) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = walk.kvh, part = walk.part;
  Place at;
  // a sequence's last queries, which have the most keys, first
  if (!find_tile<kQueries>(queries_of(A), keys_of(A), A.n_seqs, group.each, slots - 1 - walk.slot, lane, &at)) return;
  const Sequence sq = at.mine, sk = at.other;
  const int t0 = at.row;

  const int behind = sk.len - sq.len, n_rows = sq.len * group.each;  // causal: token i attends keys 0 .. i + behind
  const int w_first = t0 + 32 * wave, r = min(w_first + a, n_rows - 1);
  const int token = group.tokens(r), head = kvh * group.each + r - token * group.each;
  const size_t row = (size_t)sq.start + token;
  auto keys_to = [&](int i) { return A.causal ? max(0, min(sk.len, i + behind + 1)) : sk.len; };
  const int mine = keys_to(token);  // of this lane's query
  // of the wave's; a wave behind the last row has nothing to do
  const int w_least = keys_to(group.tokens(min(w_first, n_rows - 1)));
  const int w_most = w_first < n_rows ? keys_to(group.tokens(min(w_first + 31, n_rows - 1))) : 0;
  const int all = (keys_to(group.tokens(min(t0 + kQueries, n_rows) - 1)) + kKeys - 1) / kKeys;
  const int first = part_from(all, part, parts), tiles = part_from(all, part + 1, parts) - first;

  const uint32_t k_stride = (uint32_t)(A.k_stride * sizeof(T)), v_stride = (uint32_t)(A.v_stride * sizeof(T));
  const char* kb = (const char*)((const T*)A.k + (size_t)sk.start * A.k_stride + (size_t)kvh * HD);
  const char* vb = (const char*)((const T*)A.v + (size_t)sk.start * A.v_stride + (size_t)kvh * HD);
  auto load = [&](auto buf, int it) {
    const int k0 = (first + it) * kKeys, last = sk.len - 1 - k0;
    R::template load<kKeys, kWaves>(s_kv[buf][0], kb + (size_t)k0 * k_stride, k_stride, last, wave, lane);
    R::template load<kKeys, kWaves>(s_kv[buf][1], vb + (size_t)k0 * v_stride, v_stride, last, wave, lane);
  };
  first_tile(tiles, load);
  // the rows by way of the second tile's place
  char* place = s_kv[1][0] + 32 * wave * R::kBytes;
  const size_t heads = (size_t)kvh * group.each * HD;
  const WaveRows<T, HD> my(min(w_first, n_rows - 1), n_rows, group);
  Frag qf[HD / 16];
  my.load(place, (const T*)A.q + (size_t)sq.start * A.q_stride + heads, A.q_stride, lane);
  dma_wait();
#pragma unroll
  for (int c = 0; c < HD / 16; ++c) qf[c] = my.operand(place, lane, c);
  RowReader<T, HD> rows(lane);
  ColReader<T, HD> cols(lane);

  f32x16 o[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(o[d]);
  const float c2 = A.scale * kLog2e;  // scores are kept in units of log 2
  float m_run = -3.4e38f, l_run = 0.f;
  through_tiles(tiles, load, [&](auto buf, int it) {
    const int k0 = (first + it) * kKeys;
    if (k0 >= w_most) return;  // (the same for the whole wave)
    rows.renew();
    cols.renew();
    constexpr int B = kKeys / 32, C = HD / 16, D = HD / 32;
    // blocks of 32 keys at a time: fp32's long products are left out where no row of the wave has keys
    constexpr int kAt = sizeof(T) == 2 ? B : 1;
    const bool all_blocks = k0 + 32 * (B - 1) < w_most;
    static_assert(B == 2, "one block or both");
    f32x16 s[B];
#pragma unroll
    for (int b = 0; b < B; ++b) clear(s[b]);
    Frag fr[2][2], fc[2][D];
    auto read_row = [&](auto g, Frag(&f)[2]) {
#pragma unroll
      for (int k = 0; k < 2; ++k) f[k] = rows(s_kv[buf][0], 32 * (2 * g / C), (2 * g + k) % C);
    };
    auto read_col = [&](auto g, Frag(&f)[D]) {
#pragma unroll
      for (int d = 0; d < D; ++d) f[d] = cols(s_kv[buf][1], 16 * g, d);
    };
    auto scores = [&](auto b) {
      read_row(std::integral_constant<int, b * C / 2>(), fr[0]);
      groups<kAt * C / 2, 2>(
          fr, [&](auto g, Frag(&f)[2]) { read_row(std::integral_constant<int, g + b * C / 2>(), f); },
          [&](auto g, Frag(&f)[2]) {
#pragma unroll
            for (int k = 0; k < 2; ++k) mma(f[k], qf[(2 * g + k) % C], s[b + 2 * g / C]);
          });
    };
    scores(std::integral_constant<int, 0>());
    if constexpr (kAt < B) {
      if (all_blocks) scores(std::integral_constant<int, 1>());
    }
    read_col(std::integral_constant<int, 0>(), fc[0]);
    if (k0 + kKeys > w_least) {
      int limit = mine;
      asm volatile("" : "+v"(limit));  // (a branch, and not a comparison per score in every tile)
#pragma unroll
      for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 32 * b + 16 * (e >> 3) + 8 * half + (e & 7) >= limit) s[b][e] = -INFINITY;
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
    // bf16 probabilities: each is off by at most 2^-8 of itself, as far as the output's own rounding moves it, and the
    // errors of many keys largely cancel; their sum is that of the unrounded ones
    Frag p[2 * B], rest[2 * B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], c2, -m_run));
        l_run += s[b][e];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        operand_of(s[b], i, p[2 * b + i]);
        if constexpr (kTwice) rest_of(s[b], i, p[2 * b + i], rest[2 * b + i]);
      }
    }
    auto values = [&](auto b) {
      groups<2 * kAt, D>(
          fc, [&](auto g, Frag(&f)[D]) { read_col(std::integral_constant<int, g + 2 * b>(), f); },
          [&](auto g, Frag(&f)[D]) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
              mma(f[d], p[g + 2 * b], o[d]);
              if constexpr (kTwice) mma(f[d], rest[g + 2 * b], o[d]);
            }
          });
    };
    values(std::integral_constant<int, 0>());
    if constexpr (kAt < B) {
      if (all_blocks) {
        read_col(std::integral_constant<int, 2>(), fc[0]);
        values(std::integral_constant<int, 1>());
      }
    }
  });
  const float l = l_run + __shfl_xor(l_run, 32, 64);
  if (parts > 1) {
    if (w_first + a >= n_rows) return;
    float* p = partial + partial_at<HD>(part, A, row, head);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) store8(p + 32 * d + 16 * i + 8 * half, o[d], i, 1.f);
    if (half == 0) *reinterpret_cast<float2*>(p + HD) = make_float2(m_run, l);
    return;
  }
  // a query without keys: nothing, and the logarithm of nothing
  const float by = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  lds_barrier();  // nobody reads tiles any more
  if (w_first >= n_rows) return;
  my.store(place, o, by, (T*)A.out + (size_t)sq.start * A.out_stride + heads, A.out_stride, lane);
  if (half == 0 && w_first + a < n_rows) A.lse[(size_t)head * A.n_q + row] = l == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l)) * kLn2;
}

// The parts of the rows of a tile, in order: a thread takes four values of a row.  Bound by its trips to memory: the place, then
// eight parts at a time (72B's one token 4.4 to 5.1 us).
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_attention_merge(AttentionArgs A, int slots, int parts, const float* __restrict__ partial) {
  const int each = A.heads / A.kv_heads, kvh = (int)blockIdx.x / slots;
  Place at;
  if (!find_tile<kQueries>(queries_of(A), keys_of(A), A.n_seqs, each, (int)blockIdx.x % slots, threadIdx.x & 63, &at)) return;
  const Sequence sq = at.mine;
  constexpr int kLanes = HD / 4;
  const int r = at.row + (int)blockIdx.y * (256 / kLanes) + threadIdx.x / kLanes, c = 4 * (threadIdx.x % kLanes);
  if (r >= sq.len * each) return;
  const size_t row = (size_t)sq.start + r / each;
  const int head = kvh * each + r % each;
  // eight parts' loads at a time, all of them on the way together
  float m = -3.4e38f, l = 0.f, o[4] = {};
  for (int k0 = 0; k0 < parts; k0 += 8) {
    float2 ml[8];
    float4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* p = partial + partial_at<HD>(min(k0 + k, parts - 1), A, row, head);
      ml[k] = *reinterpret_cast<const float2*>(p + HD);
      x[k] = *reinterpret_cast<const float4*>(p + c);
    }
    float most = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = fmaxf(most, ml[k].x);
    const float old = __builtin_amdgcn_exp2f(m - most);
    m = most;
    l *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= old;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float by = k0 + k < parts ? __builtin_amdgcn_exp2f(ml[k].x - m) : 0.f;
      l = fmaf(ml[k].y, by, l);
      o[0] = fmaf(x[k].x, by, o[0]), o[1] = fmaf(x[k].y, by, o[1]), o[2] = fmaf(x[k].z, by, o[2]), o[3] = fmaf(x[k].w, by, o[3]);
    }
  }
  const float by = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= by;
  T* op = (T*)A.out + row * A.out_stride + (size_t)head * HD + c;
  if constexpr (sizeof(T) == 2) {
    const uint2 u = make_uint2((uint32_t)round_bf16(o[0]) | (uint32_t)round_bf16(o[1]) << 16,
                               (uint32_t)round_bf16(o[2]) | (uint32_t)round_bf16(o[3]) << 16);
    *reinterpret_cast<uint2*>(op) = u;
  } else {
    *reinterpret_cast<float4*>(op) = make_float4(o[0], o[1], o[2], o[3]);
  }
  if (c == 0) A.lse[(size_t)head * A.n_q + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

uint64_t part_bytes(const AttentionArgs& a) { return 4ull * a.n_q * a.heads * (a.head_dim + 4); }
template <typename T>
int key_parts(const AttentionArgs& a) {
  const int64_t walks = (int64_t)tile_slots(a.n_q, a.heads / a.kv_heads, a.n_seqs, kQueries) * a.kv_heads;
  return walk_parts(walks, (double)a.n_k / a.n_seqs / kKeys, a.causal && a.n_q == a.n_k,
                    walk_cost<T>(1.0, 1.6, 4, a.head_dim), part_bytes(a));
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const AttentionArgs& a, float* partial) {
  const int slots = tile_slots(a.n_q, a.heads / a.kv_heads, a.n_seqs, kQueries), parts = key_parts<T>(a);
  auto run = [&](auto kernel) {
    kernel<<<walk_grid<true>(slots, parts, a.kv_heads), 64 * kWaves, 0, s>>>(a, group_of(a), slots, parts, partial);
  };
  if (sizeof(T) == 2 && few_pairs(a))
    run(k_packed_attention<T, HD, sizeof(T) == 2>);
  else
    run(k_packed_attention<T, HD, false>);
  if (parts > 1) k_attention_merge<T, HD><<<dim3(slots * a.kv_heads, kQueries * HD / 1024), 256, 0, s>>>(a, slots, parts, partial);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_of(hipStream_t s, const AttentionArgs& a, float* partial) {
  return a.head_dim == 32   ? launch<T, 32>(s, a, partial)
         : a.head_dim == 64 ? launch<T, 64>(s, a, partial)
                            : launch<T, 128>(s, a, partial);
}

}  // namespace

size_t packed_attention_workspace(const AttentionArgs& a) { return parts_room(part_bytes(a)); }

hipError_t launch_packed_attention(hipStream_t s, int dtype, const AttentionArgs& a, void* ws) {
  return dtype == ROLLOUT_DTYPE_BF16 ? launch_of<uint16_t>(s, a, (float*)ws) : launch_of<float>(s, a, (float*)ws);
}

}  // namespace rollout
