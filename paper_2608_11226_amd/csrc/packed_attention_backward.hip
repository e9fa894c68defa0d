// The gradient of packed attention.
//
//   p_ij = e^(s_ij - lse_i),  D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i)
//   dv_j = sum_i p_ij do_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
//
// (sums over the queries of all heads that share a key's head).  Probabilities are formed again from the scores.  Two kernels
// do so, one for the keys' gradients and one for the queries': seven products of the size of q k^T where one that adds up
// queries' gradients atomically has five, but every sum has an order of its own that does not depend on scheduling.
//
// Bound by the matrix products and what feeds them: 8,192 tokens at 40 on 8 heads of 128 take 900 us for the queries and 1,286 for
// the keys (products are at work in 0.70 and 0.65 of the compute units' cycles) and 56 to join the keys' parts; the 7B update's 16
// sequences 87, 134 and 17 (0.32 and 0.38: short walks, and the longest ones end alone); fp32 at the 7B heads 1,015, 1,455 and 39.
// Did not pay: the scores' exponentials issued beside the other product (7B 230 us, so 244), workgroups of eight waves that share
// out a tile's rows and add up in LDS instead of half of the parts (7B 222, so 241; 14B 2,120, so 2,125), and as many parts as a
// walk's own length asks for (some dies then wait for the others).
//
// Probabilities and ds enter the second products as bf16 where the inputs are bf16: each is off by at most 2^-8 of itself, as
// far as the result's own rounding moves it.
#include "packed_attention.h"

namespace rollout {
namespace {

constexpr int kWaves = 4;

// Queries' gradients.  A workgroup takes 128 rows, a row being a token's query of one of the heads that share a key's, a wave 32 of
// them, whose q and do stay in registers, and walks over tiles of 64 keys.  Scores have keys as rows and queries as columns, as
// in the forward pass, and where there are few rows the keys are dealt out to several workgroups as there.  It leaves
// -lse / scale and -D of every row behind ([n_q][heads]), which the keys' gradients need.
constexpr int kDqRows = 32 * kWaves, kDqKeys = 64;

template <typename T, int HD, bool kTwice>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_attention_dq(AttentionGradArgs A, Group group, int slots, int parts,
                                                                                 float2* __restrict__ stats,
                                                                                 float* __restrict__ partial) {
  typedef Rows<T, HD> R;
  typedef typename R::Frag Frag;
  __shared__ __align__(16) char s_kv[2][2][kDqKeys * R::kBytes];
  static_assert(2 * kDqKeys == kDqRows, "a tile's place holds the workgroup's rows");
  Walk walk;
  if (!find_walk<true>(slots, parts, A.kv_heads, &walk)) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = walk.kvh, part = walk.part;
  Place at;
  if (!find_tile<kDqRows>(queries_of(A), keys_of(A), A.n_seqs, group.each, slots - 1 - walk.slot, lane, &at)) return;
  const Sequence sq = at.mine, sk = at.other;
  const int t0 = at.row;
  const int behind = sk.len - sq.len, n_rows = sq.len * group.each;
  const int w_first = t0 + 32 * wave, r = min(w_first + a, n_rows - 1);
  const int token = group.tokens(r), head = kvh * group.each + r - token * group.each;
  const size_t row = (size_t)sq.start + token;
  auto keys_to = [&](int i) { return A.causal ? max(0, min(sk.len, i + behind + 1)) : sk.len; };
  const int mine = keys_to(token);
  // a wave behind the last row has nothing to do
  const int w_least = keys_to(group.tokens(min(w_first, n_rows - 1)));
  const int w_most = w_first < n_rows ? keys_to(group.tokens(min(w_first + 31, n_rows - 1))) : 0;
  const int all = (keys_to(group.tokens(min(t0 + kDqRows, n_rows) - 1)) + kDqKeys - 1) / kDqKeys;
  const int first = part_from(all, part, parts), tiles = part_from(all, part + 1, parts) - first;

  const uint32_t k_stride = (uint32_t)(A.k_stride * sizeof(T)), v_stride = (uint32_t)(A.v_stride * sizeof(T));
  const char* kb = (const char*)((const T*)A.k + (size_t)sk.start * A.k_stride + (size_t)kvh * HD);
  const char* vb = (const char*)((const T*)A.v + (size_t)sk.start * A.v_stride + (size_t)kvh * HD);
  auto load = [&](auto buf, int it) {
    const int k0 = (first + it) * kDqKeys, last = sk.len - 1 - k0;
    R::template load<kDqKeys, kWaves>(s_kv[buf][0], kb + (size_t)k0 * k_stride, k_stride, last, wave, lane);
    R::template load<kDqKeys, kWaves>(s_kv[buf][1], vb + (size_t)k0 * v_stride, v_stride, last, wave, lane);
  };
  // the rows by way of LDS: q and do at once, out with the first tile
  char *place = s_kv[1][0] + 32 * wave * R::kBytes, *other = s_kv[0][0] + 32 * wave * R::kBytes;
  const size_t heads = (size_t)kvh * group.each * HD;
  const WaveRows<T, HD> mine_of(min(w_first, n_rows - 1), n_rows, group);
  mine_of.load(place, (const T*)A.q + (size_t)sq.start * A.q_stride + heads, A.q_stride, lane);
  mine_of.load(other, (const T*)A.dout + (size_t)sq.start * A.dout_stride + heads, A.dout_stride, lane);
  const float lse = A.lse[(size_t)head * A.n_q + row];
  dma_wait();
  Frag qf[HD / 16], df[HD / 16];
#pragma unroll
  for (int c = 0; c < HD / 16; ++c) qf[c] = mine_of.operand(place, lane, c), df[c] = mine_of.operand(other, lane, c);
  lds_barrier();
  mine_of.load(place, (const T*)A.out + (size_t)sq.start * A.out_stride + heads, A.out_stride, lane);
  first_tile(tiles, load);
  float2 my = make_float2(0.f, 0.f);  // lse in units of log 2, and D
  dma_wait();
#pragma unroll
  for (int c = 0; c < HD / 16; ++c) {
    const Frag o = mine_of.operand(place, lane, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) my.y = fmaf((float)o[e], (float)df[c][e], my.y);
  }
  my.y += __shfl_xor(my.y, 32, 64);
  // a query without keys: no probabilities
  my.x = lse == -INFINITY ? INFINITY : lse * kLog2e;
  if (part == 0 && half == 0 && w_first + a < n_rows) stats[row * A.heads + head] = make_float2(lse == -INFINITY ? lse : -lse / A.scale, -my.y);
  RowReader<T, HD> rows(lane);
  ColReader<T, HD> cols(lane);

  f32x16 dq[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(dq[d]);
  const float c2 = A.scale * kLog2e;
  through_tiles(tiles, load, [&](auto buf, int it) {
    constexpr int C = HD / 16, D = HD / 32, kUnroll = sizeof(T) == 2 ? kDqKeys / 32 : 1;  // (fp32: registers)
#pragma unroll kUnroll
    for (int b = 0; b < kDqKeys / 32; ++b) {
      const int k0 = (first + it) * kDqKeys + 32 * b;
      if (k0 >= w_most) return;  // (the same for the whole wave)
      rows.renew();
      cols.renew();
      f32x16 s, dp;
      clear(s);
      clear(dp);
      Frag fr[2][2], fc[2][D];
      auto read_row = [&](auto g, Frag(&f)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k) f[k] = rows(2 * g < C ? s_kv[buf][0] : s_kv[buf][1], 32 * b, (2 * g + k) % C);
      };
      auto read_col = [&](auto g, Frag(&f)[D]) {
#pragma unroll
        for (int d = 0; d < D; ++d) f[d] = cols(s_kv[buf][0], 32 * b + 16 * g, d);
      };
      read_row(std::integral_constant<int, 0>(), fr[0]);
      groups<C, 2>(fr, read_row, [&](auto g, Frag(&f)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if constexpr (2 * g < C)
            mma(f[k], qf[(2 * g + k) % C], s);
          else
            mma(f[k], df[(2 * g + k) % C], dp);
        }
      });
      read_col(std::integral_constant<int, 0>(), fc[0]);
      if (k0 + 32 > w_least) {
        int limit = mine;
        asm volatile("" : "+v"(limit));  // (a branch, and not a comparison per score in every tile)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 16 * (e >> 3) + 8 * half + (e & 7) >= limit) s[e] = -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c2, -my.x)) * (dp[e] - my.y);
      Frag ds[2], rest[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        operand_of(dp, i, ds[i]);
        if constexpr (kTwice) rest_of(dp, i, ds[i], rest[i]);
      }
      groups<2, D>(fc, read_col, [&](auto g, Frag(&f)[D]) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
          mma(f[d], ds[g], dq[d]);
          if constexpr (kTwice) mma(f[d], rest[g], dq[d]);
        }
      });
    }
  });
  if (parts > 1) {
    if (w_first + a >= n_rows) return;
    float* out = partial + (((size_t)part * A.n_q + row) * A.heads + head) * HD + 8 * half;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) store8(out + 32 * d + 16 * i, dq[d], i, A.scale);
    return;
  }
  lds_barrier();  // nobody reads tiles any more
  if (w_first >= n_rows) return;
  mine_of.store(place, dq, A.scale, (T*)A.dq + (size_t)sq.start * A.dq_stride + heads, A.dq_stride, lane);
}

// Keys' gradients.  A workgroup takes 128 keys, a wave 32 of them, whose k and v stay in registers, and walks over tiles of 32
// rows.  Scores have queries as rows and keys as columns, so that a lane holds one key's.
constexpr int kBackKeys = 32 * kWaves, kBackRows = 32;

template <typename T, int HD, bool kTwice>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 2 ? 2 : 1) void k_attention_dkv(AttentionGradArgs A, Group group, int slots, int parts,
                                                                                  const float2* __restrict__ stats,
                                                                                  float* __restrict__ partial) {
  typedef Rows<T, HD> R;
  typedef typename R::Frag Frag;
  __shared__ __align__(16) char s_q[2][kBackRows * R::kBytes];
  __shared__ __align__(16) char s_do[2][kBackRows * R::kBytes];
  __shared__ __align__(16) float s_stat[2][2][kBackRows];
  // 128 dimensions: registers for all of k and v are some 20 too many, and what the compiler then keeps in scratch memory waits for
  // the tiles on their way: six of v's eight operands lie in LDS, in fp32, with one workgroup in a compute unit, all of them, and all
  // where products are doubled (with 64 bytes of a lane in scratch memory all the same: calls that are a launch)
  constexpr int C = HD / 16, D = HD / 32, kKept = HD < 128 ? C : sizeof(T) == 2 && !kTwice ? 2 : 0;
  __shared__ __align__(16) Frag s_v[kKept < C ? kWaves : 1][kKept < C ? C - kKept : 1][64];
  Walk walk;
  if (!find_walk<false>(slots, parts, A.kv_heads, &walk)) return;
  const int lane = threadIdx.x & 63, a = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int each = group.each, kvh = walk.kvh, part = walk.part;
  Place at;
  if (!find_tile<kBackKeys>(keys_of(A), queries_of(A), A.n_seqs, 1, walk.slot, lane, &at)) return;
  const Sequence sk = at.mine, sq = at.other;
  const int t0 = at.row;
  const int behind = sk.len - sq.len, n_rows = sq.len * each;

  const int w_first = t0 + 32 * wave, kj = w_first + a;
  const size_t row = (size_t)sk.start + min(kj, sk.len - 1);
  // causal: key j is attended from token j - behind on
  auto from = [&](int j) { return A.causal ? max(0, min(j - behind, sq.len)) * each : 0; };
  const int head_tile = from(t0) / kBackRows, all = (n_rows + kBackRows - 1) / kBackRows - head_tile;
  const int first = head_tile + part_from(all, part, parts), tiles = head_tile + part_from(all, part + 1, parts) - first;
  const int mine = from(kj);
  // a wave behind the last key has nothing to do
  const int w_least = w_first < sk.len ? from(w_first) : INT32_MAX, w_most = from(w_first + 31);

  const uint32_t q_stride = (uint32_t)(A.q_stride * sizeof(T)), do_stride = (uint32_t)(A.dout_stride * sizeof(T));
  const size_t head = (size_t)kvh * each;
  const char* qb = (const char*)((const T*)A.q + (size_t)sq.start * A.q_stride + head * HD);
  const char* dob = (const char*)((const T*)A.dout + (size_t)sq.start * A.dout_stride + head * HD);
  const float2* sb = stats + (size_t)sq.start * A.heads + head;
  int token = group.tokens(first * kBackRows), over = first * kBackRows - token * each;  // of the first row that is loaded next
  const int more = group.tokens(kBackRows), more_over = kBackRows - more * each;
  auto load = [&](auto buf, int it) {
    const int last = n_rows - 1 - (first + it) * kBackRows;
    const char* q0 = qb + (size_t)token * q_stride;
    const char* do0 = dob + (size_t)token * do_stride;
    if (wave == 0) {
      const uint32_t x = (uint32_t)(min(a, last) + over), t = (uint32_t)group.tokens((int)x);
      dma_lds4_at(sb + (size_t)token * A.heads, (t * (uint32_t)(A.heads - each) + x) * 8 + 4 * half, s_stat[buf]);
    }
    R::template load_with<kBackRows, kWaves>(wave, lane, [&](int row, uint32_t offset, int place) {
      const uint32_t x = (uint32_t)(min(row, last) + over), t = (uint32_t)group.tokens((int)x);
      const uint32_t at = (x - t * (uint32_t)each) * R::kBytes + offset;
      dma_lds16_at(q0, t * q_stride + at, s_q[buf] + place);
      dma_lds16_at(do0, t * do_stride + at, s_do[buf] + place);
    });
    token += more, over += more_over;
    if (over >= each) over -= each, ++token;
  };
  first_tile(tiles, load);
  Frag kf[C], vf[kKept ? kKept : 1];
  {
    const T* kp = (const T*)A.k + row * A.k_stride + (size_t)kvh * HD + 8 * half;
    const T* vp = (const T*)A.v + row * A.v_stride + (size_t)kvh * HD + 8 * half;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      kf[c] = load_operand(kp + 16 * c);
      if (c < kKept)
        vf[c < kKept ? c : 0] = load_operand(vp + 16 * c);
      else
        s_v[wave][c - kKept][lane] = load_operand(vp + 16 * c);
    }
  }
  RowReader<T, HD> rows(lane);
  ColReader<T, HD> cols(lane);
  // here: no wait for them among the tiles
#pragma unroll
  for (int c = 0; c < C; ++c) asm volatile("" : "+v"(kf[c]));
#pragma unroll
  for (int c = 0; c < kKept; ++c) asm volatile("" : "+v"(vf[c]));

  f32x16 dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) clear(dk[d]), clear(dv[d]);
  const float c2 = A.scale * kLog2e;
  through_tiles(tiles, load, [&](auto buf, int it) {
    const int i0 = (first + it) * kBackRows;
    if (i0 + kBackRows <= w_least) return;  // (the same for the whole wave)
    rows.renew();
    cols.renew();
    // bf16: the sums start from -lse / scale and -D, which costs their last bits and no register
    constexpr bool kStart = sizeof(T) == 2;
    f32x16 s, dp;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = kStart ? s_stat[buf][0][16 * (e >> 3) + 8 * half + (e & 7)] : 0.f;
      dp[e] = kStart ? s_stat[buf][1][16 * (e >> 3) + 8 * half + (e & 7)] : 0.f;
    }
    Frag fr[2][4], fc[2][D];
    auto read_row = [&](auto g, Frag(&f)[4]) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = (2 * g + k) % C;
        f[k] = rows(2 * g < C ? s_q[buf] : s_do[buf], 0, c);
        if (2 * g >= C && c >= kKept) f[2 + k] = s_v[wave][c - kKept][lane];
      }
    };
    auto read_col = [&](auto g, Frag(&f)[D]) {
#pragma unroll
      for (int d = 0; d < D; ++d) f[d] = cols(g % 2 ? s_q[buf] : s_do[buf], 16 * (g / 2), d);
    };
    read_row(std::integral_constant<int, 0>(), fr[0]);
    groups<C, 4>(fr, read_row, [&](auto g, Frag(&f)[4]) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = (2 * g + k) % C;
        if constexpr (2 * g < C)
          mma(f[k], kf[c], s);
        else
          mma(f[k], c < kKept ? vf[c < kKept ? c : 0] : f[2 + k], dp);
      }
    });
    read_col(std::integral_constant<int, 0>(), fc[0]);
    if (i0 < w_most || i0 + kBackRows > n_rows) {
      int limit = mine;
      asm volatile("" : "+v"(limit));  // (a branch, and not a comparison per score in every tile)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = i0 + 16 * (e >> 3) + 8 * half + (e & 7);
        if (i < limit || i >= n_rows) s[e] = -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int i = 16 * (e >> 3) + 8 * half + (e & 7);
      s[e] = __builtin_amdgcn_exp2f((kStart ? s[e] : s[e] + s_stat[buf][0][i]) * c2);
      dp[e] = s[e] * (kStart ? dp[e] : dp[e] + s_stat[buf][1][i]);
    }
    Frag p[2], ds[2], p_rest[2], ds_rest[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      operand_of(s, i, p[i]), operand_of(dp, i, ds[i]);
      if constexpr (kTwice) rest_of(s, i, p[i], p_rest[i]), rest_of(dp, i, ds[i], ds_rest[i]);
    }
    groups<4, D>(fc, read_col, [&](auto g, Frag(&f)[D]) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        if constexpr (g % 2) {
          mma(f[d], ds[g / 2], dk[d]);
          if constexpr (kTwice) mma(f[d], ds_rest[g / 2], dk[d]);
        } else {
          mma(f[d], p[g / 2], dv[d]);
          if constexpr (kTwice) mma(f[d], p_rest[g / 2], dv[d]);
        }
      }
    });
  });
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

// Eight neighbours of the parts' sums, in order, to an output; eight parts' are on the way together.
template <typename T>
__device__ __forceinline__ void join8(T* out, const float* p, size_t apart, int parts) {
  float t[8] = {};
  for (int k0 = 0; k0 < parts; k0 += 8) {
    float x[8][8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k0 + k < parts) ld8(p + (k0 + k) * apart, 0, x[k]);  // (the same for the whole wave)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k0 + k < parts)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += x[k][e];
  }
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x4*>(out) = pack16(t);
  else
    st8(out, 0, t);
}

// The parts' sums of a tile of keys.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join_dkv(AttentionGradArgs A, int parts, const float* __restrict__ partial) {
  Place at;
  if (!find_tile<kBackKeys>(keys_of(A), queries_of(A), A.n_seqs, 1, (int)blockIdx.x, threadIdx.x & 63, &at)) return;
  const Sequence sk = at.mine;
  const int t0 = at.row;
  const int width = A.kv_heads * A.head_dim, chunks = width / 8, rows = min(kBackKeys, sk.len - t0);
  const size_t all = (size_t)A.n_k * width;
  const bool v = blockIdx.y & 1;
  T* out = (T*)(v ? A.dv : A.dk);
  const int64_t stride = v ? A.dv_stride : A.dk_stride;
  for (int i = (int)(blockIdx.y >> 1) * 256 + threadIdx.x; i < rows * chunks; i += (int)(gridDim.y >> 1) * 256) {
    const size_t row = (size_t)sk.start + t0 + i / chunks;
    const int c = i % chunks * 8;
    join8(out + row * stride + c, partial + (v ? all : 0) + row * width + c, 2 * all, parts);
  }
}

// The parts' sums of a tile of 128 tokens.
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join_dq(AttentionGradArgs A, int parts, const float* __restrict__ partial) {
  Place at;
  if (!find_tile<128>(queries_of(A), keys_of(A), A.n_seqs, 1, (int)blockIdx.x, threadIdx.x & 63, &at)) return;
  const Sequence sq = at.mine;
  const int t0 = at.row;
  const int width = A.heads * A.head_dim, chunks = width / 8, rows = min(128, sq.len - t0);
  for (int i = (int)blockIdx.y * 256 + threadIdx.x; i < rows * chunks; i += (int)gridDim.y * 256) {
    const size_t row = (size_t)sq.start + t0 + i / chunks;
    const int c = i % chunks * 8;
    join8((T*)A.dq + row * A.dq_stride + c, partial + row * width + c, (size_t)A.n_q * width, parts);
  }
}

uint64_t dkv_part_bytes(const AttentionArgs& a) { return 8ull * a.n_k * a.kv_heads * a.head_dim; }
uint64_t dq_part_bytes(const AttentionArgs& a) { return 4ull * a.n_q * a.heads * a.head_dim; }
template <typename T>
int row_parts(const AttentionArgs& a) {
  const int64_t walks = (int64_t)tile_slots(a.n_k, 1, a.n_seqs, kBackKeys) * a.kv_heads;
  return walk_parts(walks, (double)a.n_q * (a.heads / a.kv_heads) / a.n_seqs / kBackRows, a.causal && a.n_q == a.n_k,
                    walk_cost<T>(1.3, 2.0, 4, a.head_dim), dkv_part_bytes(a));
}
template <typename T>
int key_parts(const AttentionArgs& a) {
  const int64_t walks = (int64_t)tile_slots(a.n_q, a.heads / a.kv_heads, a.n_seqs, kDqRows) * a.kv_heads;
  return walk_parts(walks, (double)a.n_k / a.n_seqs / kDqKeys, a.causal && a.n_q == a.n_k,
                    walk_cost<T>(2.0, 2.8, 6, a.head_dim), dq_part_bytes(a));
}

// workgroups for a tile's 128 rows of `width` values: a thread takes one chunk of eight, or several where there are many tiles
int join_groups(int slots, int width) { return std::max(1, std::min(width / 16, std::max(8, 4096 / slots))); }

size_t stats_bytes(const AttentionArgs& a) { return ((size_t)a.n_q * a.heads * 8 + 15) / 16 * 16; }

template <typename T, int HD, bool kTwice>
hipError_t launch(hipStream_t s, const AttentionGradArgs& a, char* ws) {
  float2* stats = (float2*)ws;
  float* partial = (float*)(ws + stats_bytes(a));  // of the queries, then of the keys
  const int q_slots = tile_slots(a.n_q, a.heads / a.kv_heads, a.n_seqs, kDqRows), kp = key_parts<T>(a);
  const int join_slots = tile_slots(a.n_q, 1, a.n_seqs, 128);
  k_attention_dq<T, HD, kTwice><<<walk_grid<true>(q_slots, kp, a.kv_heads), 64 * kWaves, 0, s>>>(a, group_of(a), q_slots, kp, stats, partial);
  if (kp > 1) k_attention_join_dq<T><<<dim3(join_slots, join_groups(join_slots, a.heads * HD)), 256, 0, s>>>(a, kp, partial);
  const int slots = tile_slots(a.n_k, 1, a.n_seqs, kBackKeys);
  const int rp = row_parts<T>(a);
  k_attention_dkv<T, HD, kTwice><<<walk_grid<false>(slots, rp, a.kv_heads), 64 * kWaves, 0, s>>>(a, group_of(a), slots, rp, stats, partial);
  if (rp > 1) k_attention_join_dkv<T><<<dim3(slots, 2 * join_groups(slots, a.kv_heads * HD)), 256, 0, s>>>(a, rp, partial);
  return hipGetLastError();
}

template <typename T, bool kTwice>
hipError_t launch_of(hipStream_t s, const AttentionGradArgs& a, char* ws) {
  return a.head_dim == 32   ? launch<T, 32, kTwice>(s, a, ws)
         : a.head_dim == 64 ? launch<T, 64, kTwice>(s, a, ws)
                            : launch<T, 128, kTwice>(s, a, ws);
}

}  // namespace

size_t packed_attention_backward_workspace(const AttentionArgs& a) {
  return stats_bytes(a) + std::max(parts_room(dkv_part_bytes(a)), parts_room(dq_part_bytes(a)));
}

hipError_t launch_packed_attention_backward(hipStream_t s, int dtype, const AttentionGradArgs& a, void* ws) {
  if (dtype == ROLLOUT_DTYPE_FP32) return launch_of<float, false>(s, a, (char*)ws);
  return few_pairs(a) ? launch_of<uint16_t, true>(s, a, (char*)ws) : launch_of<uint16_t, false>(s, a, (char*)ws);
}

}  // namespace rollout
