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
//
// Both directions are bound by HBM: 4,096 rows of 152,064 bf16 logits (an eighth of them padding) are read at 6.2 TB/s (177
// us), with the vector ALU busy four fifths of that time (nine instructions an element, the exponential among them), and
// their gradient is read and written at 5.9 TB/s (375 us).  A large copy reaches 4.75 TB/s on this card, a fill 6.9.
#include "update.h"

#include <type_traits>

namespace rollout {
namespace {

constexpr int RB = 256;  // threads of a row's workgroup
constexpr int RW = RB / 64;
constexpr int kUnits = 4;  // 16-byte loads in flight a lane
constexpr int kMaxUnits = kMaxTopVocab / 256, kMaxPer = kMaxUnits / 64;  // of a row, of a lane, where alternatives are taken
constexpr int kMaxChunks = 64;     // a lane each when parts are joined
// Workgroups that a launch of few rows is split into: 515 bf16 rows of 152,064 38.5 us with 1,024, 32.7 with 2,048, 34.4 with
// 8,192; 256 fp32 rows with 20 alternatives 37.0, 36.4 and 36.6.
constexpr int kWorkgroups = 2048;
constexpr int kWhole = 64;         // units of a row that is not split
constexpr int kWaveRows = 2048;    // rows from which such a row is one wave's
constexpr int kMaxGrid = 1 << 20;
constexpr int kBatch = 4;          // 16-byte loads in flight a thread in the gradient
constexpr size_t kLastLevelBytes = 256u << 20;
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

// Lane i: the maximum over the wave of keys i % 4.  Neighbours first share out the four between them, so that the steps across
// the wave are those of one key (512 rows of 152,064 bf16 ids with 5 alternatives 37.4 us; each key by itself 38.7).
__device__ __forceinline__ uint32_t wave_max_of_four(const uint32_t (&key)[4]) {
  const int lane = threadIdx.x & 63;
  const auto dpp = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true);
  };
  constexpr std::integral_constant<int, 0xB1> next{};     // quad_perm: lane ^ 1
  constexpr std::integral_constant<int, 0x4E> second{};   // lane ^ 2
  constexpr std::integral_constant<int, 0x124> ror4{};    // a row's lanes turned by four, by eight
  constexpr std::integral_constant<int, 0x128> ror8{};
  const bool odd = lane & 1, upper = lane & 2;
  const uint32_t a = max(odd ? key[1] : key[0], dpp(odd ? key[0] : key[1], next));
  const uint32_t b = max(odd ? key[3] : key[2], dpp(odd ? key[2] : key[3], next));
  uint32_t c = max(upper ? b : a, dpp(upper ? a : b, second));
  c = max(c, dpp(c, ror4));
  c = max(c, dpp(c, ror8));
  const auto rows = __builtin_amdgcn_permlane16_swap(c, c, false, false);
  c = max((uint32_t)rows[0], (uint32_t)rows[1]);
  const auto halves = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  return max((uint32_t)halves[0], (uint32_t)halves[1]);
}

// Key of the k-th of the lanes' keys (1 <= k <= 64), in every lane: bit by bit the largest that k of them reach (64 rows of
// 152,064 fp32 ids with 8 alternatives 16.4 us; counting lane by lane how many stand before each, 17.9).
__device__ __forceinline__ uint32_t kth_key(uint32_t key, int k) {
  uint32_t bound = 0;
#pragma unroll
  for (int b = 31; b >= 0; --b) {
    const uint32_t more = bound | 1u << b;
    if (__popcll(__ballot(key >= more)) >= k) bound = more;
  }
  return bound;
}

// The row's top values by (value descending, id ascending), one by one, by one wave: where very many values are equal.
// keys: the keys of the maxima of the row's units (64 x N consecutive ids).  The top values lie in the top units by
// (maximum, position): a unit that is not among them has as many values before its own as there are alternatives.
// Every one of these units offers its best value not yet taken, and the best offer is taken, top times.
template <typename T>
__device__ void take_top_in_turn(const T* row, int V, int top, const uint32_t* keys, int nseg, float m, float temperature,
                                 float ln_s, int32_t* ids, float* logp) {
  constexpr int N = Chunk16<T>::N;
  const int lane = threadIdx.x & 63;
  const int n = min(top, nseg);
  uint32_t key = 0;  // lane j: key of the unit it holds, and the unit
  int unit = 0x7FFFFFFF;
  uint32_t bound = 0xFFFFFFFFu;  // the unit chosen last, and its key
  int after = -1;
  for (int r = 0; r < n; ++r) {
    uint32_t best = 0;
    int at = 0;
    for (int i = lane; i < nseg; i += 64) {
      const uint32_t k = keys[i];
      if (k > best && (k < bound || (k == bound && i > after))) best = k, at = i;
    }
    const uint32_t top_key = wave_max_u32(best);
    const uint32_t low = wave_max_u32(best == top_key ? 0x7FFFFFFFu - (uint32_t)at : 0u);
    bound = top_key, after = (int)(0x7FFFFFFFu - low);
    if (lane == r) key = top_key, unit = after;
  }
  // in the order of their ids, so that the first of equal offers is the lowest id
  int rank = 0;
  for (int r = 0; r < n; ++r) rank += __builtin_amdgcn_readlane(unit, r) < unit;
  key = (uint32_t)__builtin_amdgcn_ds_permute(4 * (lane < n ? rank : lane), (int)key);
  unit = __builtin_amdgcn_ds_permute(4 * (lane < n ? rank : lane), unit);
  int last = -1;  // lane j: id of the last of its unit's values that were taken and equal its offer
  for (int r = 0; r < top; ++r) {
    const uint32_t best = wave_max_u32(lane < n ? key : 0);
    const int j = __ffsll((unsigned long long)__ballot(lane < n && key == best)) - 1;
    const int u = __builtin_amdgcn_readlane(unit, j), taken = __builtin_amdgcn_readlane(last, j);
    const int id0 = (u * 64 + lane) * N;
    float v[N];
    unpack16(load_row(row, id0, V), v);
    int hit = 0x7FFFFFFF;
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
      if (key_of(v[i]) == best && id0 + i > taken && id0 + i < V) hit = id0 + i;
    const int who = __ffsll((unsigned long long)__ballot(hit != 0x7FFFFFFF)) - 1;
    const int id = __builtin_amdgcn_readlane(hit, who);
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
      logp[r] = (of_key(best) - m) / temperature - ln_s;
    }
  }
}

struct TopLds {
  uint32_t sample[RB];
  int units[kMaxUnits];
  uint2 found[RB];
  int count;
};

// The same by a workgroup, where no more than RB values stand at or above a bound that at least `top` values reach.  Such
// a bound is the top-th of 64 maxima of disjoint parts of the row: of the units' maxima, every 64th in a lane's part, or,
// in rows of fewer units than alternatives, of the threads' own values (128 rows of 32,003 bf16 ids, 63 units, with 5: 25.9
// us so, 19.1 by units).  Only units whose maximum reaches the bound are read.  The values found are ranked at once, every
// thread counting those before its own.  (Twice the threads: 256 bf16 rows with 32 32.6 instead of 35.2 us, but 300 rows of
// 1,024 ids 14.3 instead of 12.4.)
template <typename T>
__device__ void take_top(const T* row, int V, int top, const uint32_t* keys, int nseg, TopLds& lds, float m,
                         float temperature, float ln_s, int32_t* ids, float* logp, const uint32_t (&mine)[kMaxPer]) {
  constexpr int N = Chunk16<T>::N;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) lds.count = 0;
  uint32_t part = 0;
  int n = 0;  // units to read, the same in every wave
  if (nseg >= top) {
#pragma unroll
    for (int i = 0; i < kMaxPer; ++i) part = max(part, mine[i]);
    part = kth_key(part, top);
#pragma unroll
    for (int i = 0; i < kMaxPer; ++i) {
      const unsigned long long b = __ballot(mine[i] >= part);
      if (!b) continue;
      if (wave == 0 && mine[i] >= part) lds.units[n + __popcll(b & ((1ull << lane) - 1))] = i * 64 + lane;
      n += __popcll(b);
    }
  } else {
    for (int i = threadIdx.x * N; i < V; i += RB * N) {
      float v[N];
      unpack16(load_row(row, i, V), v);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (i + j < V) part = max(part, key_of(v[j]));
    }
    lds.sample[threadIdx.x] = part;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < RW; ++w) part = max(part, lds.sample[w * 64 + lane]);
    part = kth_key(part, top);
    n = nseg;
    if (wave == 0 && lane < nseg) lds.units[lane] = lane;
  }
  __syncthreads();
  const float least = part ? of_key(part) : -INFINITY;
  constexpr int kAhead = 8;
  for (int r0 = wave; r0 < n; r0 += RW * kAhead) {
    u32x4 raw[kAhead];
    int id0[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (r0 + j * RW < n) {
        id0[j] = (__builtin_amdgcn_readfirstlane(lds.units[r0 + j * RW]) * 64 + lane) * N;
        raw[j] = load_row(row, id0[j], V);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (r0 + j * RW >= n) break;
      float v[N];
      unpack16(raw[j], v);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (v[i] >= least && id0[j] + i < V) {
          const int at = atomicAdd(&lds.count, 1);
          if (at < RB) lds.found[at] = make_uint2(key_of(v[i]), (uint32_t)(id0[j] + i));
        }
      }
    }
  }
  __syncthreads();
  const int count = lds.count;
  if (count > RB) {
    if (wave == 0) take_top_in_turn(row, V, top, keys, nseg, m, temperature, ln_s, ids, logp);
  } else if (threadIdx.x < count) {
    const uint2 own = lds.found[threadIdx.x];
    int place = 0;
    for (int j0 = 0; j0 < count; j0 += 8) {
      uint2 q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = lds.found[j0 + j];  // RB is a multiple of 8
#pragma unroll
      for (int j = 0; j < 8; ++j)
        place += j0 + j < count && (q[j].x > own.x || (q[j].x == own.x && q[j].y < own.y));
    }
    if (place < top) {
      ids[place] = (int)own.y;
      logp[place] = (of_key(own.x) - m) / temperature - ln_s;
    }
  }
  __syncthreads();  // the next row's use of the LDS
}

// The token's logit (NaN: there is no such id, or no token is asked for).
template <typename T>
__device__ __forceinline__ float token_logit(const LogprobArgs& a, int row, int token) {
  return a.logp && token < a.vocab ? ldf((const T*)a.z + (int64_t)row * a.stride, (size_t)token) : NAN;
}
// What a row's maximum and sums come to (one lane); x: its token's logit.
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int row, float x, const Soft& r) {
  const bool bad = !(r.s == r.s);
  const float ln_s = logf(r.s);
  if (a.logp) a.logp[row] = bad ? NAN : x == -INFINITY ? -INFINITY : (x - r.m) / a.temperature - ln_s;
  if (a.entropy) a.entropy[row] = bad ? NAN : r.m == -INFINITY ? 0.f : ln_s - kLn2 * r.w / r.s;
  if (a.stats) {
    a.stats[2 * (size_t)row] = bad ? NAN : r.m;
    a.stats[2 * (size_t)row + 1] = bad ? NAN : ln_s;
  }
}
__device__ __forceinline__ void finish_padding(const LogprobArgs& a, int row) {
  if (a.logp) a.logp[row] = 0.f;
  if (a.entropy) a.entropy[row] = 0.f;
  if (a.stats) a.stats[2 * (size_t)row] = 0.f, a.stats[2 * (size_t)row + 1] = 0.f;
}

// Maximum and sums over the units [lo, hi) of a row, by `waves` waves of which this is number `wave`: this lane's part.
// Units of one batch are summed apart from what came before: a small term is added to a sum of a few, not to a sum
// that one large value dominates.
template <typename T, bool KEYS>
__device__ __forceinline__ Soft scan_units(const T* zr, int V, float c, int lo, int hi, int wave, int waves,
                                           uint32_t* keys) {
  constexpr int N = Chunk16<T>::N;
  const int lane = threadIdx.x & 63;
  Soft a = {-INFINITY, 0.f, 0.f};
  for (int u0 = lo + wave * kUnits; u0 < hi; u0 += waves * kUnits) {
    u32x4 raw[kUnits];
    if (u0 + kUnits <= hi && (int64_t)(u0 + kUnits) * 64 * N <= V) {
#pragma unroll
      for (int j = 0; j < kUnits; ++j) raw[j] = stream16(zr + (u0 + j) * 64 * N + lane * N);
    } else {
      u32x4 none;  // nothing but -inf
#pragma unroll
      for (int i = 0; i < 4; ++i) none[i] = N == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
      for (int j = 0; j < kUnits; ++j)
        raw[j] = u0 + j < hi ? load_row(zr, (u0 + j) * 64 * N + lane * N, V) : none;
    }
    float bm = -INFINITY;
    static_assert(kUnits == 4);
    uint32_t key[kUnits];  // of the units' maxima
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      float v[N];
      unpack16(raw[j], v);
      float um = v[0];
#pragma unroll
      for (int i = 1; i < N; ++i) um = fmaxf(um, v[i]);
      bm = fmaxf(bm, um);
      if (KEYS) key[j] = key_of(um);
    }
    if (KEYS) {
      const uint32_t k = wave_max_of_four(key);
      if (lane < kUnits && u0 + lane < hi) keys[u0 + lane] = k;
    }
    bm = fmaxf(a.m, bm);
    const float mm = finite_or_zero(bm);
    a = moved(a, bm, c);
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      float v[N];
      unpack16(raw[j], v);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float t = (v[i] - mm) * c, e = __builtin_amdgcn_exp2f(t);
        s += e;
        w = fmaf(e, fmaxf(t, kLow), w);
      }
    }
    a.s += s;
    a.w += w;
  }
  return a;
}

// A wave's lanes joined, the same in every lane.
__device__ __forceinline__ Soft joined_wave(Soft a, float c) {
  a = moved(a, wave_max_f32(a.m), c);
  a.s = wave_sum_f32(a.s);
  a.w = wave_sum_f32(a.w);
  return a;
}

__host__ __device__ constexpr int units_of(int V, int N) { return (int)(((int64_t)V + 64 * N - 1) / (64 * N)); }

// A part of a row: chunk blockIdx.y of units_a_chunk units, by TEAM waves (a workgroup's other waves do other rows).
// With one chunk and no alternatives it is the whole row and its outputs are written here; otherwise the part goes to
// part[row][chunk] and k_logprobs_join does the rest.
template <typename T, int TEAM, bool KEYS>
__global__ __launch_bounds__(RB) void k_logprobs(LogprobArgs a, float c, int units_a_chunk, Soft* __restrict__ part,
                                                 uint32_t* __restrict__ keys) {
  constexpr int N = Chunk16<T>::N;
  __shared__ Soft team[RW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nseg = units_of(a.vocab, N), chunks = gridDim.y, chunk = blockIdx.y;
  const int lo = chunk * units_a_chunk, hi = min(lo + units_a_chunk, nseg);
  for (int row = blockIdx.x * (RW / TEAM) + wave / TEAM; row < a.rows; row += gridDim.x * (RW / TEAM)) {
    const int token = a.tokens ? a.tokens[row] : 0;
    if (token < 0) {
      if (!part && lane == 0 && wave % TEAM == 0) finish_padding(a, row);
      continue;  // the same for a whole team
    }
    const T* zr = (const T*)a.z + (int64_t)row * a.stride;
    const float x = part ? 0.f : token_logit<T>(a, row, token);  // on its way meanwhile
    Soft r = joined_wave(scan_units<T, KEYS>(zr, a.vocab, c, lo, hi, wave % TEAM, TEAM,
                                             KEYS ? keys + (int64_t)row * nseg : nullptr), c);
    if (TEAM > 1) {
      __syncthreads();
      if (lane == 0) team[wave] = r;
      __syncthreads();
      if (wave) continue;
      r = joined_wave(lane < TEAM ? team[lane] : Soft{-INFINITY, 0.f, 0.f}, c);
    }
    if (lane == 0) {
      if (part)
        part[(int64_t)row * chunks + chunk] = r;
      else
        finish_row(a, row, x, r);
    }
  }
}

// A row's parts joined, and its alternatives: one workgroup a row with alternatives, otherwise one wave.  Bound by its chain
// of reads (parts and keys, units, the token's logit) and by the ranking: 64 rows with 8 alternatives 6.0 us, 256 with 20 8.3,
// of which 4 are the launch and the first reads.
template <typename T, bool TOP>
__global__ __launch_bounds__(RB) void k_logprobs_join(LogprobArgs a, float c, int chunks, const Soft* __restrict__ part,
                                                      const uint32_t* __restrict__ keys) {
  constexpr int N = Chunk16<T>::N;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int step = TOP ? 1 : RW;
  for (int row = blockIdx.x * step + (TOP ? 0 : wave); row < a.rows; row += gridDim.x * step) {
    // everything that is needed first is asked for at once
    const int nseg = units_of(a.vocab, N);
    const Soft mine = lane < chunks ? part[(int64_t)row * chunks + lane] : Soft{-INFINITY, 0.f, 0.f};
    uint32_t unit_keys[kMaxPer];
    if (TOP)
#pragma unroll
      for (int i = 0; i < kMaxPer; ++i) unit_keys[i] = i * 64 + lane < nseg ? keys[(int64_t)row * nseg + i * 64 + lane] : 0u;
    const int token = a.tokens ? a.tokens[row] : 0;
    const size_t t0 = (size_t)row * a.top;
    if (token < 0) {
      if (lane == 0 && (!TOP || wave == 0)) finish_padding(a, row);
      if (TOP && threadIdx.x < a.top) a.top_ids[t0 + threadIdx.x] = -1, a.top_logp[t0 + threadIdx.x] = 0.f;
      continue;
    }
    const float x = token_logit<T>(a, row, token);
    const Soft r = joined_wave(mine, c);
    if constexpr (TOP) {
      __shared__ TopLds lds;
      if (!(r.s == r.s)) {
        if (threadIdx.x < a.top) a.top_ids[t0 + threadIdx.x] = -1, a.top_logp[t0 + threadIdx.x] = NAN;
      } else {
        // a row of -inf alone: every distance to the maximum is -inf
        take_top((const T*)a.z + (int64_t)row * a.stride, a.vocab, a.top, keys + (int64_t)row * nseg, nseg, lds,
                 finite_or_zero(r.m), a.temperature, r.m == -INFINITY ? 0.f : logf(r.s), a.top_ids + t0, a.top_logp + t0,
                 unit_keys);
      }
    }
    if (lane == 0 && (!TOP || wave == RW - 1)) finish_row(a, row, x, r);
  }
}

// z and dz may be the same matrix: a thread reads its values before it writes them.  `team` threads (a power of two) do one
// step of a row, `loads` (at most kBatch) times 16 bytes a thread; a workgroup does several short rows.  More than one step a
// workgroup is slower (4,096 x 152,064 bf16 488 us with five, 480 with one).  What is written is not read again soon; what is
// read may be in the last-level cache if the matrix fits there (beyond: matrices of more than that): 512 x 152,064 bf16 read
// past the caches 64.7 us, through them 55.3; 4,096 rows 488 and 496.
template <typename T>
__global__ __launch_bounds__(RB) void k_logprobs_backward(LogprobGradArgs a, int team, int loads, bool beyond) {
  constexpr int N = Chunk16<T>::N;
  const int V = a.vocab, each = RB / team;
  const int i0 = (blockIdx.x * team * loads + (threadIdx.x & (team - 1))) * N;
  const float inv_t = 1.f / a.temperature, c = kLog2e / a.temperature;
  for (int64_t r0 = (int64_t)blockIdx.y * each + threadIdx.x / team; r0 < a.rows; r0 += (int64_t)gridDim.y * each) {
    const int row = (int)r0;
    const T* zr = (const T*)a.z + (int64_t)row * a.stride;
    T* dr = (T*)a.dz + (int64_t)row * a.dz_stride;
    const int token = a.tokens[row];
    const float m = a.stats[2 * (size_t)row], ln_s = a.stats[2 * (size_t)row + 1];
    const float g = a.g[row], h = a.h ? a.h[row] : 0.f, H = a.h ? a.entropy[row] : 0.f;
    const bool dead = token < 0 || (g == 0.f && h == 0.f) || m == -INFINITY;
    const float l2 = ln_s * kLog2e, gt = g * inv_t, ht = h * inv_t;
    const float spoil = token >= V ? NAN : 0.f;
    u32x4 raw[kBatch];
    if (!dead) {
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int i = i0 + b * team * N;
        if (b >= loads || i >= V) break;
        if (i + N > V)
          raw[b] = load_row(zr, i, V);
        else
          raw[b] = beyond ? stream16(zr + i) : load16(zr + i);
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = i0 + b * team * N;
      if (b >= loads || i >= V) break;
      float d[N];
      if (dead) {
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] = 0.f;
      } else {
        float v[N];
        unpack16(raw[b], v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float t = fmaf(v[j] - m, c, -l2), p = __builtin_amdgcn_exp2f(t);
          const float k = fmaf(ht, fmaf(fmaxf(t, kLow), kLn2, H), gt) + spoil;
          d[j] = -p * k;
        }
        if ((unsigned)(token - i) < (unsigned)N) {
#pragma unroll
          for (int j = 0; j < N; ++j) d[j] += i + j == token ? gt : 0.f;
        }
      }
      if (i + N <= V) {
        stream16(dr + i, pack16(d));
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (i + j < V) put(dr + i + j, d[j]);
      }
    }
  }
}

struct Split {
  int chunks, units;  // of a row; units of a chunk
};
// Enough workgroups for the whole card where rows are few; a wave's share of a chunk is one batch of loads at least.
// Chunks are whole batches of a workgroup's loads, the nearest number of them, so that no wave does a rest alone (64 rows of
// 152,064 fp32 ids with 8 alternatives 19.3 us with chunks of 19 units, 18.0 with 16; bf16 17.6 and 16.3).
// Short rows stay whole, whose second kernel would take longer than the loads it shares out (8,192 fp32 ids, 1 and 64 rows:
// 5.2 and 5.4 us whole, 6.8 and 7.5 split; 32,003 ids 7.7 and 10.7 whole, 7.1 and 8.5 split); with alternatives there is a
// second kernel anyway (128 rows of 32,003 bf16 ids with 5 19.1 us whole, 15.7 split; 300 of 8,192 fp32 15.1 and 14.3).
constexpr int kBatchUnits = RW * kUnits;
int most_chunks(int nseg, bool join) { return nseg <= kWhole && !join ? 1 : std::min(kMaxChunks, nseg / kBatchUnits); }
Split split_of(int rows, int nseg, bool join) {
  const int want = std::max(1, std::min(most_chunks(nseg, join), kWorkgroups / rows));
  if (want == 1) return {1, nseg};
  int units = (nseg + want - 1) / want;
  const int whole = std::max(kBatchUnits, (units + kBatchUnits / 2) / kBatchUnits * kBatchUnits);
  units = (nseg + whole - 1) / whole <= kMaxChunks ? whole : (units + kBatchUnits - 1) / kBatchUnits * kBatchUnits;
  return {(nseg + units - 1) / units, units};
}

template <typename T, bool KEYS>
void forward(hipStream_t s, const LogprobArgs& a, char* ws) {
  constexpr int N = Chunk16<T>::N;
  const float c = (float)(1.4426950408889634 / (double)a.temperature);
  const int nseg = units_of(a.vocab, N);
  // A wave a row where rows are short and many, so that no wave waits for others over a few loads (fp32, 20,000 rows of 2,064
  // ids 29 us, 37 by workgroups; bf16, 4,000 of 4,099 12.2 and 15.5, 12,000 of 32,003 128 and 153, of 32,000 125 and 120).
  // Fewer rows are too few waves (bf16, 1,500 of 4,099 8.1 and 7.3, of 32,003 26.8 and 24.8; 1,100 of 16,000 fp32 21.4 and
  // 16.1).
  const bool waves = nseg <= kUnits || (nseg <= kWhole && a.rows >= kWaveRows);
  const Split p = waves ? Split{1, nseg} : split_of(a.rows, nseg, KEYS);
  const bool join = KEYS || p.chunks > 1;
  Soft* part = join ? (Soft*)ws : nullptr;
  uint32_t* keys = KEYS ? (uint32_t*)(part + (size_t)a.rows * p.chunks) : nullptr;
  if (waves)
    hipLaunchKernelGGL((k_logprobs<T, 1, KEYS>), dim3(std::min((a.rows + RW - 1) / RW, kMaxGrid)), dim3(RB), 0, s, a, c, nseg,
                       part, keys);
  else
    hipLaunchKernelGGL((k_logprobs<T, RW, KEYS>), dim3(std::min(a.rows, kMaxGrid), p.chunks), dim3(RB), 0, s, a, c, p.units,
                       part, keys);
  if (join)
    hipLaunchKernelGGL((k_logprobs_join<T, KEYS>), dim3(std::min(KEYS ? a.rows : (a.rows + RW - 1) / RW, kMaxGrid)), dim3(RB), 0,
                       s, a, c, p.chunks, part, keys);
}

template <typename T>
void backward(hipStream_t s, const LogprobGradArgs& a) {
  constexpr int N = Chunk16<T>::N;
  const bool beyond = (size_t)a.rows * a.vocab * sizeof(T) > kLastLevelBytes;
  int team = 1;
  while (team < RB && team * N * kBatch < a.vocab) team *= 2;
  // steps of about the same size: a row a little longer than a step is not a step and a rest
  const int all = (a.vocab + team * N - 1) / (team * N), steps = (all + kBatch - 1) / kBatch, loads = (all + steps - 1) / steps;
  const int each = RB / team;
  hipLaunchKernelGGL(k_logprobs_backward<T>, dim3(steps, std::min((a.rows + each - 1) / each, 65535)), dim3(RB), 0, s, a, team,
                     loads, beyond);
}

}  // namespace

// Parts, and the keys of the units, for the type with more units.  As many parts as any number of rows up to this one has, so
// that the workspace of a large call serves small ones.
size_t logprobs_workspace(int rows, int vocab, int top) {
  const size_t units = units_of(vocab, 4);
  // r rows have at most kWorkgroups / r chunks each and half as many again where these are rounded to whole batches, and at
  // most kWorkgroups / 2 rows have more than one
  const size_t split = most_chunks((int)units, top > 0) > 1 ? std::min((size_t)rows * kMaxChunks, 2 * (size_t)kWorkgroups) : 0;
  return (top ? std::max((size_t)rows, split) : split) * sizeof(Soft) + (top ? (size_t)rows * units * 4 : 0);
}

hipError_t launch_logprobs(hipStream_t s, int dtype, const LogprobArgs& a, void* ws) {
  if (dtype == ROLLOUT_DTYPE_BF16)
    a.top ? forward<uint16_t, true>(s, a, (char*)ws) : forward<uint16_t, false>(s, a, (char*)ws);
  else
    a.top ? forward<float, true>(s, a, (char*)ws) : forward<float, false>(s, a, (char*)ws);
  return hipGetLastError();
}

hipError_t launch_logprobs_backward(hipStream_t s, int dtype, const LogprobGradArgs& a) {
  dtype == ROLLOUT_DTYPE_BF16 ? backward<uint16_t>(s, a) : backward<float>(s, a);
  return hipGetLastError();
}

}  // namespace rollout
