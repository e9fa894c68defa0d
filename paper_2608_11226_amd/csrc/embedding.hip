// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   out_n = scale E[id_n];     dE_v = scale sum over n with id_n = v of g_n   (+ the old dE_v)
//
// The gradient sorts (id, position) pairs by id with a stable radix sort, so that a row's tokens stand together in
// token order, and adds up each run in an order that follows from its place among them: no atomics on floats, the same bits on
// every such call.  A run's length is anything from one to all of the tokens (text repeats its frequent ids), so runs are cut at
// fixed places of the sorted order: every 32 entries (16 in batches of some hundreds to some ten thousand tokens) that belong to
// one id are summed beforehand, and in long batches every 32 such sums once more.
//
// Both are bound by HBM where there is much to move: 49,152 rows of 3,584 looked up in 186 us (705 MB written beside some 150 MB
// of scattered rows), their gradient into 152,064 fp32 rows in 491 us (2.18 GB, most of it zeros, beside 308 MB of gathered
// rows: 5.1 TB/s).  Small gradients are three launches (2,048 tokens x 128: sort 8.8, rows 6.2, long rows 5.8 us).
#include "update.h"

#include <type_traits>

namespace rollout {
namespace {

constexpr int EB = 256;
// Figures below are of the gradient of 49,152 tokens x 3,584 (bf16, text-like ids) into 152,064 fp32 rows, in all its launches,
// and of 2,048 tokens x 128 (fp32) into 1,024 rows.
// Entries of a piece (and pieces of a large piece): 1 << piece_shift(n, dim).  Pieces of 32 are best where there is much to add
// (16, 32 and 64: 510, 488 and 484 us, 60,000 tokens x 640 88.8, 80.2 and 84.0), of 16 where the steps one after another count
// (2,048 x 128 21.1, 23.5 and 25.7, 8,000 x 1,000 45.7, 48.8 and more, 16,000 x 1,000 49.1 and 52.6), and neither in
// between (24,000 x 1,000 63.8 and 63.3, 28,000 x 640 55.5 and 55.1, 16,000 x 2,048 59.3 and 58.3).  Few text-like tokens have
// no run of 32 (300 x 128 16.5 and 13.8, 300 x 1,000 22.4 and 20.5; 500 x 128 17.7 and 18.1, 600 x 1,000 23.4 and 23.8).
constexpr int kPieceShift = 5, kPiece = 1 << kPieceShift;
constexpr int kFewTokens = 400, kSmallPieceTokens = 1 << 15, kSmallPieceValues = 1 << 24;
inline int piece_shift(int n, int dim) {
  return n >= kFewTokens && n < kSmallPieceTokens && (int64_t)n * dim <= kSmallPieceValues ? kPieceShift - 1 : kPieceShift;
}
constexpr int kAhead = 8;                // rows in flight
constexpr int kEntries = 8;              // sorted entries whose rows a workgroup does (4, 8, 16: 483, 494, 498 us; 60,000 x
                                         // 640 67, 62 and 62; 2,048 x 128 20.2, 19.5 and 20.7)
// Rows without tokens: about this many values a workgroup (4,096 491 us, 16,384 493, 65,536 501), if that leaves this many
// workgroups.
constexpr int kRowValues = 16384, kRowWorkgroups = 8192, kMaxRowWorkgroups = 1 << 23;
// Threads and most workgroups of the long rows (256 threads 515 us instead of 493, 128 workgroups 505).
constexpr int kLongThreads = 1024, kLongWorkgroups = 512;
// From so many pieces on (65,536 tokens) pieces are summed to large ones first: one id's 2,047 pieces are 64 steps of a long
// row's groups, and the kernel that sums them takes 7 us whether there is such an id or not.
constexpr int kManyPieces = 2048;
// Bytes of zeros that a launch of the sort writes beside it (none 526 us, 80 MB 497, 160 MB 493, 320 MB 496; 5,000 tokens by
// tiles into a bf16 table 231, 203, 201 and 226), that of the long rows (none 497 us, 96 MB 494, 200 MB 486),
// and a workgroup (300 tokens into 152,064 x 3,584 fp32: 16 KB 362 us, 64 KB 433, 256 KB 382).
constexpr size_t kSortFill = 160u << 20, kLongFill = 96u << 20, kFill = 16384;
constexpr int kMaxFillBlocks = 1 << 20;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortWaves = EB / 64;
constexpr int kMaxTiles = 256;
constexpr int kHeld = 4;                 // keys that a lane holds on to
// Up to so many tokens one workgroup sorts alone, in LDS (6,000 x 640 34.3 us, by tiles 36.0, 5,000 x 1,000 33.6 and 41.1;
// 7,900 x 640 would take 39.5 and by tiles 35.8).
constexpr int kSmallSort = 6144, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;

// ---------------------------------------------------------------------------
// pieces of rows: P values from any element on, of which n exist
// ---------------------------------------------------------------------------
struct Half8 {
  typedef uint32_t Raw __attribute__((ext_vector_type(2), aligned(2), may_alias));  // four bf16 values
};

template <int P>
__device__ __forceinline__ void load_values(const float* p, int n, float (&v)[P]) {
  static_assert(P == 4);
  if (n >= 4) {
    unpack16(load16(p), v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < n ? p[j] : 0.f;
  }
}
template <int P>
__device__ __forceinline__ void load_values(const uint16_t* p, int n, float (&v)[P]) {
  if (n >= P) {
    if constexpr (P == 8) {
      unpack16(load16(p), v);
    } else {
      const Half8::Raw r = *reinterpret_cast<const Half8::Raw*>(p);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        v[2 * j] = __uint_as_float(r[j] << 16);
        v[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < P; ++j) v[j] = j < n ? bf16_to_f32(p[j]) : 0.f;
  }
}
// The same four values as they stand in memory, to be widened where they are used.
template <typename T>
struct Raw4;
template <>
struct Raw4<float> {
  u32x4 r;
};
template <>
struct Raw4<uint16_t> {
  uint32_t r[2];
};
__device__ __forceinline__ Raw4<float> load_raw(const float* p, int n) {
  if (n >= 4) return {load16(p)};
  float v[4];
  load_values(p, n, v);
  return {pack16(v)};
}
__device__ __forceinline__ Raw4<uint16_t> load_raw(const uint16_t* p, int n) {
  if (n >= 4) {
    const Half8::Raw q = *reinterpret_cast<const Half8::Raw*>(p);
    return {{q[0], q[1]}};
  }
  uint32_t v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = j < n ? p[j] : 0u;
  return {{v[0] | v[1] << 16, v[2] | v[3] << 16}};
}
__device__ __forceinline__ void add_raw(float (&v)[4], const Raw4<float>& q) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(q.r[i]);
}
__device__ __forceinline__ void add_raw(float (&v)[4], const Raw4<uint16_t>& q) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[2 * i] += __uint_as_float(q.r[i] << 16);
    v[2 * i + 1] += __uint_as_float(q.r[i] & 0xFFFF0000u);
  }
}
// Results are not read again soon: stores past the caches.
template <int P>
__device__ __forceinline__ void store_values(float* p, int n, const float (&v)[P]) {
  static_assert(P == 4);
  if (n >= 4) {
    stream16(p, pack16(v));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = v[j];
  }
}
template <int P>
__device__ __forceinline__ void store_values(uint16_t* p, int n, const float (&v)[P]) {
  if (n >= P) {
    if constexpr (P == 8) {
      stream16(p, pack16(v));
    } else {
      Half8::Raw r;
#pragma unroll
      for (int j = 0; j < 2; ++j) r[j] = (uint32_t)round_bf16(v[2 * j]) | ((uint32_t)round_bf16(v[2 * j + 1]) << 16);
      __builtin_nontemporal_store(r, reinterpret_cast<Half8::Raw*>(p));
    }
  } else {
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (j < n) p[j] = round_bf16(v[j]);
  }
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
// A workgroup a token, 16 bytes a lane of the wider type, kAhead of them on their way (a wave a token: 197 to 201 us instead
// of 186 in the case above).
template <typename T, typename O>
__global__ __launch_bounds__(EB) void k_embedding(const T* __restrict__ table, int vocab, int dim,
                                                  const int32_t* __restrict__ tokens, int n, float scale,
                                                  O* __restrict__ out) {
  constexpr int P = sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4, kAhead = 4;
  for (int row = blockIdx.x; row < n; row += gridDim.x) {
    const int id = tokens[row];
    const bool have = id >= 0 && id < vocab;
    const T* src = table + (size_t)(have ? id : 0) * dim;
    O* dst = out + (size_t)row * dim;
    for (int c0 = threadIdx.x * P; c0 < dim; c0 += EB * P * kAhead) {
      float v[kAhead][P];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int c = c0 + k * EB * P;
        if (c < dim && have) load_values(src + c, dim - c, v[k]);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int c = c0 + k * EB * P;
        if (c >= dim) break;
#pragma unroll
        for (int j = 0; j < P; ++j) v[k][j] = have ? v[k][j] * scale : id < 0 ? 0.f : NAN;
        store_values(dst + c, dim - c, v[k]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// stable sort of (id, position)
// ---------------------------------------------------------------------------
// an id's key: itself, or vocab (behind all rows) where no row belongs to it
__device__ __forceinline__ int key_of_token(int id, int vocab) { return id >= 0 && id < vocab ? id : vocab; }

// One stable step of a wave: 64 keys (valid: this lane holds one) take their places after all that came before.
// place[d] is the next free place of digit d.
__device__ __forceinline__ int take_place(uint32_t* place, int digit, bool valid, int bits) {
  unsigned long long same = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot((digit >> b) & 1);
    same &= (digit >> b) & 1 ? set : ~set;
  }
  const int lane = threadIdx.x & 63;
  const int rank = __popcll(same & ((1ull << lane) - 1));
  const uint32_t first = valid ? place[digit] : 0;
  __builtin_amdgcn_wave_barrier();
  if (valid && rank == 0) place[digit] = first + (uint32_t)__popcll(same);
  __builtin_amdgcn_wave_barrier();
  return (int)(first + rank);
}

struct SortPass {
  const int32_t* tokens;  // the first pass reads these, later ones key_in and pos_in
  const int32_t *key_in, *pos_in;
  int32_t *key_out, *pos_out;
  int n, vocab, shift, bits, sub;  // sub: keys of a wave
};

__device__ __forceinline__ int key_at(const SortPass& p, int i) {
  return p.tokens ? key_of_token(p.tokens[i], p.vocab) : p.key_in[i];
}

// Zeros over a range of bytes (both types' zeros; a multiple of two bytes, anywhere): `each` of them a workgroup.
struct Fill {
  char* to;
  size_t bytes, each;
};
typedef uint32_t Any16 __attribute__((ext_vector_type(4), aligned(2), may_alias));
int fill_blocks(const Fill& f) { return (int)((f.bytes + f.each - 1) / f.each); }
__device__ __forceinline__ void fill_zeros(const Fill& f, int block) {
  const size_t lo = (size_t)block * f.each, hi = lo + f.each < f.bytes ? lo + f.each : f.bytes;
  for (size_t i = lo + threadIdx.x * 16; i < hi; i += blockDim.x * 16) {
    if (i + 16 <= hi) {
      const u32x4 zero = {0, 0, 0, 0};
      __builtin_nontemporal_store(zero, reinterpret_cast<Any16*>(f.to + i));
    } else {
      for (size_t j = i; j < hi; j += 2) *reinterpret_cast<uint16_t*>(f.to + j) = 0;
    }
  }
}

// A pass of the sort is two launches: the digits of every tile (a workgroup's keys) are counted, then every workgroup adds up
// the other tiles' counts itself and places its keys.  49,152 tokens take 4.8 and 8.2 us a pass without the zeros beside them.
// (The next pass's counts by atomics on memory while keys are placed, a launch less: 16,000 tokens x 640 48.0 instead of 41.4
// us at the time.)
// The workgroups behind the tiles zero a share of the table: the sort leaves most of the card free.
//
// Digit counts into hist[tile][digit].  The first pass also empties the rows' runs and the list of long rows.
__global__ __launch_bounds__(EB) void k_sort_count(SortPass p, int tiles, uint32_t* __restrict__ hist, int2* __restrict__ runs,
                                                   int32_t* __restrict__ longs, Fill fill) {
  __shared__ uint32_t cnt[kDigits];
  if ((int)blockIdx.x >= tiles) return fill_zeros(fill, blockIdx.x - tiles);
  for (int d = threadIdx.x; d < kDigits; d += EB) cnt[d] = 0;
  __syncthreads();
  const int lo = min((int64_t)blockIdx.x * p.sub * kSortWaves, (int64_t)p.n);
  const int hi = (int)min((int64_t)lo + (int64_t)p.sub * kSortWaves, (int64_t)p.n);
  const int mask = (1 << p.bits) - 1;
  for (int i = lo + threadIdx.x; i < hi; i += EB) atomicAdd(&cnt[(key_at(p, i) >> p.shift) & mask], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < kDigits; d += EB) hist[(size_t)blockIdx.x * kDigits + d] = cnt[d];
  if (runs && blockIdx.x == 0 && threadIdx.x == 0) *longs = 0;
  if (runs)
    for (int v = blockIdx.x * EB + threadIdx.x; v < p.vocab; v += tiles * EB) runs[v] = make_int2(0, 0);
}

__global__ __launch_bounds__(EB) void k_sort_place(SortPass p, int tiles, const uint32_t* __restrict__ hist, Fill fill) {
  static_assert(kDigits == 2 * EB && kDigits == 8 * 64);
  __shared__ uint32_t counts[2][kSortWaves][kDigits];
  __shared__ uint32_t place[kSortWaves][kDigits];
  __shared__ uint32_t total[kSortWaves];
  if ((int)blockIdx.x >= tiles) return fill_zeros(fill, blockIdx.x - tiles);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mask = (1 << p.bits) - 1;
  for (int i = threadIdx.x; i < kSortWaves * kDigits; i += EB) (&place[0][0])[i] = 0;
  __syncthreads();
  const int lo = (int)min(((int64_t)blockIdx.x * kSortWaves + wave) * p.sub, (int64_t)p.n);
  const int hi = (int)min((int64_t)lo + p.sub, (int64_t)p.n);
  int held[kHeld];  // the wave's first keys
#pragma unroll
  for (int j = 0; j < kHeld; ++j) held[j] = lo + j * 64 + lane < hi ? key_at(p, lo + j * 64 + lane) : -1;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (held[j] >= 0) atomicAdd(&place[wave][(held[j] >> p.shift) & mask], 1u);
  for (int i = lo + kHeld * 64 + lane; i < hi; i += 64) atomicAdd(&place[wave][(key_at(p, i) >> p.shift) & mask], 1u);
  // The counts of all tiles and of the earlier ones: a lane adds up eight digits of every fourth tile, then thread t the four
  // waves' sums of digits 2 t and 2 t + 1.
  {
    uint32_t sum[8] = {}, early[8] = {};
#pragma unroll 4
    for (int t = wave; t < tiles; t += kSortWaves) {
      const uint4* h = reinterpret_cast<const uint4*>(hist + (size_t)t * kDigits + 8 * lane);
      const uint4 x = h[0], y = h[1];
      const uint32_t q[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[i] += q[i];
        early[i] += t < (int)blockIdx.x ? q[i] : 0u;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) counts[0][wave][8 * lane + i] = sum[i], counts[1][wave][8 * lane + i] = early[i];
  }
  __syncthreads();
  uint32_t all[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      all[j] += counts[0][w][2 * threadIdx.x + j];
      before[j] += counts[1][w][2 * threadIdx.x + j];
    }
  // exclusive scan over the digits
  uint32_t sum = all[0] + all[1];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t q = __shfl_up(sum, o, 64);
    if (lane >= o) sum += q;
  }
  if (lane == 63) total[wave] = sum;
  __syncthreads();
  uint32_t base = sum - all[0] - all[1];
  for (int w = 0; w < wave; ++w) base += total[w];
  uint32_t at[2] = {base + before[0], base + all[0] + before[1]};
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = place[w][2 * threadIdx.x + j];
      place[w][2 * threadIdx.x + j] = at[j];
      at[j] += c;
    }
  __syncthreads();
  int from[kHeld];  // their positions
#pragma unroll
  for (int j = 0; j < kHeld; ++j) from[j] = held[j] >= 0 && !p.tokens ? p.pos_in[lo + j * 64 + lane] : lo + j * 64 + lane;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const bool valid = held[j] >= 0;
    if (!__ballot(valid)) break;
    const int to = take_place(place[wave], (held[j] >> p.shift) & mask, valid, p.bits);
    if (valid) p.key_out[to] = held[j], p.pos_out[to] = from[j];
  }
  for (int i0 = lo + kHeld * 64; i0 < hi; i0 += 64) {
    const int i = i0 + lane;
    const bool valid = i < hi;
    const int key = valid ? key_at(p, i) : 0;
    const int to = take_place(place[wave], (key >> p.shift) & mask, valid, p.bits);
    if (valid) {
      p.key_out[to] = key;
      p.pos_out[to] = p.tokens ? i : p.pos_in[i];
    }
  }
}

// Where the runs of sorted keys begin and end: what entry i knows of it.
__device__ __forceinline__ void note_run(const int32_t* key, int i, int n, int vocab, int2* runs) {
  const int k = key[i];
  if (k >= vocab) return;
  if (i == 0 || key[i - 1] != k) runs[k].x = i;
  if (i == n - 1 || key[i + 1] != k) runs[k].y = i + 1;
}

// All passes by one workgroup, in LDS, for n up to kSmallSort, and the runs; the other workgroups zero the table.
__global__ __launch_bounds__(kSmallThreads) void k_sort_small(const int32_t* __restrict__ tokens, int n, int vocab, int passes,
                                                              int bits, int32_t* __restrict__ key_out,
                                                              int32_t* __restrict__ pos_out, int2* __restrict__ runs,
                                                              int32_t* __restrict__ longs, Fill fill) {
  __shared__ int32_t lds[4 * kSmallSort];  // keys and positions, of two buffers
  __shared__ uint32_t place[kSmallWaves][kDigits];
  __shared__ uint32_t total[kDigits / 64];
  if (blockIdx.x) return fill_zeros(fill, blockIdx.x - 1);
  if (threadIdx.x == 0) *longs = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = ((n + kSmallWaves - 1) / kSmallWaves + 63) & ~63;
  const int mask = (1 << bits) - 1;
  int32_t *key = lds, *pos = lds + n, *key2 = lds + 2 * n, *pos2 = lds + 3 * n;
  for (int i = threadIdx.x; i < n; i += kSmallThreads) key[i] = key_of_token(tokens[i], vocab), pos[i] = i;
  const int lo = min(wave * sub, n), hi = min(lo + sub, n);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int i = threadIdx.x; i < kSmallWaves << bits; i += kSmallThreads) place[i >> bits][i & mask] = 0;
    __syncthreads();
    for (int i = lo + lane; i < hi; i += 64) atomicAdd(&place[wave][(key[i] >> shift) & mask], 1u);
    __syncthreads();
    uint32_t all = 0, sum = 0;
    if ((int)threadIdx.x <= mask) {
      for (int w = 0; w < kSmallWaves; ++w) all += place[w][threadIdx.x];
      sum = all;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t q = __shfl_up(sum, o, 64);
      if (lane >= o) sum += q;
    }
    if (lane == 63 && wave < kDigits / 64) total[wave] = sum;
    __syncthreads();
    if ((int)threadIdx.x <= mask) {
      uint32_t at = sum - all;
      for (int w = 0; w < wave; ++w) at += total[w];
      for (int w = 0; w < kSmallWaves; ++w) {
        const uint32_t c = place[w][threadIdx.x];
        place[w][threadIdx.x] = at;
        at += c;
      }
    }
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + lane;
      const bool valid = i < hi;
      const int k = valid ? key[i] : 0;
      const int to = take_place(place[wave], (k >> shift) & mask, valid, bits);
      if (valid) key2[to] = k, pos2[to] = pos[i];
    }
    __syncthreads();
    int32_t* t = key;
    key = key2, key2 = t;
    t = pos, pos = pos2, pos2 = t;
  }
  for (int i = threadIdx.x; i < n; i += kSmallThreads) {
    key_out[i] = key[i], pos_out[i] = pos[i];
    note_run(key, i, n, vocab, runs);
  }
}

// ---------------------------------------------------------------------------
// sums of runs
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(EB) void k_embedding_runs(const int32_t* __restrict__ key, int n, int vocab,
                                                       int2* __restrict__ runs) {
  const int i = blockIdx.x * EB + threadIdx.x;
  if (i < n) note_run(key, i, n, vocab, runs);
}

// How a workgroup shares out a slab of a row (4 EB columns at most): `width` threads (a power of two, at most EB) side by
// side do four columns each; the groups of them share out what is added up.
struct Shape {
  int width, groups, group, col;  // group and first column of this thread
};
__device__ __forceinline__ Shape shape_of(int width) {
  return {width, (int)blockDim.x / width, (int)threadIdx.x / width, ((int)threadIdx.x & (width - 1)) * 4};
}

// v += rows lo .. hi of g (those that pos names, or with pos NULL these themselves) at columns c .. c + 3, in order.  All lanes
// of a group call it, also those behind the last column: half a wave (a group has whole ones) reads 32 positions at once, a
// lane each, so that a batch of rows waits for itself alone (16,000 tokens into 2,064 x 640, bf16 into fp32, 56.0 -> 43.8 us;
// batches of 4 rows 45.7, of 16 44.5).
template <typename T>
__device__ __forceinline__ void add_rows(float (&v)[4], const T* g, const int32_t* pos, int lo, int hi, int dim, int c) {
  const int half = threadIdx.x & 32;
  for (int i0 = lo; i0 < hi; i0 += 32) {
    int mine = i0 + (threadIdx.x & 31);
    if (pos) mine = pos[min(mine, hi - 1)];
    const int end = min(i0 + 32, hi);
    for (int i = i0; i < end; i += kAhead) {
      Raw4<T> q[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int at = __shfl(mine, half + ((i - i0 + j) & 31), 64);
        if (i + j < end && c < dim) q[j] = load_raw(g + (size_t)at * dim + c, dim - c);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < end && c < dim) add_raw(v, q[j]);
    }
  }
}
// the group's share of lo .. hi
template <typename T>
__device__ __forceinline__ void add_share(float (&v)[4], const Shape& sh, const T* g, const int32_t* pos, int lo, int hi,
                                          int dim, int c) {
  const int each = (hi - lo + sh.groups - 1) / sh.groups;
  add_rows(v, g, pos, min(lo + sh.group * each, hi), min(lo + (sh.group + 1) * each, hi), dim, c);
}
// The groups' sums joined in the groups' order, for group 0.  All threads call it; lds holds a float4 each.
__device__ __forceinline__ void join_groups(float (&v)[4], const Shape& sh, float4* lds) {
  if (sh.groups == 1) return;
  __syncthreads();
  lds[threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
  __syncthreads();
  if (sh.group == 0)
    for (int g = 1; g < sh.groups; ++g) {
      const float4 q = lds[g * sh.width + threadIdx.x];
      v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
    }
}

// whole pieces [p, q) and whole large pieces [P, Q) of a run
struct Pieces {
  int p, q, P, Q;
};
__device__ __forceinline__ Pieces pieces_of(int2 run, int shift) {
  Pieces r;
  r.p = (run.x + (1 << shift) - 1) >> shift, r.q = max(run.y >> shift, r.p);
  r.P = (r.p + kPiece - 1) / kPiece, r.Q = max(r.q / kPiece, r.P);
  return r;
}
__device__ __forceinline__ bool whole_piece(const int32_t* key, int p, int shift, int n, int vocab) {
  return p < n >> shift && key[p << shift] < vocab && key[p << shift] == key[((p + 1) << shift) - 1];
}

// dst row = scale * sum (+ dst row)
template <typename O, bool ACC>
__device__ __forceinline__ void write_row(O* dst, int dim, int c, float scale, float (&v)[4]) {
  if (ACC) {
    float old[4];
    load_values(dst + c, dim - c, old);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fmaf(scale, v[j], old[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= scale;
  }
  store_values(dst + c, dim - c, v);
}

// Rows whose runs begin among the kEntries sorted entries from `first` on and hold no whole piece, at the thread's columns.
// The entries are read at once, whatever rows they belong to (a run of one would otherwise cost a row of latencies), and a
// row is written where its run ends; the last run's entries behind these follow.
template <typename T, typename O, bool ACC>
__device__ __forceinline__ void do_entries(const T* g, const int32_t* key, const int32_t* pos, int n, int vocab, int dim,
                                           float scale, const int2* runs, int shift, int first, int c, O* table) {
  const int count = min(kEntries, n - first);
  int k[kEntries], at[kEntries];
#pragma unroll
  for (int j = 0; j < kEntries; ++j) {
    k[j] = key[first + min(j, count - 1)];
    at[j] = pos[first + min(j, count - 1)];
  }
  const int before = first > 0 ? key[first - 1] : -1;
  const int final = k[kEntries - 1];
  const int end = final < vocab ? runs[final].y : n;  // of the last run
  Raw4<T> q[kEntries];
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (c < dim) q[j] = load_raw(g + (size_t)at[j] * dim + c, dim - c);
  int begin = -1, row = before;  // of the run that is being added up (none so far), and its row
  float v[4] = {};
  bool more = true;
#pragma unroll
  for (int j = 0; j < kEntries; ++j) {
    more &= j < count && k[j] < vocab;
    if (more) {
      if (k[j] != row) {
        if (begin >= 0 && c < dim) write_row<O, ACC>(table + (size_t)row * dim, dim, c, scale, v);
        begin = first + j;
        row = k[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.f;
      }
      if (c < dim) add_raw(v, q[j]);
    }
  }
  if (begin < 0) return;
  const int stop = row == final ? end : begin;  // a run before invalid ids has ended
  const Pieces r = pieces_of(make_int2(begin, stop), shift);
  if (r.p < r.q) return;
  add_rows(v, g, pos, first + count, max(stop, first + count), dim, c);
  if (c < dim) write_row<O, ACC>(table + (size_t)row * dim, dim, c, scale, v);
}

// Rows lo .. hi that have no tokens, `each` a workgroup.
struct ZeroRows {
  int lo, hi, each;
};
template <typename O>
__device__ __forceinline__ void zero_rows(const ZeroRows& z, int block, int dim, const Shape& sh, const int2* runs, O* table) {
  const float zero[4] = {};
  const int lo = z.lo + block * z.each, hi = min(lo + z.each, z.hi);
  for (int row = lo + sh.group; row < hi; row += sh.groups) {
    const int2 run = runs[row];
    if (run.y > run.x) continue;
    for (int c = sh.col; c < dim; c += 4 * sh.width) store_values(table + (size_t)row * dim + c, dim - c, zero);
  }
}

// Three kinds of workgroups in one launch, so that the sums run beside the writing of the many rows without tokens (which
// is most of the time at a large vocabulary): `pieces` slabs of sums of pieces, then `starts` slabs of rows that begin among
// some entries, and, mixed in between, `zeros` of rows without tokens.  Workgroups of pieces also list the rows that have
// them (`longs`: how many, then the first piece of each, in any order).
template <typename T, typename O, bool ACC>
__global__ __launch_bounds__(EB) void k_embedding_rows(const T* __restrict__ g, const int32_t* __restrict__ key,
                                                       const int32_t* __restrict__ pos, int n, int vocab, int dim,
                                                       float scale, const int2* __restrict__ runs, int shift, int width,
                                                       int slabs, int pieces, int starts, int zeros, ZeroRows z,
                                                       float* __restrict__ sums, int32_t* __restrict__ longs,
                                                       O* __restrict__ table) {
  __shared__ float4 lds[EB];
  const Shape sh = shape_of(width);
  const int64_t busy = pieces + starts, all = busy + zeros;
  const int b = (int)(blockIdx.x * busy / all);
  if (b == (int)((blockIdx.x + 1) * busy / all)) return zero_rows(z, blockIdx.x - b, dim, sh, runs, table);
  if (b < pieces) {
    const int p = b / slabs, c = (b % slabs) * 4 * EB + sh.col;
    if (!whole_piece(key, p, shift, n, vocab)) return;
    // the first of its run: the run does not reach back over the whole piece before
    if (threadIdx.x == 0 && b % slabs == 0 && (p == 0 || key[(p - 1) << shift] != key[p << shift]))
      longs[1 + atomicAdd(longs, 1)] = p;
    float v[4] = {};
    add_share(v, sh, g, pos, p << shift, (p + 1) << shift, dim, c);
    join_groups(v, sh, lds);
    if (sh.group == 0 && c < dim) {
      float* dst = sums + (size_t)p * dim + c;  // read again soon
      if (c + 4 <= dim)
        store16(dst, pack16(v));
      else
        for (int j = 0; c + j < dim; ++j) dst[j] = v[j];
    }
    return;
  }
  const int first = ((b - pieces) / slabs * sh.groups + sh.group) * kEntries, c = ((b - pieces) % slabs) * 4 * EB + sh.col;
  if (first < n) do_entries<T, O, ACC>(g, key, pos, n, vocab, dim, scale, runs, shift, first, c, table);
}

// Large pieces (kPiece pieces) of one id, a slab of columns a workgroup.
__global__ __launch_bounds__(EB) void k_embedding_large(const int32_t* __restrict__ key, int n, int vocab, int dim, int width,
                                                        int slabs, const float* __restrict__ sums,
                                                        float* __restrict__ large) {
  __shared__ float4 lds[EB];
  const Shape sh = shape_of(width);
  const int P = blockIdx.x / slabs, c = (blockIdx.x % slabs) * 4 * EB + sh.col, p0 = P * kPiece * kPiece;
  if (key[p0] >= vocab || key[p0] != key[p0 + kPiece * kPiece - 1]) return;
  float v[4] = {};
  add_share(v, sh, sums, nullptr, P * kPiece, P * kPiece + kPiece, dim, c);
  join_groups(v, sh, lds);
  if (sh.group == 0 && c < dim)
    for (int j = 0; j < 4 && c + j < dim; ++j) large[(size_t)P * dim + c + j] = v[j];
}

// Rows whose runs hold whole pieces, as listed: few, with much to add, so the workgroup is large and its groups share that
// out.  The workgroups from `busy` on zero rows without tokens.
template <typename T, typename O, bool ACC>
__global__ __launch_bounds__(kLongThreads) void k_embedding_long_rows(const T* __restrict__ g, const int32_t* __restrict__ key,
                                                            const int32_t* __restrict__ pos, int dim, float scale,
                                                            const int2* __restrict__ runs, int shift, int width, int slabs,
                                                            const int32_t* __restrict__ longs, int busy, ZeroRows z,
                                                            const float* __restrict__ sums, const float* __restrict__ large,
                                                            O* __restrict__ table) {
  __shared__ float4 lds[kLongThreads];
  const Shape sh = shape_of(width);
  if ((int)blockIdx.x >= busy) return zero_rows(z, blockIdx.x - busy, dim, sh, runs, table);
  const int64_t count = (int64_t)longs[0] * slabs;
  for (int64_t b = blockIdx.x; b < count; b += busy) {
    const int c = (int)(b % slabs) * 4 * EB + sh.col, row = key[longs[1 + b / slabs] << shift];
    const int2 run = runs[row];
    const Pieces r = pieces_of(run, shift);
    float v[4] = {};
    add_share(v, sh, g, pos, run.x, r.p << shift, dim, c);
    if (large && r.P < r.Q) {
      add_share(v, sh, sums, nullptr, r.p, r.P * kPiece, dim, c);
      add_share(v, sh, large, nullptr, r.P, r.Q, dim, c);
      add_share(v, sh, sums, nullptr, r.Q * kPiece, r.q, dim, c);
    } else {
      add_share(v, sh, sums, nullptr, r.p, r.q, dim, c);
    }
    add_share(v, sh, g, pos, r.q << shift, run.y, dim, c);
    join_groups(v, sh, lds);
    if (sh.group == 0 && c < dim) write_row<O, ACC>(table + (size_t)row * dim, dim, c, scale, v);
  }
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

// how the keys 0 .. vocab are sorted
struct SortPlan {
  int passes, bits, sub, tiles;
};
SortPlan sort_plan(int n, int vocab) {
  int b = 1;
  while (b < 31 && (vocab >> b)) ++b;
  SortPlan p;
  p.passes = (b + kDigitBits - 1) / kDigitBits;
  p.bits = (b + p.passes - 1) / p.passes;
  // at most kMaxTiles tiles: every workgroup of a pass reads all of their counts (at least 256 keys a wave: 8,000 x 1,000 45.9
  // instead of 42.4 us, 44,112 x 1,000 66.7 instead of 65.5; at least 64: 42.2 and 69.3)
  p.sub = std::max(128, (int)(((int64_t)n + kMaxTiles * kSortWaves - 1) / (kMaxTiles * kSortWaves) + 63) & ~63);
  p.tiles = (int)(((int64_t)n + (int64_t)p.sub * kSortWaves - 1) / ((int64_t)p.sub * kSortWaves));
  return p;
}

struct Parts {
  size_t key[2], pos[2], hist, runs, longs, sums, large, bytes;
};
Parts parts_of(int n, int vocab, int dim) {
  Parts w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  for (int i = 0; i < 2; ++i) w.key[i] = take((size_t)n * 4), w.pos[i] = take((size_t)n * 4);
  w.hist = take((size_t)kMaxTiles * kDigits * 4);
  w.runs = take((size_t)vocab * sizeof(int2));
  // sizes that no smaller n or dim exceeds, small pieces or not
  const size_t small = std::min((size_t)n, (size_t)kSmallPieceTokens);
  const size_t values = std::min((size_t)n * dim, (size_t)kSmallPieceValues);
  w.longs = take((std::max((size_t)n / kPiece, small / (kPiece / 2)) + 1) * 4);
  w.sums = take(std::max((size_t)(n / kPiece) * dim, values / (kPiece / 2)) * 4);
  w.large = take((size_t)(n / kPiece / kPiece) * dim * 4);
  w.bytes = off;
  return w;
}

// Who zeroes the rows without tokens.  The small sort's launch zeroes the whole table beside it, for few rows are then written
// twice (300 tokens into 152,064 x 3,584 fp32 414 -> 374 us at the time).  The other sort and the long rows leave most of the
// card's memory bandwidth unused for some microseconds a launch, so each of their launches zeroes about as much as fits there:
// first the sort's, from the table's end (all rows, for no one knows yet which have tokens), then that of the long rows, then the one of
// the other rows.
struct ZeroPlan {
  int rows_end, long_end;  // [0, rows_end), [rows_end, long_end), and the sort's [long_end, vocab)
};
ZeroPlan zero_plan(const EmbeddingGradArgs& a, size_t row_bytes, bool small, int launches, int pieces) {
  if (a.accumulate || small) return {0, 0};
  const auto held = [&](size_t bytes, int rows) { return (int)std::min(bytes / row_bytes, (size_t)rows); };
  ZeroPlan z;
  z.long_end = a.vocab - held(kSortFill * launches, a.vocab);
  z.rows_end = z.long_end - (pieces ? held(kLongFill, z.long_end) : 0);
  return z;
}

template <typename T, typename O, bool ACC>
void backward(hipStream_t s, const EmbeddingGradArgs& a, char* ws) {
  const Parts w = parts_of(a.n, a.vocab, a.dim);
  int32_t *key = (int32_t*)(ws + w.key[0]), *pos = (int32_t*)(ws + w.pos[0]);
  int2* runs = (int2*)(ws + w.runs);
  int32_t* longs = (int32_t*)(ws + w.longs);
  const SortPlan sp = sort_plan(a.n, a.vocab);
  const bool small = a.n <= kSmallSort;
  const int launches = small ? 1 : 2 * sp.passes, shift = piece_shift(a.n, a.dim), pieces = a.n >> shift;
  const size_t row_bytes = (size_t)a.dim * sizeof(O);
  const ZeroPlan z = zero_plan(a, row_bytes, small, launches, pieces);
  // the sort's share of the zeros, launch by launch
  char* fill_at = (char*)a.table + (ACC ? 0 : z.long_end * row_bytes);
  char* const fill_end = (char*)a.table + (ACC ? 0 : a.vocab * row_bytes);
  int left = launches;
  const auto next_fill = [&] {
    const size_t bytes = (size_t)(fill_end - fill_at) / left-- / 16 * 16;
    Fill f = {fill_at, left ? bytes : (size_t)(fill_end - fill_at), kFill};
    f.each = std::max(kFill, (f.bytes / kMaxFillBlocks + 16) / 16 * 16);
    fill_at += f.bytes;
    return f;
  };
  if (small) {
    const Fill f = next_fill();
    hipLaunchKernelGGL(k_sort_small, dim3(1 + fill_blocks(f)), dim3(kSmallThreads), 0, s, a.tokens, a.n, a.vocab, sp.passes,
                       sp.bits, key, pos, runs, longs, f);
  } else {
    uint32_t* hist = (uint32_t*)(ws + w.hist);
    for (int i = 0; i < sp.passes; ++i) {
      const int to = (sp.passes - 1 - i) & 1, from = to ^ 1;  // the last pass ends in the first pair
      const SortPass p = {i ? nullptr : a.tokens, (int32_t*)(ws + w.key[from]), (int32_t*)(ws + w.pos[from]),
                          (int32_t*)(ws + w.key[to]), (int32_t*)(ws + w.pos[to]), a.n, a.vocab, i * sp.bits, sp.bits, sp.sub};
      Fill f = next_fill();
      hipLaunchKernelGGL(k_sort_count, dim3(sp.tiles + fill_blocks(f)), dim3(EB), 0, s, p, sp.tiles, hist,
                         i ? (int2*)nullptr : runs, longs, f);
      f = next_fill();
      hipLaunchKernelGGL(k_sort_place, dim3(sp.tiles + fill_blocks(f)), dim3(EB), 0, s, p, sp.tiles, hist, f);
    }
  }
  float *sums = (float*)(ws + w.sums), *large = (float*)(ws + w.large);
  int width = 32;  // threads of a row
  while (width < EB && width * 4 < a.dim) width *= 2;
  const int slabs = (int)(((int64_t)a.dim + 4 * EB - 1) / (4 * EB));
  if (!small) hipLaunchKernelGGL(k_embedding_runs, dim3((a.n + EB - 1) / EB), dim3(EB), 0, s, key, a.n, a.vocab, runs);
  const int entries = EB / width * kEntries;  // of a workgroup
  const int64_t starts = ((int64_t)a.n + entries - 1) / entries * slabs;
  // rows without tokens: some kRowValues values a workgroup where there are many of them, and never more than kMaxRowWorkgroups,
  // with which the launch stays below 2^32 threads
  const int each = std::max({1, std::min(a.vocab / kRowWorkgroups, kRowValues / a.dim), a.vocab / kMaxRowWorkgroups + 1});
  const int zeros = (z.rows_end + each - 1) / each, long_zeros = (z.long_end - z.rows_end + each - 1) / each;
  hipLaunchKernelGGL((k_embedding_rows<T, O, ACC>), dim3((unsigned)((int64_t)pieces * slabs + starts + zeros)), dim3(EB), 0, s,
                     (const T*)a.g, key, pos, a.n, a.vocab, a.dim, a.scale, runs, shift, width, slabs, pieces * slabs,
                     (int)starts, zeros, ZeroRows{0, z.rows_end, each}, sums, longs, (O*)a.table);
  if (!pieces) return;
  // sums of sums where a run may have so many pieces that a workgroup would be long at them
  const int larges = pieces < kManyPieces ? 0 : pieces / kPiece;
  if (larges)
    hipLaunchKernelGGL(k_embedding_large, dim3(larges * slabs), dim3(EB), 0, s, key, a.n, a.vocab, a.dim, width, slabs, sums,
                       large);
  // at most as many as fit on the card beside each other; each does several rows if there are more
  const int busy = (int)std::min((int64_t)pieces * slabs, (int64_t)kLongWorkgroups);
  hipLaunchKernelGGL((k_embedding_long_rows<T, O, ACC>), dim3(busy + long_zeros), dim3(kLongThreads), 0, s, (const T*)a.g, key,
                     pos, a.dim, a.scale, runs, shift, width, slabs, longs, busy, ZeroRows{z.rows_end, z.long_end, each}, sums,
                     larges ? large : nullptr, (O*)a.table);
}

template <typename T, typename O>
void lookup(hipStream_t s, const EmbeddingArgs& a) {
  hipLaunchKernelGGL((k_embedding<T, O>), dim3(std::min(a.n, 1 << 20)), dim3(EB), 0, s, (const T*)a.table, a.vocab, a.dim,
                     a.tokens, a.n, a.scale, (O*)a.out);
}

}  // namespace

hipError_t launch_embedding(hipStream_t s, int table_dtype, int out_dtype, const EmbeddingArgs& a) {
  if (table_dtype == ROLLOUT_DTYPE_BF16)
    out_dtype == ROLLOUT_DTYPE_BF16 ? lookup<uint16_t, uint16_t>(s, a) : lookup<uint16_t, float>(s, a);
  else
    out_dtype == ROLLOUT_DTYPE_BF16 ? lookup<float, uint16_t>(s, a) : lookup<float, float>(s, a);
  return hipGetLastError();
}

size_t embedding_backward_workspace(int n, int vocab, int dim) { return parts_of(n, vocab, dim).bytes; }

hipError_t launch_embedding_backward(hipStream_t s, int grad_dtype, int table_dtype, const EmbeddingGradArgs& a, void* ws) {
  const auto run = [&](auto* g, auto* t) {
    typedef std::remove_pointer_t<decltype(g)> T;
    typedef std::remove_pointer_t<decltype(t)> O;
    a.accumulate ? backward<T, O, true>(s, a, (char*)ws) : backward<T, O, false>(s, a, (char*)ws);
  };
  float* const f = nullptr;
  uint16_t* const b = nullptr;
  if (grad_dtype == ROLLOUT_DTYPE_BF16)
    table_dtype == ROLLOUT_DTYPE_BF16 ? run(b, b) : run(b, f);
  else
    table_dtype == ROLLOUT_DTYPE_BF16 ? run(f, b) : run(f, f);
  return hipGetLastError();
}

}  // namespace rollout
