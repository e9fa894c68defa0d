// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   out_n = scale E[id_n];     dE_v = scale sum over n with id_n = v of g_n   (+ the old dE_v)
//
// The gradient sorts (id, position) pairs by id with a stable radix sort, so that a row's tokens stand together in
// token order, and sums each run in that order: no atomics on floats, the same bits on every call.  A run's length is
// anything from one to all of the tokens (text repeats its frequent ids), so runs are cut at fixed places of the sorted
// order: every 64 entries that belong to one id are summed beforehand, and every 64 such sums once more; a row then
// adds at most 63 entries, 63 sums, the sums of 4,096, 63 sums and 63 entries.
#include "update.h"

namespace rollout {
namespace {

constexpr int EB = 256;
constexpr int kPiece = 64;               // entries of a piece, and pieces of a large piece
constexpr int kAhead = 8;                // rows in flight
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortWaves = EB / 64;
constexpr int kMaxTiles = 256;
constexpr int kSmallSort = 4096, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
// N values from any element on, of which n exist
template <int N>
__device__ __forceinline__ void load_values(const float* p, int n, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    if (i + 4 <= n) {
      float q[4];
      unpack16(load16(p + i), q);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = q[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = i + j < n ? p[i + j] : 0.f;
    }
  }
}
template <int N>
__device__ __forceinline__ void load_values(const uint16_t* p, int n, float (&v)[N]) {
  static_assert(N == 8);
  if (n >= 8) {
    unpack16(load16(p), v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? bf16_to_f32(p[j]) : 0.f;
  }
}
template <int N>
__device__ __forceinline__ void store_values(float* p, int n, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    if (i + 4 <= n) {
      const float q[4] = {v[i], v[i + 1], v[i + 2], v[i + 3]};
      store16(p + i, pack16(q));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < n) p[i + j] = v[i + j];
    }
  }
}
template <int N>
__device__ __forceinline__ void store_values(uint16_t* p, int n, const float (&v)[N]) {
  static_assert(N == 8);
  if (n >= 8) {
    store16(p, pack16(v));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = round_bf16(v[j]);
  }
}

template <typename T, typename O>
__global__ __launch_bounds__(EB) void k_embedding(const T* __restrict__ table, int vocab, int dim,
                                                  const int32_t* __restrict__ tokens, int n, float scale,
                                                  O* __restrict__ out) {
  for (int row = blockIdx.x; row < n; row += gridDim.x) {
    const int id = tokens[row];
    const T* src = table + (size_t)max(0, min(id, vocab - 1)) * dim;
    O* dst = out + (size_t)row * dim;
    for (int c = threadIdx.x * 8; c < dim; c += EB * 8) {
      float v[8];
      if (id >= 0 && id < vocab) {
        load_values(src + c, dim - c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= scale;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = id < 0 ? 0.f : NAN;
      }
      store_values(dst + c, dim - c, v);
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

// Digit counts of every tile (a workgroup's keys) into hist[tile][digit].  The first pass also empties the rows' runs.
__global__ __launch_bounds__(EB) void k_sort_count(SortPass p, uint32_t* __restrict__ hist, int2* __restrict__ runs) {
  __shared__ uint32_t cnt[kDigits];
  for (int d = threadIdx.x; d < kDigits; d += EB) cnt[d] = 0;
  __syncthreads();
  const int lo = min((int64_t)blockIdx.x * p.sub * kSortWaves, (int64_t)p.n);
  const int hi = (int)min((int64_t)lo + (int64_t)p.sub * kSortWaves, (int64_t)p.n);
  const int mask = (1 << p.bits) - 1;
  for (int i = lo + threadIdx.x; i < hi; i += EB) atomicAdd(&cnt[(key_at(p, i) >> p.shift) & mask], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < kDigits; d += EB) hist[(size_t)blockIdx.x * kDigits + d] = cnt[d];
  if (runs)
    for (int v = blockIdx.x * EB + threadIdx.x; v < p.vocab; v += gridDim.x * EB) runs[v] = make_int2(0, 0);
}

__global__ __launch_bounds__(EB) void k_sort_place(SortPass p, const uint32_t* __restrict__ hist) {
  static_assert(kDigits == 2 * EB);
  __shared__ uint32_t place[kSortWaves][kDigits];
  __shared__ uint32_t total[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mask = (1 << p.bits) - 1;
  for (int i = threadIdx.x; i < kSortWaves * kDigits; i += EB) (&place[0][0])[i] = 0;
  __syncthreads();
  const int lo = (int)min(((int64_t)blockIdx.x * kSortWaves + wave) * p.sub, (int64_t)p.n);
  const int hi = (int)min((int64_t)lo + p.sub, (int64_t)p.n);
  for (int i = lo + lane; i < hi; i += 64) atomicAdd(&place[wave][(key_at(p, i) >> p.shift) & mask], 1u);
  // digits 2 t and 2 t + 1 of thread t: all counts, and those of earlier tiles
  uint32_t all[2] = {0, 0}, before[2] = {0, 0};
  const int tiles = gridDim.x;
  for (int t = 0; t < tiles; ++t) {
    const uint2 h = *reinterpret_cast<const uint2*>(hist + (size_t)t * kDigits + 2 * threadIdx.x);
    all[0] += h.x, all[1] += h.y;
    if (t < (int)blockIdx.x) before[0] += h.x, before[1] += h.y;
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
  for (int i0 = lo; i0 < hi; i0 += 64) {
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

// All passes by one workgroup, in LDS, for n up to kSmallSort; the other workgroups empty the rows' runs.
__global__ __launch_bounds__(kSmallThreads) void k_sort_small(const int32_t* __restrict__ tokens, int n, int vocab, int passes,
                                                              int bits, int32_t* __restrict__ key_out,
                                                              int32_t* __restrict__ pos_out, int2* __restrict__ runs) {
  __shared__ int32_t lds[4 * kSmallSort];  // keys and positions, of two buffers
  __shared__ uint32_t place[kSmallWaves][kDigits];
  __shared__ uint32_t total[kDigits / 64];
  if (blockIdx.x) {
    for (int v = (blockIdx.x - 1) * kSmallThreads + threadIdx.x; v < vocab; v += (gridDim.x - 1) * kSmallThreads)
      runs[v] = make_int2(0, 0);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = ((n + kSmallWaves - 1) / kSmallWaves + 63) & ~63;
  const int mask = (1 << bits) - 1;
  int32_t *key = lds, *pos = lds + n, *key2 = lds + 2 * n, *pos2 = lds + 3 * n;
  for (int i = threadIdx.x; i < n; i += kSmallThreads) key[i] = key_of_token(tokens[i], vocab), pos[i] = i;
  const int lo = min(wave * sub, n), hi = min(lo + sub, n);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int i = threadIdx.x; i < kSmallWaves * kDigits; i += kSmallThreads) (&place[0][0])[i] = 0;
    __syncthreads();
    for (int i = lo + lane; i < hi; i += 64) atomicAdd(&place[wave][(key[i] >> shift) & mask], 1u);
    __syncthreads();
    uint32_t all = 0, sum = 0;
    if (threadIdx.x < kDigits) {
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
    if (threadIdx.x < kDigits) {
      uint32_t at = sum - all;
      for (int w = 0; w < wave; ++w) at += total[w];
      for (int w = 0; w < kSmallWaves; ++w) {
        const uint32_t c = place[w][threadIdx.x];
        place[w][threadIdx.x] = at;
        at += c;
      }
    }
    __syncthreads();
    const bool done = pass == passes - 1;
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + lane;
      const bool valid = i < hi;
      const int k = valid ? key[i] : 0;
      const int to = take_place(place[wave], (k >> shift) & mask, valid, bits);
      if (valid) {
        (done ? key_out : key2)[to] = k;
        (done ? pos_out : pos2)[to] = pos[i];
      }
    }
    __syncthreads();
    int32_t* t = key;
    key = key2, key2 = t;
    t = pos, pos = pos2, pos2 = t;
  }
}

// ---------------------------------------------------------------------------
// sums of runs
// ---------------------------------------------------------------------------
// v += g rows pos[lo .. hi) at the thread's columns, in order, kAhead loads in flight
template <typename T, int N>
__device__ __forceinline__ void add_rows(float (&v)[N], const T* g, const int32_t* pos, int lo, int hi, int dim, int c) {
  for (int i = lo; i < hi; i += kAhead) {
    float q[kAhead][N];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      load_values(g + (size_t)pos[min(i + j, hi - 1)] * dim + c, dim - c, q[j]);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i + j < hi)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += q[j][k];
  }
}
// the same over rows lo .. hi of a matrix of sums
template <int N>
__device__ __forceinline__ void add_sums(float (&v)[N], const float* s, int lo, int hi, int dim, int c) {
  for (int i = lo; i < hi; i += kAhead) {
    float q[kAhead][N];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) load_values(s + (size_t)min(i + j, hi - 1) * dim + c, dim - c, q[j]);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i + j < hi)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += q[j][k];
  }
}

// Pieces of one id: their sums.  Every piece also notes where the runs of its entries begin and end.
template <typename T>
__global__ __launch_bounds__(EB) void k_embedding_pieces(const T* __restrict__ g, const int32_t* __restrict__ key,
                                                         const int32_t* __restrict__ pos, int n, int vocab, int dim,
                                                         int2* __restrict__ runs, float* __restrict__ sums) {
  const int p0 = blockIdx.x * kPiece;  // n is at most 2^31 - 4096
  if (threadIdx.x < kPiece) {
    const int i = p0 + threadIdx.x;
    if (i < n && key[i] < vocab) {
      if (i == 0 || key[i - 1] != key[i]) runs[key[i]].x = i;
      if (i == n - 1 || key[i + 1] != key[i]) runs[key[i]].y = i + 1;
    }
  }
  if (p0 + kPiece > n || key[p0] != key[p0 + kPiece - 1] || key[p0] >= vocab) return;
  for (int c = threadIdx.x * 8; c < dim; c += EB * 8) {
    float v[8] = {};
    add_rows(v, g, pos, p0, p0 + kPiece, dim, c);
    store_values(sums + (size_t)blockIdx.x * dim + c, dim - c, v);
  }
}

// Large pieces (64 pieces) of one id.
__global__ __launch_bounds__(EB) void k_embedding_large(const int32_t* __restrict__ key, int n, int vocab, int dim,
                                                        const float* __restrict__ sums, float* __restrict__ large) {
  const int p0 = blockIdx.x * kPiece * kPiece;
  if (p0 + kPiece * kPiece > n || key[p0] != key[p0 + kPiece * kPiece - 1] || key[p0] >= vocab) return;
  for (int c = threadIdx.x * 8; c < dim; c += EB * 8) {
    float v[8] = {};
    add_sums(v, sums, blockIdx.x * kPiece, blockIdx.x * kPiece + kPiece, dim, c);
    store_values(large + (size_t)blockIdx.x * dim + c, dim - c, v);
  }
}

// Rows of the table.  ACC: one workgroup per sorted entry, that does the row whose run begins there and adds to it;
// otherwise one per row, rows without tokens becoming zero.
template <typename T, typename O, bool ACC>
__global__ __launch_bounds__(EB) void k_embedding_rows(const T* __restrict__ g, const int32_t* __restrict__ key,
                                                       const int32_t* __restrict__ pos, int n, int vocab, int dim,
                                                       float scale, const int2* __restrict__ runs,
                                                       const float* __restrict__ sums, const float* __restrict__ large,
                                                       O* __restrict__ table) {
  for (int b = blockIdx.x; b < (ACC ? n : vocab); b += gridDim.x) {
    int row = b;
    if (ACC) {
      row = key[b];
      if (row >= vocab || (b > 0 && key[b - 1] == row)) continue;
    }
    const int2 run = runs[row];
    O* dst = table + (size_t)row * dim;
    // whole pieces [p, q) and whole large pieces [P, Q) of the run
    const int p = (run.x + kPiece - 1) / kPiece, q = max(run.y / kPiece, p);
    const int P = (p + kPiece - 1) / kPiece, Q = max(q / kPiece, P);
    for (int c = threadIdx.x * 8; c < dim; c += EB * 8) {
      float v[8] = {};
      if (run.y > run.x) {
        if (p < q) {
          add_rows(v, g, pos, run.x, p * kPiece, dim, c);
          if (P < Q) {
            add_sums(v, sums, p, P * kPiece, dim, c);
            add_sums(v, large, P, Q, dim, c);
            add_sums(v, sums, Q * kPiece, q, dim, c);
          } else {
            add_sums(v, sums, p, q, dim, c);
          }
          add_rows(v, g, pos, q * kPiece, run.y, dim, c);
        } else {
          add_rows(v, g, pos, run.x, run.y, dim, c);
        }
      }
      if (ACC) {
        float old[8];
        load_values(dst + c, dim - c, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(scale, v[j], old[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= scale;
      }
      store_values(dst + c, dim - c, v);
    }
  }
}

size_t align16(size_t v) { return (v + 255) / 256 * 256; }

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
  // at most kMaxTiles tiles: every workgroup of a pass reads all of their counts
  p.sub = std::max(256, (int)(((int64_t)n + kMaxTiles * kSortWaves - 1) / (kMaxTiles * kSortWaves) + 63) & ~63);
  p.tiles = (int)(((int64_t)n + (int64_t)p.sub * kSortWaves - 1) / ((int64_t)p.sub * kSortWaves));
  return p;
}

struct Parts {
  size_t key[2], pos[2], hist, runs, sums, large, bytes;
};
Parts parts_of(int n, int vocab, int dim) {
  Parts w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align16(off + bytes);
    return o;
  };
  for (int i = 0; i < 2; ++i) w.key[i] = take((size_t)n * 4), w.pos[i] = take((size_t)n * 4);
  w.hist = take((size_t)kMaxTiles * kDigits * 4);
  w.runs = take((size_t)vocab * sizeof(int2));
  w.sums = take((size_t)(n / kPiece) * dim * 4);
  w.large = take((size_t)(n / kPiece / kPiece) * dim * 4);
  w.bytes = off;
  return w;
}

template <typename T, typename O>
void backward(hipStream_t s, const EmbeddingGradArgs& a, char* ws) {
  const Parts w = parts_of(a.n, a.vocab, a.dim);
  int32_t *key = (int32_t*)(ws + w.key[0]), *pos = (int32_t*)(ws + w.pos[0]);
  int2* runs = (int2*)(ws + w.runs);
  const SortPlan sp = sort_plan(a.n, a.vocab);
  const int clear = (a.vocab + kSmallThreads * 4 - 1) / (kSmallThreads * 4);
  if (a.n <= kSmallSort) {
    hipLaunchKernelGGL(k_sort_small, dim3(1 + std::min(clear, 1024)), dim3(kSmallThreads), 0, s, a.tokens, a.n,
                       a.vocab, sp.passes, sp.bits, key, pos, runs);
  } else {
    uint32_t* hist = (uint32_t*)(ws + w.hist);
    for (int i = 0; i < sp.passes; ++i) {
      const int to = (sp.passes - 1 - i) & 1, from = to ^ 1;  // the last pass ends in the first pair
      const SortPass p = {i ? nullptr : a.tokens, (int32_t*)(ws + w.key[from]), (int32_t*)(ws + w.pos[from]),
                          (int32_t*)(ws + w.key[to]), (int32_t*)(ws + w.pos[to]), a.n, a.vocab, i * sp.bits, sp.bits, sp.sub};
      hipLaunchKernelGGL(k_sort_count, dim3(sp.tiles), dim3(EB), 0, s, p, hist, i ? (int2*)nullptr : runs);
      hipLaunchKernelGGL(k_sort_place, dim3(sp.tiles), dim3(EB), 0, s, p, hist);
    }
  }
  float *sums = (float*)(ws + w.sums), *large = (float*)(ws + w.large);
  hipLaunchKernelGGL(k_embedding_pieces<T>, dim3((a.n + kPiece - 1) / kPiece), dim3(EB), 0, s, (const T*)a.g, key, pos, a.n,
                     a.vocab, a.dim, runs, sums);
  if (a.n >= kPiece * kPiece)
    hipLaunchKernelGGL(k_embedding_large, dim3(a.n / (kPiece * kPiece)), dim3(EB), 0, s, key, a.n, a.vocab, a.dim, sums, large);
  if (a.accumulate)
    hipLaunchKernelGGL((k_embedding_rows<T, O, true>), dim3(std::min(a.n, 1 << 20)), dim3(EB), 0, s, (const T*)a.g, key, pos,
                       a.n, a.vocab, a.dim, a.scale, runs, sums, large, (O*)a.table);
  else
    hipLaunchKernelGGL((k_embedding_rows<T, O, false>), dim3(std::min(a.vocab, 1 << 20)), dim3(EB), 0, s, (const T*)a.g, key,
                       pos, a.n, a.vocab, a.dim, a.scale, runs, sums, large, (O*)a.table);
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
  if (grad_dtype == ROLLOUT_DTYPE_BF16)
    table_dtype == ROLLOUT_DTYPE_BF16 ? backward<uint16_t, uint16_t>(s, a, (char*)ws) : backward<uint16_t, float>(s, a, (char*)ws);
  else
    table_dtype == ROLLOUT_DTYPE_BF16 ? backward<float, uint16_t>(s, a, (char*)ws) : backward<float, float>(s, a, (char*)ws);
  return hipGetLastError();
}

}  // namespace rollout
