// What the kernels of packed attention and of its gradient share: where a workgroup's tile lies, tiles of rows in LDS, and
// the matrix products over them.
//
// A product of two 32 x 32 blocks is v_mfma_f32_32x32x16_bf16 or eight times v_mfma_f32_32x32x2_f32.  Both take eight values
// per lane of each operand, row (A) or column (B) lane % 32, and for bf16 the contraction index 8 (lane / 32) + 0 .. 7; for
// fp32 instruction i takes the ith of them, so that the same eight stand for the same indices.  The result has column
// lane % 32, and in register e the row 8 (e / 4) + 4 (lane / 32) + e % 4.  Where a block's rows are handed over in the order
// of row_perm, register e holds row 16 (e / 8) + 8 (lane / 32) + e % 8 instead: eight neighbours, which are the B operand of
// the next product over these rows and 16 bytes of an output.
#pragma once

#include "update.h"

namespace rollout {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

__device__ __forceinline__ int row_perm(int a) { return (a & ~12) | ((a & 4) << 1) | ((a & 8) >> 1); }

template <typename T>
struct Operand;
template <>
struct Operand<uint16_t> {
  typedef bf16x8 Frag;
};
template <>
struct Operand<float> {
  typedef f32x8 Frag;
};

__device__ __forceinline__ void mma(const bf16x8& a, const bf16x8& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(const f32x8& a, const f32x8& b, f32x16& c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
}

__device__ __forceinline__ void clear(f32x16& c) {
#pragma unroll
  for (int e = 0; e < 16; ++e) c[e] = 0.f;
}

// registers 8 i .. 8 i + 7 of a result as an operand; bf16 rounds to nearest
__device__ __forceinline__ void operand_of(const f32x16& c, int i, bf16x8& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (__bf16)c[8 * i + e];
}
__device__ __forceinline__ void operand_of(const f32x16& c, int i, f32x8& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = c[8 * i + e];
}

// What operand_of's rounding took from b: with kTwice a product a b takes it as well.  Without it results are farther off than
// those that are rounded once: outputs 1.05 (2 keys) to 1.35 times (900), gradients 1.4 times whatever the number of keys, as a root
// mean square; in calls of few pairs of a query and a key, by the luck of few roundings, 1.0 to 2.8 times (gradients; emulated calls
// of four heads).  There the second product is in nobody's way, and they are as near as those so (three queries of 68 keys, gradient,
// 16 us with and without); in larger ones it costs more than it gives (one query of 768 keys at 28 heads, gradient, 21 us, so 23; 16 x
// 500 to 2,000 tokens at four heads of 32 32 us, so 44).  The rule is one on the call, by its allocated rows: a sequence that is called
// with many others has other last bits than alone.
inline bool few_pairs(const AttentionArgs& a) { return (double)a.n_q * a.heads * ((double)a.n_k / a.n_seqs) <= 16384.0; }
__device__ __forceinline__ void rest_of(const f32x16& c, int i, const bf16x8& f, bf16x8& rest) {
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = (__bf16)(c[8 * i + e] - (float)f[e]);
}
__device__ __forceinline__ void rest_of(const f32x16&, int, const f32x8&, f32x8&) {}

// eight neighbours of an output row (aligned to 16 bytes)
__device__ __forceinline__ void store8(uint16_t* p, const f32x16& c, int i, float by) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c[8 * i + e] * by;
  *reinterpret_cast<u32x4*>(p) = pack16(v);
}
__device__ __forceinline__ void store8(float* p, const f32x16& c, int i, float by) {
  float4 lo, hi;
  lo.x = c[8 * i] * by, lo.y = c[8 * i + 1] * by, lo.z = c[8 * i + 2] * by, lo.w = c[8 * i + 3] * by;
  hi.x = c[8 * i + 4] * by, hi.y = c[8 * i + 5] * by, hi.z = c[8 * i + 6] * by, hi.w = c[8 * i + 7] * by;
  reinterpret_cast<float4*>(p)[0] = lo;
  reinterpret_cast<float4*>(p)[1] = hi;
}

// A run of rows in LDS, HD values each, without gaps.  The 16-byte chunks of a row stand in an order of its own (chunk c at
// c ^ swizzle(row)): the 16 rows that a row read takes at a time differ in it, and the four rows of two neighbouring transposing
// reads fall on banks of their own (conflicts counted in the keys' gradients: none).
template <typename T, int HD>
struct Rows {
  static constexpr int kBytes = HD * (int)sizeof(T);  // of a row
  static constexpr int kChunks = kBytes / 16;
  typedef typename Operand<T>::Frag Frag;

  static __host__ __device__ constexpr int swizzle(int row) {
    if constexpr (kChunks >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    if constexpr (kChunks == 8) return ((row & 2) << 1) | ((row >> 2) & 3);
    return (row >> 2) & 3;
  }
  // byte offset of chunk c of a row
  static __device__ __forceinline__ int at(int row, int c) { return row * kBytes + ((c ^ swizzle(row)) << 4); }

  // N rows dealt out to loads of NW waves.  issue(row, offset, place): the row that the lane has 16 bytes of, at `offset` of it,
  // and the bytes behind the tile's beginning where the wave's lie, the lane's 16 lane bytes behind that.
  template <int N, int NW, typename F>
  static __device__ __forceinline__ void load_with(int wave, int lane, F issue) {
    constexpr int kPer = 64 / kChunks;  // rows of an instruction
    constexpr int kInstr = N * kChunks / 64;
    static_assert(N * kChunks % 64 == 0 && kChunks <= 64, "whole loads");
#pragma unroll
    for (int i = 0; i < (kInstr + NW - 1) / NW; ++i) {
      if (kInstr % NW != 0 && i * NW + wave >= kInstr) break;
      const int first = (i * NW + wave) * kPer;
      const int row = first + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
      issue(row, (uint32_t)(c << 4), first * kBytes);
    }
  }
  // src: the first row, the same for the whole wave; stride in bytes; rows behind `last` (>= 0) are copies of it.
  template <int N, int NW>
  static __device__ __forceinline__ void load(char* lds, const char* src, uint32_t stride, int last, int wave, int lane) {
    load_with<N, NW>(wave, lane, [&](int row, uint32_t offset, int place) {
      dma_lds16_at(src, (uint32_t)min(row, last) * stride + offset, lds + place);
    });
  }
};

// Reading a tile as an operand: block (32 rows from row0) as it lies (contraction over the row's values), or transposed
// (contraction over 16 of its rows).  The swizzle makes an address the lane's own part with constants exclusive-ored into it:
// one instruction for each of them and no register kept, where registers are what is short (`renew`, once a tile, hides the
// part's origin from the compiler, which would otherwise keep them all).
template <typename T, int HD>
struct RowReader {
  typedef Rows<T, HD> R;
  int base;
  __device__ __forceinline__ explicit RowReader(int lane) : base(R::at(row_perm(lane & 31), (lane >> 5) * ((int)sizeof(T) / 2))) {}
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(base)); }
  // rows row0 + row_perm(lane % 32), values 16 c + 8 (lane / 32) + 0 .. 7
  __device__ __forceinline__ typename R::Frag operator()(const char* tile, int row0, int c) const {
    typename R::Frag f;
    const char* p = tile + row0 * R::kBytes;
    const int at = base ^ (c * 16 * (int)sizeof(T));
    if constexpr (sizeof(T) == 2) {
      f = *reinterpret_cast<const bf16x8*>(p + at);
    } else {
      const float4 lo = *reinterpret_cast<const float4*>(p + at), hi = *reinterpret_cast<const float4*>(p + (at ^ 16));
      f[0] = lo.x, f[1] = lo.y, f[2] = lo.z, f[3] = lo.w, f[4] = hi.x, f[5] = hi.y, f[6] = hi.z, f[7] = hi.w;
    }
    return f;
  }
};

template <typename T, int HD>
struct ColReader;

// A group of 16 lanes reads four rows of 16 values with the transposing load: lane j gives the address of four values of row
// j / 4, and gets value j of each row.  Values are asked for in the order of row_perm.
template <int HD>
struct ColReader<uint16_t, HD> {
  typedef Rows<uint16_t, HD> R;
  static constexpr int kFour = (R::swizzle(4) ^ R::swizzle(0)) << 4;  // how the swizzle of rows 4 .. 7 differs from that of 0 .. 3
  int base;
  __device__ __forceinline__ explicit ColReader(int lane) {
    const int j = lane & 15, g = lane >> 4;
    const int q = j & 3, part = ((q & 1) << 1) | (q >> 1);  // 4-value part of the 16, in the order 0, 2, 1, 3
    base = R::at(8 * (g >> 1) + (j >> 2), 2 * (g & 1) + (part >> 1)) + 8 * (part & 1);
  }
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(base)); }
  // rows row0 + 8 (lane / 32) + 0 .. 7 (row0 a multiple of 16) of value 32 d + row_perm(lane % 32)
  __device__ __forceinline__ bf16x8 operator()(const char* tile, int row0, int d) const {
    typedef __attribute__((address_space(3))) s16x4* Lds;
    const char* p = tile + row0 * R::kBytes;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + (base ^ (d << 6))));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * R::kBytes + (base ^ (d << 6) ^ kFour)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

template <int HD>
struct ColReader<float, HD> {
  typedef Rows<float, HD> R;
  int col, half;
  __device__ __forceinline__ explicit ColReader(int lane) : col(row_perm(lane & 31)), half(lane >> 5) {}
  __device__ __forceinline__ void renew() {}
  __device__ __forceinline__ f32x8 operator()(const char* tile, int row0, int d) const {
    f32x8 f;
    const int c = 32 * d + col;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[e] = *reinterpret_cast<const float*>(tile + row0 * R::kBytes + R::at(8 * half + e, c >> 2) + 4 * (c & 3));
    return f;
  }
};

// eight values of a row in global memory as an operand
__device__ __forceinline__ bf16x8 load_operand(const uint16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ f32x8 load_operand(const float* p) {
  const float4 lo = reinterpret_cast<const float4*>(p)[0], hi = reinterpret_cast<const float4*>(p)[1];
  f32x8 f;
  f[0] = lo.x, f[1] = lo.y, f[2] = lo.z, f[3] = lo.w, f[4] = hi.x, f[5] = hi.y, f[6] = hi.z, f[7] = hi.w;
  return f;
}

// Sequence s of a packed matrix of n rows: first row and length.
struct Sequence {
  int start, len;
};
__device__ __forceinline__ Sequence sequence_at(const int32_t* starts, const int32_t* lens, int s, int n) {
  const int a = max(0, min(starts[s], n)), b = max(a, min(starts[s + 1], n));
  return {a, lens ? max(0, min(lens[s], b - a)) : b - a};
}

// How many query heads share a key's, and division by it: x / each = x inverse / 2^32 for x < 2^26, each <= 64.  (What a
// workgroup works out before its first tile is as much as some tiles take: few divisions, none of them in 64 bits.)
struct Group {
  int each;
  uint32_t inverse;
  __device__ __forceinline__ int tokens(int rows) const { return each == 1 ? rows : (int)__umulhi((uint32_t)rows, inverse); }
};
inline Group group_of(const AttentionArgs& a) {
  const int each = a.heads / a.kv_heads;
  return {each, (uint32_t)(((uint64_t)1 << 32) / (uint64_t)each + 1)};
}

// The query heads that share a key's are taken together: `each` of them make as many rows of a token, and a sequence of len
// tokens is a run of len * each rows (token by token).  The tiles of B rows of all sequences are numbered
// start_s * each / B + s + (tile in s): no two have the same number, the numbers ascend with s, and there are at most
// n * each / B + n_seqs of them, so no list of tiles has to be made first.  Numbers that no tile has are skipped.
__host__ __device__ __forceinline__ int tile_slots(int n, int each, int n_seqs, int B) { return n * each / B + n_seqs; }

// A tile of one side's rows (`mine`, with `each` rows a token): its sequence, there and on the other side, and its first row.
struct Place {
  Sequence mine, other;
  int row;
};
struct Side {
  const int32_t *starts, *lens;
  int n;
};
__device__ __forceinline__ Side queries_of(const AttentionArgs& A) { return {A.q_starts, A.q_lens, A.n_q}; }
__device__ __forceinline__ Side keys_of(const AttentionArgs& A) { return {A.k_starts, A.k_lens, A.n_k}; }

// false: no tile has the number.  64 lanes probe at a time, each with all that there is to know of its sequence, so that the last
// probe's answer is at hand without another trip to memory.  Whatever the starts hold, only entries 0 .. n_seqs are read.
template <int B>
__device__ __forceinline__ bool find_tile(const Side& mine, const Side& other, int n_seqs, int each, int slot, int lane, Place* p) {
  int lo = 0, hi = n_seqs;
  for (;;) {
    const int step = (hi - lo + 63) >> 6, at = lo + lane * step, s = min(at, hi - 1);
    const Sequence x = sequence_at(mine.starts, mine.lens, s, mine.n), y = sequence_at(other.starts, other.lens, s, other.n);
    const int first = (int)((uint32_t)(x.start * each) / B) + s;
    const int k = __popcll(__ballot(at < hi && first <= slot)) - 1;
    if (k < 0) return false;
    if (step == 1) {
      p->mine = {__builtin_amdgcn_readlane(x.start, k), __builtin_amdgcn_readlane(x.len, k)};
      p->other = {__builtin_amdgcn_readlane(y.start, k), __builtin_amdgcn_readlane(y.len, k)};
      p->row = (slot - __builtin_amdgcn_readlane(first, k)) * B;
      return p->row >= 0 && p->row < p->mine.len * each;
    }
    lo += k * step;
    hi = min(lo + step, hi);
  }
}

// A wave's 32 rows of a sequence from row `first` on (n_rows of them in all), a row being a token's values of one of the `each`
// heads that share a key's.  They come and go through LDS, whole rows at a time: lanes that read and wrote their own row, 16 bytes
// of it with each instruction, would touch 32 lines with every one.
template <typename T, int HD>
struct WaveRows {
  typedef Rows<T, HD> R;
  int token, over, last;  // of the first row, the heads before it there, and the last row (< 32; rows behind it are copies of it)
  Group group;
  __device__ __forceinline__ WaveRows(int first, int n_rows, const Group& g)
      : token(g.tokens(first)), over(first - token * g.each), last(min(31, n_rows - 1 - first)), group(g) {}
  // where row i lies behind the first token's first head, for tokens `stride` bytes apart
  __device__ __forceinline__ uint32_t offset(int i, uint32_t stride) const {
    const int x = i + over, t = group.tokens(x);
    return (uint32_t)t * stride + (uint32_t)(x - t * group.each) * R::kBytes;
  }
  // into the wave's 32 rows of LDS; p: the sequence's first token, at the first of the heads
  __device__ __forceinline__ void load(char* lds, const T* p, int64_t stride, int lane) const {
    const char* base = (const char*)(p + (size_t)token * stride);
    R::template load_with<32, 1>(0, lane, [&](int row, uint32_t at, int place) {
      dma_lds16_at(base, offset(min(row, last), (uint32_t)(stride * sizeof(T))) + at, lds + place);
    });
  }
  // lane's row as an operand, once it is there
  static __device__ __forceinline__ typename R::Frag operand(const char* lds, int lane, int c) {
    const char* p = lds + R::at(lane & 31, (2 * c + (lane >> 5)) * ((int)sizeof(T) / 2));
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const bf16x8*>(p);
    } else {
      const float4 lo = *reinterpret_cast<const float4*>(p);
      const float4 hi = *reinterpret_cast<const float4*>(lds + R::at(lane & 31, (2 * c + (lane >> 5)) * 2 + 1));
      return f32x8{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    }
  }
  // results with a row per lane, `by` times, through the wave's 32 rows of LDS
  __device__ __forceinline__ void store(char* lds, const f32x16 (&o)[HD / 32], float by, T* p, int64_t stride, int lane) const {
    const int a = lane & 31, half = lane >> 5;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = (4 * d + 2 * i + half) * ((int)sizeof(T) / 2);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = o[d][8 * i + e] * by;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x4*>(lds + R::at(a, c)) = pack16(v);
        } else {
          *reinterpret_cast<float4*>(lds + R::at(a, c)) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(lds + R::at(a, c + 1)) = make_float4(v[4], v[5], v[6], v[7]);
        }
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    char* base = (char*)(p + (size_t)token * stride);
    R::template load_with<32, 1>(0, lane, [&](int row, uint32_t at, int place) {
      if (row > last) return;
      *reinterpret_cast<u32x4*>(base + offset(row, (uint32_t)(stride * sizeof(T))) + at) = *reinterpret_cast<const u32x4*>(lds + place + 16 * lane);
    });
  }
};

// Tiles 0 .. n - 1 pass through two buffers in LDS: while one is worked on, the next is on the way.  load(buffer, tile) issues a
// tile's loads, step(buffer, tile) works on it.  The buffer is a compile-time number, so that it is part of the LDS
// instructions' offsets.  first_tile comes before what else a workgroup has to read.  (Three buffers of half a tile, two of them
// on the way, took the 14B gradient of 8,192 tokens from 2,204 to 2,240 us: a tile's products take longer than its way.)
template <int B, typename Load, typename Step>
__device__ __forceinline__ bool one_tile(int it, int n, Load& load, Step& step) {
  if (it >= n) return false;
  dma_wait_barrier<0>();  // the tile is there for every wave, and nobody reads the one before it any more
  if (it + 1 < n) load(std::integral_constant<int, 1 - B>(), it + 1);
  step(std::integral_constant<int, B>(), it);
  return true;
}
template <typename Load>
__device__ __forceinline__ void first_tile(int n, Load& load) {
  if (n > 0) load(std::integral_constant<int, 0>(), 0);
}
template <typename Load, typename Step>
__device__ __forceinline__ void through_tiles(int n, Load& load, Step step) {
  for (int it = 0; one_tile<0>(it, n, load, step) && one_tile<1>(it + 1, n, load, step); it += 2) {
  }
}

// N groups of W operands from LDS, each group's loads on the way while the products of the one before it run.  load(g, f) reads
// group g, use(g, f) multiplies by it; the first group may have been read before (read_ahead).  Left to itself the compiler
// reads every operand into the same registers just before its product, whose time then is that of the read.
// (of products and memory; other VALU and SALU may move)
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x6); }
template <int N, int W, int g, typename Frag, typename Load, typename Use>
__device__ __forceinline__ void group(Frag (&f)[2][W], Load& load, Use& use) {
  if constexpr (g + 1 < N) load(std::integral_constant<int, g + 1>(), f[(g + 1) & 1]);
  keep_order();
  use(std::integral_constant<int, g>(), f[g & 1]);
  keep_order();
  if constexpr (g + 1 < N) group<N, W, g + 1>(f, load, use);
}
template <int N, int W, typename Frag, typename Load, typename Use>
__device__ __forceinline__ void groups(Frag (&f)[2][W], Load load, Use use) {
  group<N, W, 0>(f, load, use);
}

// A workgroup's walk: a number of a tile, and the part of it, for a key's head.  Workgroups are dealt out to the eight dies in
// turn, and each die has its own cache: a die takes whole runs (the walks of a head, or of a head's part) as far as they can be
// shared out evenly, and of the others every die (or every die of two or four) takes walks in turn, so that each has as many
// long ones.  Walks of a run: its tiles, with their parts beside each other (kParts) or of one part alone.  false: none.
// (Heads to dies one by one left some dies with the long walks: fp32 at the 7B heads 889 us, so 716.)
struct Walk {
  int slot, part, kvh;
};
template <bool kParts>
__host__ __device__ __forceinline__ void walk_runs(int slots, int parts, int kv_heads, uint32_t* length, uint32_t* runs, uint32_t* whole,
                                                   uint32_t* rest) {
  *length = (uint32_t)(kParts ? slots * parts : slots);
  *runs = (uint32_t)(kParts ? kv_heads : kv_heads * parts);
  *whole = *runs / 8 * *length;                  // walks of a die in whole runs
  *rest = (*runs % 8 * *length + 7) / 8;         // in the others, at most
  if (*runs % 8 == 1 || *runs % 8 == 2 || *runs % 8 == 4) *rest = (*length + 8 / (*runs % 8) - 1) / (8 / (*runs % 8));
}
template <bool kParts>
__device__ __forceinline__ bool find_walk(int slots, int parts, int kv_heads, Walk* w) {
  uint32_t length, runs, whole, rest;
  walk_runs<kParts>(slots, parts, kv_heads, &length, &runs, &whole, &rest);
  const uint32_t die = blockIdx.x & 7, mine = blockIdx.x >> 3, left = runs & 7;
  uint32_t run, at;
  if (mine < whole) {
    const uint32_t k = mine / length;
    run = 8 * k + die, at = mine - k * length;
  } else if (left == 1 || left == 2 || left == 4) {
    const uint32_t dies = 8 / left;  // of a run
    run = runs - left + die / dies, at = (mine - whole) * dies + die % dies;
    if (at >= length) return false;
  } else {
    const uint32_t i = (mine - whole) * 8 + die, k = i / length;
    if (k >= left) return false;
    run = runs - left + k, at = i - k * length;
  }
  const uint32_t k = parts == 1 ? (kParts ? at : run) : (kParts ? at : run) / (uint32_t)parts;
  w->part = (int)((kParts ? at : run) - k * (uint32_t)parts);
  w->slot = (int)(kParts ? k : at), w->kvh = (int)(kParts ? run : k);
  return true;
}
template <bool kParts>
inline unsigned walk_grid(int slots, int parts, int kv_heads) {
  uint32_t length, runs, whole, rest;
  walk_runs<kParts>(slots, parts, kv_heads, &length, &runs, &whole, &rest);
  return 8 * (whole + rest);
}
// the share of a part of n tiles: n parts is less than 2^31
__device__ __forceinline__ int part_from(int n, int part, int parts) { return parts == 1 ? n * part : (int)((uint32_t)(n * part) / (uint32_t)parts); }

// Into how many parts the walks of a launch over `tiles` tiles each are cut, whose sums a second launch joins: by what a whole
// walk takes (alone_us a tile, or shared_us a tile in every one of the card's 512 places where there are more walks than
// places), the third of a walk that the last ones run on, and the parts' sums, which are written and read again.  The constants
// are fitted to sweeps of the parts at a dozen shapes, and the choice is within 3% of the best there (with and without parts: 72B's
// one token 70 and 149 us, 7B gradient 228 and 256, 1,024 tokens' gradient 89 and 264, 14B gradient 2,127 and 2,325).
// No more parts than their sums have room for: the workspace of a large call has to do for small ones, which have more parts, so
// it goes by the size of a part's sums alone.
constexpr int kMaxParts = 64;
constexpr uint64_t kPartsRoom = 256ull << 20;
inline uint64_t parts_room(uint64_t part_bytes) { return std::min(kMaxParts * part_bytes, kPartsRoom); }
struct WalkCost {
  double alone_us, shared_us;
  double least;  // tiles of a part (one query of 1,024 to 4,096 keys, gradient: 38 us with 3, 40 with 4, 42 with 2)
};
// bf16: as measured with 128 dimensions, and 0.7 and 0.55 of that with 64 and 32 (the gradient of 2 x 500 to 1,500 tokens at 16 heads
// of 64 63 us, at 1.0 of it 72, of 4 x 500 to 1,000 at 14 on 2 heads 56 and 66).  fp32: a product of 32 x 32 x 2 values takes 64
// cycles, and those are all that counts (one token over 500 to 1,000 keys 28 us, with bf16's figures 77).
template <typename T>
inline WalkCost walk_cost(double alone_us, double shared_us, int products, int head_dim) {
  if (sizeof(T) == 2) {
    const double share = head_dim == 128 ? 1.0 : head_dim == 64 ? 0.7 : 0.55;
    return {share * alone_us, share * shared_us, 3.0};
  }
  const double us = products * head_dim / 2 * 64 / 2400.0;
  return {us, 2.0 * us, 1.0};
}
inline int walk_parts(int64_t walks, double tiles, bool triangle, const WalkCost& each, uint64_t part_bytes) {
  const double places = 512.0, all = (triangle ? 0.55 : 1.0) * (double)walks * tiles * each.shared_us / places;
  const int most = (int)std::max<uint64_t>(1, parts_room(part_bytes) / part_bytes);
  int best = 1;
  double least = 0.0;
  for (int p = 1; p <= most && (p == 1 || tiles >= each.least * p); ++p) {
    const double walk = each.alone_us * tiles / p + 3.0;
    const double cost = std::max(walk, all) + 0.35 * walk + (p > 1 ? 5.0 + 2.0 * p * (double)part_bytes / 4.5e6 : 0.0);
    if (p == 1 || cost < least) best = p, least = cost;
  }
  return best;
}

}  // namespace rollout
