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
// c ^ swizzle(row)), so that the 16 rows of a row read and the four rows of a transposing read fall on different banks.
template <typename T, int HD>
struct Rows {
  static constexpr int kBytes = HD * (int)sizeof(T);  // of a row
  static constexpr int kChunks = kBytes / 16;
  typedef typename Operand<T>::Frag Frag;

  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (kChunks >= 16) return ((row & 7) << 1) | ((row >> 3) & 1);
    if constexpr (kChunks == 8) return ((row & 6)) | ((row >> 3) & 1);
    return (row >> 2) & 3;
  }
  // byte offset of chunk c of a row
  static __device__ __forceinline__ int at(int row, int c) { return row * kBytes + ((c ^ swizzle(row)) << 4); }

  // N rows from global memory straight into LDS, by NW waves.  src: the first row,
  // the same for the whole wave; stride in bytes; rows behind `last` (>= 0) are copies of it.
  template <int N, int NW>
  static __device__ __forceinline__ void load(char* lds, const char* src, uint32_t stride, int last, int wave, int lane) {
    constexpr int kPer = 64 / kChunks;  // rows of an instruction
    constexpr int kInstr = N * kChunks / 64;
    static_assert(N * kChunks % 64 == 0 && kChunks <= 64, "whole loads");
#pragma unroll
    for (int i = 0; i < (kInstr + NW - 1) / NW; ++i) {
      if (kInstr % NW != 0 && i * NW + wave >= kInstr) break;
      const int first = (i * NW + wave) * kPer;
      const int row = first + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
      dma_lds16_at(src, (uint32_t)min(row, last) * stride + (uint32_t)(c << 4), lds + first * kBytes);
    }
  }
};

// Reading a tile as an operand: block (32 rows from row0) as it lies (contraction over the row's values), or transposed
// (contraction over 16 of its rows).  The lane's part of the addresses is worked out once.
template <typename T, int HD>
struct RowReader {
  typedef Rows<T, HD> R;
  int base[HD / 16];
  __device__ __forceinline__ explicit RowReader(int lane) {
    const int row = row_perm(lane & 31), half = lane >> 5;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) base[c] = R::at(row, (2 * c + half) * ((int)sizeof(T) / 2));
  }
  // rows row0 + row_perm(lane % 32), values 16 c + 8 (lane / 32) + 0 .. 7
  __device__ __forceinline__ typename R::Frag operator()(const char* tile, int row0, int c) const {
    typename R::Frag f;
    const char* p = tile + row0 * R::kBytes;
    if constexpr (sizeof(T) == 2) {
      f = *reinterpret_cast<const bf16x8*>(p + base[c]);
    } else {
      const float4 lo = *reinterpret_cast<const float4*>(p + base[c]), hi = *reinterpret_cast<const float4*>(p + (base[c] ^ 16));
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
  int base[2][HD / 32];
  __device__ __forceinline__ explicit ColReader(int lane) {
    const int j = lane & 15, g = lane >> 4;
    const int q = j & 3, part = ((q & 1) << 1) | (q >> 1);  // 4-value part of the 16, in the order 0, 2, 1, 3
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = 8 * (g >> 1) + 4 * r + (j >> 2);
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) base[r][d] = R::at(row, 4 * d + 2 * (g & 1) + (part >> 1)) + 8 * (part & 1);
    }
  }
  // rows row0 + 8 (lane / 32) + 0 .. 7 (row0 a multiple of 16) of value 32 d + row_perm(lane % 32)
  __device__ __forceinline__ bf16x8 operator()(const char* tile, int row0, int d) const {
    typedef __attribute__((address_space(3))) s16x4* Lds;
    const char* p = tile + row0 * R::kBytes;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + base[0][d]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + base[1][d]));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

template <int HD>
struct ColReader<float, HD> {
  typedef Rows<float, HD> R;
  int col, half;
  __device__ __forceinline__ explicit ColReader(int lane) : col(row_perm(lane & 31)), half(lane >> 5) {}
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

// The tiles of B rows of all sequences are numbered start_s / B + s + (tile in s): no two have the same number, the numbers
// ascend with s, and there are at most n / B + n_seqs of them, so no list of tiles has to be made first.  Numbers that no
// tile has are skipped.
__host__ __device__ __forceinline__ int tile_slots(int n, int n_seqs, int B) { return n / B + n_seqs; }

// The sequence of a tile number and the tile's first row in it; false: no such tile.  64 lanes probe at a time; whatever the
// starts hold, only entries 0 .. n_seqs are read.
template <int B>
__device__ __forceinline__ bool find_tile(const int32_t* starts, const int32_t* lens, int n_seqs, int n, int slot, int lane,
                                          int* seq, Sequence* sq, int* row) {
  int lo = 0, hi = n_seqs;
  do {
    const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
    const bool before = s < hi && max(0, min(starts[s], n)) / B + s <= slot;
    const int k = __popcll(__ballot(before)) - 1;
    if (k < 0) return false;
    lo += k * step;
    hi = min(lo + step, hi);
  } while (hi - lo > 1);
  *seq = __builtin_amdgcn_readfirstlane(lo);
  *sq = sequence_at(starts, lens, *seq, n);
  *row = (slot - (sq->start / B + *seq)) * B;
  return *row >= 0 && *row < sq->len;
}

// Workgroups are dealt out to the eight dies in turn; numbered so that a die's are neighbours.  -1: none.
__device__ __forceinline__ int neighbours_on_die(int total) {
  const int per = (total + 7) >> 3;
  const int w = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  return (int)(blockIdx.x >> 3) < per && w < total ? w : -1;
}
inline unsigned die_grid(int total) { return (unsigned)((total + 7) / 8 * 8); }

}  // namespace rollout
