// Argument checks that the entry points of the update side share.
#pragma once

#include "update.h"

#include <cmath>
#include <initializer_list>
#include <string>

#include <rocprofiler-sdk-roctx/roctx.h>

namespace rollout {

struct Range {
  explicit Range(const char* name) { roctxRangePush(name); }
  ~Range() { roctxRangePop(); }
  Range(const Range&) = delete;
  Range& operator=(const Range&) = delete;
};

inline rollout_status fail(rollout_status st, const std::string& msg) {
  set_last_error(msg);
  return st;
}

inline bool is_float_type(int32_t dtype) { return dtype == ROLLOUT_DTYPE_FP32 || dtype == ROLLOUT_DTYPE_BF16; }
inline bool aligned_to(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

// [a, a + a_bytes) and [b, b + b_bytes) share a byte
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + b_bytes && y < x + a_bytes;
}

// [p, p + bytes) shares a byte with one of `rows` rows of row_bytes that are stride bytes apart (at least row_bytes): what lies
// between the rows is not theirs
inline bool overlap_rows(const void* base, size_t rows, size_t stride, size_t row_bytes, const void* p, size_t bytes) {
  const int64_t lo = (int64_t)((uintptr_t)p - (uintptr_t)base), hi = lo + (int64_t)bytes;
  const int64_t r = lo < (int64_t)row_bytes ? 0 : (lo - (int64_t)row_bytes) / (int64_t)stride + 1;  // the first that ends behind lo
  return r < (int64_t)rows && r * (int64_t)stride < hi;
}

// A buffer of a call, or (rows > 1) a matrix of rows that are stride bytes apart; NULL: absent.
struct Span {
  const char* name;
  const void* p;
  size_t bytes, rows = 1, stride = 0;
};

// Two matrices of rows: exactly where their rows are equally far apart (the columns of one buffer); with other strides, from
// first to last row.
inline bool overlap_matrices(const Span& a, const Span& b) {
  if (a.stride != b.stride) return overlap(a.p, (a.rows - 1) * a.stride + a.bytes, b.p, (b.rows - 1) * b.stride + b.bytes);
  const int64_t s = (int64_t)a.stride, d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p), wa = (int64_t)a.bytes, wb = (int64_t)b.bytes;
  // row i of a and row i + k of b: -wb < d + k s < wa
  const int64_t x = -wb - d;
  for (int64_t k = (x >= 0 ? x / s : -((-x + s - 1) / s)) + 1; d + k * s < wa; ++k)
    if (k > -(int64_t)a.rows && k < (int64_t)b.rows) return true;
  return false;
}

inline bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
  if (a.rows > 1 && b.rows > 1) return overlap_matrices(a, b);
  if (a.rows > 1) return overlap_rows(a.p, a.rows, a.stride, a.bytes, b.p, b.bytes);
  if (b.rows > 1) return overlap_rows(b.p, b.rows, b.stride, b.bytes, a.p, a.bytes);
  return overlap(a.p, a.bytes, b.p, b.bytes);
}

// Kernels read a call's inputs while other workgroups write its outputs and the workspace: all of them stand apart.
inline rollout_status check_apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span& i : ins)
      if (overlap(*o, i)) return fail(ROLLOUT_EINVAL, std::string(o->name) + " overlaps an input, " + i.name);
    for (const Span* q = outs.begin(); q != o; ++q)
      if (overlap(*o, *q)) return fail(ROLLOUT_EINVAL, std::string(o->name) + " overlaps " + q->name);
  }
  return ROLLOUT_OK;
}

// fp32 and int32 buffers
inline rollout_status check_words(std::initializer_list<const void*> buffers) {
  for (const void* p : buffers)
    if (!aligned_to(p, 4)) return fail(ROLLOUT_EINVAL, "an fp32 or int32 buffer is not aligned to 4 bytes");
  return ROLLOUT_OK;
}

// the stream (NULL: the default one) belongs to the current device
inline rollout_status check_stream(void* hip_stream) {
  int dev = -1, sdev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(ROLLOUT_EDEVICE, std::string("hipGetDevice: ") + hipGetErrorString(e));
  if (!hip_stream) return ROLLOUT_OK;
  e = hipStreamGetDevice((hipStream_t)hip_stream, &sdev);
  if (e != hipSuccess) return fail(ROLLOUT_EDEVICE, std::string("hipStreamGetDevice: ") + hipGetErrorString(e));
  if (sdev != dev) return fail(ROLLOUT_EINVAL, "the stream belongs to another device than the current one");
  return ROLLOUT_OK;
}

inline rollout_status check_workspace(const void* ws, uint64_t bytes, size_t need) {
  if (bytes < need)
    return fail(ROLLOUT_ENOMEM, "workspace of " + std::to_string(bytes) + " bytes; the call needs " + std::to_string(need));
  if (need && !ws) return fail(ROLLOUT_EINVAL, "the workspace is NULL");
  if (need && !aligned_to(ws, 16)) return fail(ROLLOUT_EINVAL, "the workspace must be aligned to 16 bytes");
  return ROLLOUT_OK;
}

inline rollout_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(ROLLOUT_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
  return ROLLOUT_OK;
}

}  // namespace rollout
