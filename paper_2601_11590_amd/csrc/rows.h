// Rows of operators that read or write them eight elements at a time, 16 bytes (fp32: 32).  Rows need not start on 16 bytes: gfx950
// takes accesses of any alignment, so odd lengths and strides run the same kernels, and only a row's last eight are taken one by one.
#pragma once

#include "op_error.h"

namespace epd {

typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t quad2;          // 16 bytes on any even address
typedef __attribute__((ext_vector_type(4), aligned(4))) float quad4;
typedef __attribute__((ext_vector_type(2), aligned(1))) uint32_t pair1;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16v8;

// elements [0, left) of p, left > 0; zeros beyond
__device__ __forceinline__ void load8(const __bf16* p, int left, float* v) {
  if (left >= 8) {
    const bf16v8 u = __builtin_bit_cast(bf16v8, *(const quad2*)p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)u[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int left, float* v) {
  if (left >= 8) {
    const quad4 a = *(const quad4*)p, b = *(const quad4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void store8(__bf16* p, int left, const float* v) {
  if (left >= 8) {
    bf16v8 u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = (__bf16)v[i];
    *(quad2*)p = __builtin_bit_cast(quad2, u);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = (__bf16)v[i];
  }
}
__device__ __forceinline__ void store8(float* p, int left, const float* v) {
  if (left >= 8) {
    quad4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
    *(quad4*)p = a; *(quad4*)(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = v[i];
  }
}

// The same in two steps, for loads ahead of their use: eight elements as they lie in memory, and what they stand for.
struct Raw8bf { bf16v8 v; };
struct Raw8f { quad4 a, b; };
template <typename T> struct raw8_of;
template <> struct raw8_of<__bf16> { typedef Raw8bf type; };
template <> struct raw8_of<float> { typedef Raw8f type; };
__device__ __forceinline__ void load_raw8(const __bf16* p, int left, Raw8bf& r) {
  if (left >= 8) {
    r.v = __builtin_bit_cast(bf16v8, *(const quad2*)p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < left ? p[i] : (__bf16)0.f;
  }
}
__device__ __forceinline__ void load_raw8(const float* p, int left, Raw8f& r) {
  if (left >= 8) {
    r.a = *(const quad4*)p; r.b = *(const quad4*)(p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.a[i] = i < left ? p[i] : 0.f; r.b[i] = 4 + i < left ? p[4 + i] : 0.f; }
  }
}
__device__ __forceinline__ void from_raw8(const Raw8bf& r, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)r.v[i];
}
__device__ __forceinline__ void from_raw8(const Raw8f& r, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
}

// 16 bytes written through to memory.  What stays dirty in the chip's 32 MB of L2 is written back when the kernel ends, and whoever comes next
// waits for it; written through, it leaves meanwhile.  Only for stores whose waves fill whole lines (128 bytes): halves of lines go out twice (a
// norm with fp32 rows, two stores each, took 1.8 times as long, bf16 rows of 1153 1.1 times).
__device__ __forceinline__ void store16_through(void* p, quad2 v) {
  typedef __attribute__((ext_vector_type(4))) uint32_t quad;
  __builtin_amdgcn_global_store_b128((__attribute__((address_space(1))) quad*)p, quad{v[0], v[1], v[2], v[3]}, "");
}
// As store8, through where writes_through says so: rows of bf16 in whole lines.
template <typename T> __device__ __forceinline__ void store8(T* p, int left, const float* v, bool through) {
  if constexpr (sizeof(T) == 2) {
    if (through && left >= 8) {
      bf16v8 u;
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = (__bf16)v[i];
      store16_through(p, __builtin_bit_cast(quad2, u));
      return;
    }
  }
  store8(p, left, v);
}
inline bool writes_through(const void* p, int64_t ld, int elem) { return elem == 2 && (uintptr_t)p % 128 == 0 && ld % 64 == 0; }

constexpr int64_t kMaxStride = 1ll << 40;

inline bool known_dtype(int dtype) { return dtype == EPD_F32 || dtype == EPD_BF16; }

// Rows of `cols` elements, `ld` apart; that of a single row is not looked at.
inline epd_status check_rows(const char* who, const char* name, const void* p, int64_t& ld, int64_t rows, int cols, int elem) {
  if (rows == 1) ld = cols;
  if (!p) return op_fail(EPD_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  if (ld < cols || ld > kMaxStride) return op_fail(EPD_ERR_SHAPE, "%s: rows of %s are %lld apart: %d .. 2^40", who, name, (long long)ld, cols);
  if ((uintptr_t)p % elem) return op_fail(EPD_ERR_INVALID_ARG, "%s: %s is not aligned to its elements", who, name);
  return EPD_OK;
}

}  // namespace epd
