// Shared by the dense operators (fqt_norm.hip, fqt_linear.hip, fqt_ortho.hip): element types,
// vector loads and stores of 8 elements, host-side checks.
#pragma once

#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "fqt_dense.h"
#include "fqt_internal.hpp"

namespace fqt {
namespace dense {

// Storage types.  bf16 is handled as its 16 bits: widening is a shift, narrowing rounds to nearest
// even and keeps NaN.
struct bf16 { uint16_t v; };
struct e4m3 { uint8_t v; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __uint_as_float(uint32_t(v.v) << 16); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  // v_cvt_pk_bf16_f32: both to nearest even, NaN stays NaN.
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  v2bf r;
  r[0] = static_cast<__bf16>(lo);
  r[1] = static_cast<__bf16>(hi);
  return __builtin_bit_cast(uint32_t, r);
}
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) {
  return bf16{uint16_t(pack_bf16(v, v))};
}

// 16 and 8 bytes at the alignment of one element: the global memory instructions of this target take
// any, and rows of odd lengths need it.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_at1 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_at1 __attribute__((ext_vector_type(2), aligned(1)));
template <typename T>
__device__ __forceinline__ u32x4 load_bytes16(const T *p) {
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const u32x4_at4 *>(p);
  else if constexpr (sizeof(T) == 2) return *reinterpret_cast<const u32x4_at2 *>(p);
  else return *reinterpret_cast<const u32x4_at1 *>(p);
}
template <typename T>
__device__ __forceinline__ void store_bytes16(T *p, u32x4 v) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4_at4 *>(p) = v;
  else *reinterpret_cast<u32x4_at2 *>(p) = v;
}

// 8 consecutive elements as float32: all of them, or the first n and zeros.
template <typename T>
__device__ __forceinline__ void load8f(const T *p, int n, float (&o)[8]) {
  if (n >= 8) {
    const u32x4 a = load_bytes16(p);
    if constexpr (sizeof(T) == 4) {
      const u32x4 b = load_bytes16(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(a[i]), o[4 + i] = __uint_as_float(b[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[2 * i] = __uint_as_float(a[i] << 16);
        o[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = i < n ? to_f32(p[i]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store8f(T *p, int n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4 a;
    if constexpr (sizeof(T) == 4) {
      u32x4 b;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
      store_bytes16(p, a);
      store_bytes16(p + 4, b);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
      store_bytes16(p, a);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// Largest code of an 8-bit type.
__host__ __device__ constexpr float code_top(int q_dtype) { return q_dtype == FQT_I8 ? 127.0f : 448.0f; }
// The code of v (already divided by its scale), rounded to nearest even, as its byte.  The clamp
// takes the last rounding of v past the top; a NaN becomes the lowest code (its row's scale is NaN).
__device__ __forceinline__ uint32_t code_i8(float v) {
  return uint32_t(int(rintf(fminf(fmaxf(v, -127.0f), 127.0f)))) & 0xFFu;
}
__device__ __forceinline__ uint32_t codes2_e4m3(float a, float b) {
  a = fminf(fmaxf(a, -448.0f), 448.0f);
  b = fminf(fmaxf(b, -448.0f), 448.0f);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xFFFFu;
}
template <int Q>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if constexpr (Q == FQT_I8)
    return code_i8(a) | (code_i8(b) << 8) | (code_i8(c) << 16) | (code_i8(d) << 24);
  else
    return codes2_e4m3(a, b) | (codes2_e4m3(c, d) << 16);
}

// ----------------------------------------------------------------------------- host checks

inline size_t elem_size(int t) { return t == FQT_F32 ? 4 : t == FQT_BF16 ? 2 : 1; }
inline bool float_type(int t) { return t == FQT_F32 || t == FQT_BF16; }
inline bool code_type(int t) { return t == FQT_I8 || t == FQT_E4M3; }
// The row stride that ld stands for, 0 if it is none.
inline int64_t row_stride(int64_t ld, int64_t cols) {
  if (ld == 0) ld = cols > 0 ? cols : 1;
  return ld >= cols && ld <= FQT_MAX_LD ? ld : 0;
}
inline bool elem_aligned(const void *p, int t) { return aligned(p, elem_size(t)); }

#define FQT_TRY_(expr)               \
  do {                               \
    const int st__ = (expr);         \
    if (st__ != FQT_OK) return st__; \
  } while (0)

}  // namespace dense
}  // namespace fqt
