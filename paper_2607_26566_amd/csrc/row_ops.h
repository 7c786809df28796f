// Rows in pieces of eight elements, and column sums: what the row-wise operators share.
#pragma once

#include "block_ops.h"

namespace t2i {

// eight consecutive elements as fp32 (16 bytes of bf16, 32 of fp32)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<bf16>(const bf16* p, float (&v)[8]) {
  const bf16x8 w = *(const bf16x8*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (bf16)v[i];
    *(bf16x8*)p = w;
  } else {
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
}

// eight elements of a row as they lie in memory (at any address: one or two loads all
// the same), and the largest of their magnitudes' bits (which order as the magnitudes
// do, infinity and NaN above)
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const bf16* p) {
    typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
    const any4 v = *(const any4*)p;
    w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
  }
  __device__ __forceinline__ void set(int i, bf16 v) {
    const uint32_t b = __builtin_bit_cast(uint16_t, v);
    w[i >> 1] |= b << (16 * (i & 1));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ uint32_t largest() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return (uint32_t)max((uint32_t)m[0], (uint32_t)m[1]) << 16;
  }
};
template <>
struct Piece<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
    const any4 a = *(const any4*)p, b = *(const any4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
};

// eight values to memory at any address of their type, or the first n of them
template <typename T>
__device__ __forceinline__ void store_piece(T* p, int n, const float (&v)[8]) {
  typedef T any4 __attribute__((ext_vector_type(sizeof(T) == 2 ? 8 : 4), aligned(sizeof(T))));
  if (n >= 8) {
    if constexpr (sizeof(T) == 2) {
      any4 o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = (T)v[i];
      *(any4*)p = o;
    } else {
      *(any4*)p = any4{v[0], v[1], v[2], v[3]};
      *(any4*)(p + 4) = any4{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}
// a piece of a row of K elements: what lies behind K is 0
template <typename T>
__device__ __forceinline__ void load_piece(const T* row, int k, int K, Piece<T>& p) {
  if (k + 8 <= K) {
    p.load(row + k);
  } else {
    p.clear();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < K) p.set(i, row[k + i]);
  }
}

// Column sums of n rows of fp32 or fp64 partials (row stride ld) in fp64: 16 columns
// per workgroup of 1024, each by 64 threads that take every 64th row (so that a
// sum's reads are all under way at once), joined in a fixed order.
template <typename S>
__device__ __forceinline__ double column_sum(const S* p, int n, size_t ld, int c, bool in) {
  __shared__ double red[64][16];
  const int s = threadIdx.x / 16, l = threadIdx.x % 16;
  double v = 0.;
  if (in) {
#pragma unroll 4
    for (int i = s; i < n; i += 64) v += (double)p[(size_t)i * ld + c];
  }
  red[s][l] = v;
  __syncthreads();
  if (s < 4) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += red[s + 4 * i][l];
  }
  __syncthreads();
  if (s < 4) red[s][l] = v;
  __syncthreads();
  return (red[0][l] + red[1][l]) + (red[2][l] + red[3][l]);
}

}  // namespace t2i
