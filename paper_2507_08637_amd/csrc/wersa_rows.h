// Rows of a matrix in registers, for the translation units whose kernels read a row once: pieces of 16 bytes, any alignment, sums over a row's threads.
#pragma once
#include "wersa_internal.h"

#include <algorithm>
#include <type_traits>

namespace wersa {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Rows of any length begin at any element: vector accesses of this device need no alignment beyond the element's.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));

// E values of a row from column `col` on, 16 bytes; columns past the end are zeros.
template <typename T> __device__ __forceinline__ u32x4 load_raw(const T *row, int col, int cols) {
  constexpr int E = 16 / sizeof(T);
  u32x4 p = u32x4{0, 0, 0, 0};
  if (col + E <= cols) {
    p = *reinterpret_cast<const u32x4_any *>(row + col);
  } else if (col < cols) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (col + i < cols) p[i * (int)sizeof(T) / 4] |= sizeof(T) == 4 ? __float_as_uint(ld(row + col + i)) : (__float_as_uint(ld(row + col + i)) >> 16) << 16 * (i & 1);
  }
  return p;
}
template <typename T, int E> __device__ __forceinline__ void spread(const u32x4 &p, float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (E == 4) v[i] = __uint_as_float(p[i]);
    else {
      v[2 * i] = __uint_as_float(p[i] << 16);
      v[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
    }
  }
}
template <typename T, int E> __device__ __forceinline__ void load_piece(const T *row, int col, int cols, float (&v)[E]) { spread<T, E>(load_raw(row, col, cols), v); }
// E weights from column `col` on; ones where there are none.
template <int E> __device__ __forceinline__ void load_weights(const float *weight, int col, int cols, float (&w)[E]) {
#pragma unroll
  for (int i0 = 0; i0 < E; i0 += 4) {
    float u[4] = {1.f, 1.f, 1.f, 1.f};
    if (weight) load_piece<float, 4>(weight, col + i0, cols, u);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i0 + i] = u[i];
  }
}
template <typename T, int E> __device__ __forceinline__ void store_piece(T *row, int col, int cols, const float (&v)[E]) {
  if (col + E <= cols) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      p[i] = E == 4 ? __float_as_uint(v[i]) : (uint32_t)f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
    *reinterpret_cast<u32x4_any *>(row + col) = p;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (col + i < cols) st(row + col + i, v[i]);
  }
}
template <typename T> __device__ __forceinline__ float rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ float rounded<bf16_t>(float v) { return bf16_to_f32(f32_to_bf16(v)); }

// Over the LANES threads of a row; with 256 of them through `part`, one value per wave.
template <int LANES> __device__ __forceinline__ float row_sum(float v, float *part) {
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v += __shfl_xor(v, d);
  if (LANES == 256) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (part[0] + part[1]) + (part[2] + part[3]);
  }
  return v;
}
// Largest magnitude as bits: a NaN is above every number.
template <int LANES> __device__ __forceinline__ uint32_t row_most(uint32_t v, float *part) {
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  if (LANES == 256) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
    v = max(max(__float_as_uint(part[0]), __float_as_uint(part[1])), max(__float_as_uint(part[2]), __float_as_uint(part[3])));
  }
  return v;
}

// Threads of a row and pieces of a thread: up to a wave one piece each, then four pieces of one wave, which needs no barrier, then a workgroup.
template <typename F> void by_width(int cols, int dtype, F f) {
#define WERSA_ROWS_AS(T, L, P) return f((T *)nullptr, std::integral_constant<int, L>{}, std::integral_constant<int, P>{})
  const int e = dtype == WERSA_F32 ? 4 : 8, pieces = (cols + e - 1) / e;
  if (dtype == WERSA_BF16) {
    if (pieces <= 8) WERSA_ROWS_AS(bf16_t, 8, 1);
    if (pieces <= 16) WERSA_ROWS_AS(bf16_t, 16, 1);
    if (pieces <= 32) WERSA_ROWS_AS(bf16_t, 32, 1);
    if (pieces <= 64) WERSA_ROWS_AS(bf16_t, 64, 1);
    if (pieces <= 128) WERSA_ROWS_AS(bf16_t, 64, 2);
    if (pieces <= 256) WERSA_ROWS_AS(bf16_t, 64, 4);
    if (pieces <= 512) WERSA_ROWS_AS(bf16_t, 256, 2);
    WERSA_ROWS_AS(bf16_t, 256, 4);
  }
  if (pieces <= 8) WERSA_ROWS_AS(float, 8, 1);
  if (pieces <= 16) WERSA_ROWS_AS(float, 16, 1);
  if (pieces <= 32) WERSA_ROWS_AS(float, 32, 1);
  if (pieces <= 64) WERSA_ROWS_AS(float, 64, 1);
  if (pieces <= 128) WERSA_ROWS_AS(float, 64, 2);
  if (pieces <= 256) WERSA_ROWS_AS(float, 64, 4);
  if (pieces <= 512) WERSA_ROWS_AS(float, 256, 2);
  if (pieces <= 1024) WERSA_ROWS_AS(float, 256, 4);
  WERSA_ROWS_AS(float, 256, 8);
#undef WERSA_ROWS_AS
}

// Workgroups of 256 threads at most in a dimension of a grid, which has fewer than 2^32 threads.
inline dim3 grid_of(int64_t groups) {
  const int64_t across = std::min<int64_t>(groups, 1 << 20);
  return dim3((unsigned)across, (unsigned)((groups + across - 1) / across));
}

inline bool misaligned(const void *p, size_t a) { return ((uintptr_t)p % a) != 0; }

}  // namespace wersa
