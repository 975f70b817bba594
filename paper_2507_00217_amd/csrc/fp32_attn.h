// What the fp32 attention kernels share: 16 x 16 blocks of v_mfma_f32_16x16x4_f32 with operands straight from global memory.
#pragma once
#include "common.h"

namespace stg {

typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

constexpr int AW = 8;                 // wavefronts per workgroup

// fragment of 16 rows (row index `row` for this lane) x HD, reduction along HD: t-th float4 at 16 t + 4 g
template <int HD> __device__ __forceinline__ void ld_rows(f32x4 (&f)[HD / 16], const float* row, int g) {
#pragma unroll
  for (int t = 0; t < HD / 16; ++t) f[t] = *reinterpret_cast<const f32x4*>(row + 16 * t + 4 * g);
}
// fragment with the reduction along the 16 rows: rows r0 + 4 g + j (clamped to the last one), HD / 16 consecutive columns from
// (HD / 16) * c on; f[j][i]: block i, MFMA j
template <int HD> __device__ __forceinline__ void ld_cols(float (&f)[4][HD / 16], const float* base, int64_t ld, int r0, int last, int c, int g) {
  constexpr int NT = HD / 16;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float* p = base + (int64_t)min(r0 + 4 * g + j, last) * ld + NT * c;
#pragma unroll
    for (int v = 0; v < NT / 4; ++v) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(p + 4 * v);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[j][4 * v + e] = t[e];
    }
  }
}
// acc[i][e] = D[column block i, row 4 g + e][c]: as float4 pieces of one row, piece q = e * (NT / 4) + v covers columns
// NT * (4 g + e) + 4 v ..
template <int HD> __device__ __forceinline__ f32x4 piece(const f32x4 (&acc)[HD / 16], int q) {
  constexpr int NT = HD / 16;
  const int e = q / (NT / 4), v = q % (NT / 4);
  return f32x4{acc[4 * v][e], acc[4 * v + 1][e], acc[4 * v + 2][e], acc[4 * v + 3][e]};
}
template <int HD> __device__ __forceinline__ int piece_col(int q, int g) {
  constexpr int NT = HD / 16;
  return NT * (4 * g + q / (NT / 4)) + 4 * (q % (NT / 4));
}
// A block of rows that some columns see and others do not (keys behind a query, rows past the end) is multiplied with weights that
// are zero for the pairs that do not count, which is right as long as the rows are finite: zero times an infinity or NaN is
// NaN.  `mul_seen`: acc += f^T . w with row 4 g + j counted only for the columns with ok[j], one row at a time, each column dropping
// the products of rows that it does not see.  It is far from the loops over the blocks, which carry no branch for it (a
// branch there costs the backward 4 %): the forward asks its last block, the only one with such pairs, whether its rows
// are finite (`odd_rows`) and leaves it for the end if they are not; the backward's wavefronts note on the way whether a score
// or delta, sums over whole rows, was not finite, and if so walk their blocks again.
template <int NT> __device__ __forceinline__ bool odd_rows(const float (&f)[4][NT]) {
  float t = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < NT; ++i) t = __builtin_fmaf(f[j][i], 0.f, t);            // 0, or NaN
  return __any(t != 0.f);
}
template <int NT> __device__ __forceinline__ void mul_seen(f32x4 (&acc)[NT], const float (&f)[4][NT], const f32x4& w, const bool (&ok)[4], int c, int g) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll 1
    for (int gg = 0; gg < 4; ++gg) {
      const bool see = __shfl((int)ok[j], 16 * gg + c, 64) != 0;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const f32x4 p = mfma4(g == gg ? f[j][i] : 0.f, g == gg ? w[j] : 0.f, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] += see ? p[e] : 0.f;
        __builtin_amdgcn_sched_barrier(0);                       // one product at a time: no registers beyond the plain path's
      }
    }
}
__device__ __forceinline__ float max_g(float v) { v = fmaxf(v, __shfl_xor(v, 16, 64)); return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float sum_g(float v) { v += __shfl_xor(v, 16, 64); return v + __shfl_xor(v, 32, 64); }

}  // namespace
}  // namespace stg
