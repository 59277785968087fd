// Tiles of scaled dot-product attention in fp32 on the matrix cores (d = 64 or 128).  The arrangement is described in
// attention_f32.hip, whose kernels and those of cross_attention_f32.hip are made of these.
#pragma once
#include "common.h"

namespace moe {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// a lane's 16-byte pieces of a row (half of its d)
template <int D> struct Pieces {
  f32x4_t v[D / 8];
  __device__ __forceinline__ void load(const float* row, int hf) {
#pragma unroll
    for (int g = 0; g < D / 8; ++g) v[g] = *reinterpret_cast<const f32x4_t*>(row + 8 * g + 4 * hf);
  }
  __device__ __forceinline__ f32x4_t piece(int g) const { return v[g]; }
};
// The floats of a block's 32 rows that the sums over rows take.  Rows past the end are copies of the last one, with a
// factor of 0.  An infinity in that row of v or dctx must not become 0 x inf there, so they are cleared before use (q and
// k need not be: their infinities make the head's scores, so all results, NaN anyway).
template <int D> struct Rows {
  float v[16][D / 32];
  __device__ __forceinline__ void load(const float* base, size_t ld, int row0, int L, int r, int hf) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      int row = row0 + 8 * (i >> 2) + 4 * hf + (i & 3);
      row = row < L ? row : L - 1;
#pragma unroll
      for (int t = 0; t < D / 32; ++t) v[i][t] = base[(size_t)row * ld + 32 * t + r];
    }
  }
  // at(row): where row `row` is
  template <typename F>
  __device__ __forceinline__ void load_at(F&& at, int row0, int L, int r, int hf) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      int row = row0 + 8 * (i >> 2) + 4 * hf + (i & 3);
      const float* const p = at(row < L ? row : L - 1);
#pragma unroll
      for (int t = 0; t < D / 32; ++t) v[i][t] = p[32 * t + r];
    }
  }
  __device__ __forceinline__ void clear_past(int row0, int L, int hf) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int t = 0; t < D / 32; ++t) v[i][t] = row0 + 8 * (i >> 2) + 4 * hf + (i & 3) < L ? v[i][t] : 0.f;
  }
  __device__ __forceinline__ float at(int i, int t) const { return v[i][t]; }
};
// 32 rows staged in LDS serve as both.  Pitch: the halves of a one-float read, four rows apart, start 32 banks apart.
template <int D> struct Staged {
  static constexpr int kPitch = D + 8, kFloats = 32 * kPitch;
  const float* rows;
  int r, hf;
  __device__ __forceinline__ f32x4_t piece(int g) const {
    return *reinterpret_cast<const f32x4_t*>(rows + r * kPitch + 8 * g + 4 * hf);
  }
  __device__ __forceinline__ float at(int i, int t) const {
    return rows[(8 * (i >> 2) + 4 * hf + (i & 3)) * kPitch + 32 * t + r];
  }
};
// the rows 32 blk .. + 31 of two operands on their way to LDS (past the end: the last one on the way, zeros in LDS)
template <int D> struct Transit {
  static constexpr int kPer = 32 * D / 4 / 256, kVecs = D / 4;
  f32x4_t a[kPer], b[kPer];
  __device__ __forceinline__ void fetch(const float* pa, size_t lda, const float* pb, size_t ldb, int blk, int L) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int f = threadIdx.x + 256 * i, c = 4 * (f % kVecs);
      int row = 32 * blk + f / kVecs;
      row = row < L ? row : L - 1;
      a[i] = *reinterpret_cast<const f32x4_t*>(pa + (size_t)row * lda + c);
      b[i] = *reinterpret_cast<const f32x4_t*>(pb + (size_t)row * ldb + c);
    }
  }
  // ata(row), atb(row): where the operands' row `row` is
  template <typename FA, typename FB>
  __device__ __forceinline__ void fetch_at(FA&& ata, FB&& atb, int blk, int L) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int f = threadIdx.x + 256 * i, c = 4 * (f % kVecs);
      int row = 32 * blk + f / kVecs;
      row = row < L ? row : L - 1;
      a[i] = *reinterpret_cast<const f32x4_t*>(ata(row) + c);
      b[i] = *reinterpret_cast<const f32x4_t*>(atb(row) + c);
    }
  }
  __device__ __forceinline__ void put(float* la, float* lb, int blk, int L) {
    if (32 * blk + 32 > L) {                                   // block-uniform
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool past = 32 * blk + (int)(threadIdx.x + 256 * i) / kVecs >= L;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          a[i][k] = past ? 0.f : a[i][k];
          b[i][k] = past ? 0.f : b[i][k];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int f = threadIdx.x + 256 * i, at = f / kVecs * Staged<D>::kPitch + 4 * (f % kVecs);
      *reinterpret_cast<f32x4_t*>(la + at) = a[i];
      *reinterpret_cast<f32x4_t*>(lb + at) = b[i];
    }
  }
};
// rows x columns over d, in two sums
template <int D, typename R>
__device__ __forceinline__ f32x16_t over_d(const R& rows, const Pieces<D>& col) {
  f32x16_t c[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) c[0][i] = c[1][i] = 0.f;
#pragma unroll
  for (int g = 0; g < D / 16; ++g) {
    const f32x4_t x[2] = {rows.piece(g), rows.piece(D / 16 + g)};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        c[h] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[h][j], col.v[h * (D / 16) + g][j], c[h], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) c[0][i] += c[1][i];
  return c[0];
}
// acc[d][column] += rows^T times c
template <int D, typename R>
__device__ __forceinline__ void over_rows(f32x16_t (&acc)[D / 32], const R& rows, const f32x16_t& c) {
#pragma unroll
  for (int t = 0; t < D / 32; t += 2) {
    f32x16_t p[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[0][i] = p[1][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) p[h] = __builtin_amdgcn_mfma_f32_32x32x2f32(rows.at(i, t + h), c[i], p[h], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) { acc[t][i] += p[0][i]; acc[t + 1][i] += p[1][i]; }
  }
}
template <int D>
__device__ __forceinline__ void clear(f32x16_t (&acc)[D / 32]) {
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
}
// acc[t][i] is d = 32 t + 8 (i/4) + 4 hf + i%4 of the lane's row
template <int D>
__device__ __forceinline__ void store_column(float* row, const f32x16_t (&acc)[D / 32], float scale, int hf) {
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4_t*>(row + 32 * t + 8 * q + 4 * hf) =
          f32x4_t{acc[t][4 * q] * scale, acc[t][4 * q + 1] * scale, acc[t][4 * q + 2] * scale, acc[t][4 * q + 3] * scale};
}

constexpr int kWaves = 4;

// the wavefronts' sums meet in wavefront 0, in order; sums: LDS, 8 KB per 64 d and wavefront but the first
template <int D>
__device__ __forceinline__ void add_up(f32x16_t (&acc)[D / 32], float (*sums)[D / 32][16][64], int wave, int lane) {
  __syncthreads();                                             // (what they held before has been read)
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[wave - 1][t][i][lane] = acc[t][i];
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] += sums[w][t][i][lane];
  }
}

}  // namespace
}  // namespace moe
