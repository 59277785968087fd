// Tiles of scaled dot-product attention on the matrix cores (bf16, d = 64 or 128): staging, fragments, the units of a step.  The
// arrangement is described in attention_mfma.hip, whose kernels and those of cross_attention.hip are made of these.
#pragma once
#include <type_traits>
#include <utility>
#include "common.h"

namespace moe {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef s16x4_t __attribute__((address_space(3))) * lds_s16x4_ptr;
typedef u32x4_t __attribute__((address_space(3))) * lds_u4_ptr;
typedef f32x4_t __attribute__((address_space(3))) * lds_f4_ptr;
typedef unsigned char __attribute__((address_space(3))) * lds_ptr;

static __device__ const u32x4_t att_zero_line = {0u, 0u, 0u, 0u};

template <int D> struct AttGeom {
  static constexpr int kRow = 2 * D, kChunks = D / 8, kBlock = 64 * kRow;      // bytes, 16-byte chunks, bytes
  static constexpr int kRowsPerCopy = 1024 / kRow, kCopies = kBlock / 4096;    // 1 KB copies per wavefront
};
template <int D>
__device__ __forceinline__ constexpr int att_swizzle(int row) {
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

#define MOE_MFMA(a, b, c)                                                                      \
  __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),                      \
                                          __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0)
// acc += a . b with acc in accumulation registers (gradients, whose tiles no vector instruction touches).  Score tiles, which
// vector instructions read, stay in vector registers (builtin above, and see the build's flag for this file): left to
// itself the compiler puts all results of a kernel into one kind and copies.  It does not see what this instruction asks
// for: 2 wait states after a vector instruction that wrote a or b (fresh_operand) and 11 before anything but the next product
// into it touches acc (settle_all; 19 for longer products).  Both stand where the source needs them; that the compiler
// puts no copy or spill in between is read from the compiled code by tests/test_attention_wait_states.py.
__device__ __forceinline__ void mfma_acc(f32x16_t& acc, const u32x4_t& a, const u32x4_t& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void fresh_operand() { asm volatile("s_nop 1"); }
// zeros in accumulation registers
__device__ __forceinline__ void clear_acc(f32x16_t& acc) {
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  asm volatile("" : "+a"(acc));
}

// f(0), f(1), .. f(N - 1), the argument a constant
template <typename F, int... I>
__device__ __forceinline__ void unroll_list(std::integer_sequence<int, I...>, F&& f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void unroll(F&& f) { unroll_list(std::make_integer_sequence<int, N>{}, f); }
// A step as units FIRST .. N - 1.  Unit u's fragment is fetched AHEAD units early by read(u); count(u) products use it, and after
// product p comes a share of the vector work, side(u, p, n): one wavefront issues in order, so what is to run under
// a product stands right behind it, and a second product right behind the first would only wait for the pipe.  Fences
// keep it that way.
template <int FIRST, int N, int AHEAD, typename Count, typename Read, typename Multiply, typename Side>
__device__ __forceinline__ void run_units(Count&& count, Read&& read, Multiply&& multiply, Side&& side) {
  u32x4_t f[AHEAD + 1];
  unroll<AHEAD>([&](auto I) __attribute__((always_inline)) {
    constexpr int u = FIRST + decltype(I)::value;
    f[u % (AHEAD + 1)] = read(std::integral_constant<int, u>{});
  });
  unroll<N - FIRST>([&](auto I) __attribute__((always_inline)) {
    constexpr std::integral_constant<int, FIRST + decltype(I)::value> U{};
    constexpr int u = FIRST + decltype(I)::value;
    constexpr int n = decltype(count(U))::value;
    if constexpr (u + AHEAD < N) f[(u + AHEAD) % (AHEAD + 1)] = read(std::integral_constant<int, u + AHEAD>{});
    unroll<n>([&](auto P) __attribute__((always_inline)) {
      multiply(U, P, f[u % (AHEAD + 1)]);
      __builtin_amdgcn_sched_barrier(0);
      side(U, P, std::integral_constant<int, n>{});
      __builtin_amdgcn_sched_barrier(0);
    });
  });
}

// wait states between the last products into the tiles and reads of them
template <int CT, int DT>
__device__ __forceinline__ void settle_all(f32x16_t (&a)[CT][DT]) {
  asm volatile("s_nop 15\n\ts_nop 3" : "+a"(a[0][0]));
#pragma unroll
  for (int i = 1; i < CT * DT; ++i) asm volatile("" : "+a"(a[i / DT][i % DT]));
}

template <typename V>
__device__ __forceinline__ u32x4_t pack8(const V& v, int first) {
  return u32x4_t{pack_bf16x2(v[first], v[first + 1]), pack_bf16x2(v[first + 2], v[first + 3]),
                 pack_bf16x2(v[first + 4], v[first + 5]), pack_bf16x2(v[first + 6], v[first + 7])};
}
// the terms of a fragment of P or dS: three bf16 terms that hold all 24 bits, or one rounded to bf16
template <int TERMS, typename V>
__device__ __forceinline__ void fragment_terms(const V& v, int first, bf16x8_bits_t (&t)[TERMS]) {
  if constexpr (TERMS == 3) split_bf16x8(v, first, t);
  else t[0] = pack8(v, first);
}
// dS = p (dp - D), rounded.  The compiler fused it with the subtractions of split_bf16x8 in some kernels and not in others: the
// terms were then those of the unrounded product, and a sequence's dq would depend on the kernel that forms it.
__device__ __forceinline__ float dscore(float p, float dp, float D) {
#pragma clang fp contract(off)
  return p * (dp - D);
}
// Every XCD (own L2) takes a contiguous range of work items: the blocks of one (sequence, head) read the same rows.
__device__ __forceinline__ unsigned xcd_contiguous(unsigned block, unsigned blocks) {
  const unsigned per_xcd = blocks / 8;
  return block < per_xcd * 8 ? (block % 8) * per_xcd + block / 8 : block;
}

// Per-lane byte offsets of this wavefront's copies of a block of 64 rows, `ld` elements apart.
template <int D>
__device__ __forceinline__ void copy_offsets(uint32_t (&off)[AttGeom<D>::kCopies], size_t ld, int wave, int lane) {
  using GM = AttGeom<D>;
#pragma unroll
  for (int q = 0; q < GM::kCopies; ++q) {
    const int row = GM::kRowsPerCopy * (GM::kCopies * wave + q) + lane / GM::kChunks;
    off[q] = (uint32_t)(row * ld * 2) + 16 * ((lane % GM::kChunks) ^ att_swizzle<D>(row));
  }
}
// Start copy q of this wavefront of the rows first .. first + 63 (RAGGED: zeros from row L on) to the LDS block at `lds`.
template <int D, bool RAGGED>
__device__ __forceinline__ void stage_copy(uint32_t lds, const bf16_t* rows, size_t ld, int first, int L,
                                           const uint32_t (&off)[AttGeom<D>::kCopies], int q, int wave, int lane) {
  using GM = AttGeom<D>;
  const bf16_t* const src = rows + (size_t)first * ld;
  lds += (wave * GM::kCopies + q) * 1024;
  if (RAGGED && first + 64 > L) {
    const int row = first + GM::kRowsPerCopy * (GM::kCopies * wave + q) + lane / GM::kChunks;
    const uint64_t at = row < L ? (uint64_t)(uintptr_t)src + off[q] : (uint64_t)(uintptr_t)&att_zero_line;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off[q]), "s"(src) : "memory");
  }
}
// Start the copies of the wavefront's own 32 CT rows (row L - 1 in place of those past it) to its own LDS block.
template <int D, int CT>
__device__ __forceinline__ void stage_own(uint32_t lds, const bf16_t* rows, size_t ld, int first, int L, int lane) {
  using GM = AttGeom<D>;
#pragma unroll
  for (int q = 0; q < 32 * CT * GM::kRow / 1024; ++q) {
    const int row = GM::kRowsPerCopy * q + lane / GM::kChunks, at = first + row < L ? first + row : L - 1;
    const uint64_t src = (uint64_t)(uintptr_t)(rows + (size_t)at * ld + 8 * ((lane % GM::kChunks) ^ att_swizzle<D>(row)));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + q * 1024), "v"(src) : "memory");
  }
}
__device__ __forceinline__ void wait_all_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// LDS addresses, relative to a staged block, of a lane's fragments.
//   rows:       lane (r, hf) reads d = 16 s + 8 hf .. + 7 of row 32 t + r
//   transposed: lane needs d = 32 dt + lane%32 of the rows 16 s + 4 hf .. + 3 (x = 0) and 16 s + 8 + 4 hf .. + 3
//               (x = 1), the k order in which a result tile's registers already hold the other operand
template <int D>
struct AttReads {
  using GM = AttGeom<D>;
  uint32_t row0, tr0;
  __device__ __forceinline__ AttReads(uint32_t lds0, int lane) {
    const int r = lane & 31, hf = lane >> 5, p16 = lane & 15, b1 = (lane >> 4) & 1, rr = p16 >> 2;
    row0 = lds0 + r * GM::kRow + ((hf ^ att_swizzle<D>(r)) << 4);
    const int sw = D == 128 ? rr << 2 : (rr >> 1) << 2;
    tr0 = lds0 + (4 * hf + rr) * GM::kRow + ((((2 * b1 + ((p16 >> 1) & 1)) ^ hf) ^ sw) << 4) + 8 * (p16 & 1);
  }
  __device__ __forceinline__ u32x4_t row(uint32_t block, int t, int s) const {
    return *(lds_u4_ptr)(uintptr_t)((row0 ^ (s << 5)) + block + t * 32 * GM::kRow);
  }
  __device__ __forceinline__ u32x4_t transposed(uint32_t block, int row16, int dt) const {
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)((tr0 ^ (dt << 6)) + block + row16 * GM::kRow));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4_ptr)(uintptr_t)((tr0 ^ (dt << 6) ^ 32) + block + (row16 + 8) * GM::kRow));
    return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// The wavefront's result tiles, element (d = 32 dt + 8 (i/4) + 4 hf + i%4, column 32 c + r) times factor, as whole
// rows of the columns first .. (not from L on), turned through the wavefront's own LDS block at `lds`.
template <int D, int CT>
__device__ __forceinline__ void store_own(const f32x16_t (&acc)[CT][D / 32], float factor, uint32_t lds, bf16_t* rows,
                                          size_t ld, int first, int L, int lane) {
  using GM = AttGeom<D>;
  typedef u32x2_t __attribute__((address_space(3))) * lds_u2_ptr;
  const int r = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(lds_u2_ptr)(uintptr_t)(lds + (32 * c + r) * GM::kRow + (((4 * dt + g) ^ att_swizzle<D>(r)) << 4) + 8 * hf) =
            u32x2_t{pack_bf16x2(acc[c][dt][4 * g] * factor, acc[c][dt][4 * g + 1] * factor),
                    pack_bf16x2(acc[c][dt][4 * g + 2] * factor, acc[c][dt][4 * g + 3] * factor)};
#pragma unroll
  for (int q = 0; q < 32 * CT * GM::kRow / 1024; ++q) {
    const int row = GM::kRowsPerCopy * q + lane / GM::kChunks, chunk = lane % GM::kChunks;
    const u32x4_t v = *(lds_u4_ptr)(uintptr_t)(lds + row * GM::kRow + ((chunk ^ att_swizzle<D>(row)) << 4));
    if (first + row < L) *reinterpret_cast<u32x4_t*>(rows + (size_t)(first + row) * ld + 8 * chunk) = v;
  }
}

}  // namespace
}  // namespace moe
