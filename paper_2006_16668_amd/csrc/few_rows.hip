// C [R,N] = A [R,K] . B [K,N] of few rows or columns, bf16: the projections of a step of generation.
//
// Bound by the way of B to the matrix cores once, and, at a few MB, by latency: so all of a block's operands are asked for at once, by copies that
// bypass the registers.  A block has 32 rows and 32 columns (64 to 32 blocks for 2048 to 1024 columns and 32 rows; neighbours share lines of
// 128 bytes and columns of B, so an XCD gets a contiguous range); its eight wavefronts take chunks of 64 k in turn, two at a
// time each, 128 KB of LDS together.  B's rows of 64 bytes need no swizzle, a transposing read takes 256 consecutive bytes per half; chunk c of
// A's rows of 128 bytes sits at c ^ (row / 2) % 8, which spreads 16 rows over all banks.  (Read as fragments from memory, 16 bytes of 32 rows at a
// time, A costs as much as B.)  Transposed as in attention_mfma.hip, C^T = B^T A^T: a lane holds columns of one row.  The
// wavefronts' sums meet in LDS, in order.
//
// PAIR: the rows are pairs of bf16, A + A_rest.  A tile has 16 of them, first terms in its rows 0 .. 15 and second ones in 16 .. 31, whose products add up: neither more
// operands nor more products than a tile of 32 rows.
#include "attention_tiles.h"

namespace moe {
namespace {

constexpr int kWaves = 8, kBytesB = 64 * 64, kBytesA = 32 * 128, kPlace = kBytesB + kBytesA, kAhead = 2;
constexpr int kLds = kWaves * kAhead * kPlace;

// B_KC: B is [N,K], its rows staged and read as A's.
template <bool PAIR, bool B_KC>
__global__ __launch_bounds__(64 * kWaves, 1) void few_rows_kernel(const bf16_t* __restrict__ A, const bf16_t* __restrict__ A_rest,
                                                                  const bf16_t* __restrict__ B, bf16_t* __restrict__ C, bf16_t* __restrict__ C_rest,
                                                                  int R, int N, int K) {
  constexpr int kRows = PAIR ? 16 : 32;
  extern __shared__ __attribute__((aligned(256))) unsigned char few_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)few_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5, p16 = lane & 15, b1 = (lane >> 4) & 1;
  const unsigned item = xcd_contiguous(blockIdx.x, gridDim.x), row_tiles = (R + kRows - 1) / kRows;
  const int col0 = (int)(item / row_tiles) * 32, row0 = (int)(item % row_tiles) * kRows;
  const uint32_t own = lds0 + wave * (kAhead * kPlace);
  const uint32_t tr0 = own + (8 * hf + (p16 >> 2)) * 64 + 32 * b1 + 8 * (p16 & 3);
  const uint32_t row_at = r * 128 + ((hf ^ ((r >> 1) & 7)) << 4), a0 = own + kBytesB + row_at, b0 = own + row_at;
  auto copy = [&](uint32_t to, const bf16_t* from, bool there) __attribute__((always_inline)) {
    const uint64_t at = there ? (uint64_t)(uintptr_t)from : (uint64_t)(uintptr_t)&att_zero_line;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(at) : "memory");
  };
  const int chunks = (K + 63) / 64;
  f32x16_t acc{};
  for (int first = wave; first < chunks; first += kWaves * kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int k0 = 64 * (first + kWaves * j);
      if (k0 >= K) break;                                      // wavefront-uniform
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (B_KC) {
          const int i = 8 * x + lane / 8, k = k0 + 8 * ((lane % 8) ^ ((i >> 1) & 7));
          copy(own + j * kPlace + x * 1024, B + (size_t)(col0 + i) * K + k, col0 + i < N && k < K);
        } else {
          const int k = k0 + 16 * x + lane / 4, c = col0 + 8 * (lane % 4);
          copy(own + j * kPlace + x * 1024, B + (size_t)k * N + c, k < K && c < N);
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = 8 * x + lane / 8, k = k0 + 8 * ((lane % 8) ^ ((i >> 1) & 7));
        const int row = row0 + i % kRows;
        copy(own + j * kPlace + kBytesB + x * 1024, (i < kRows ? A : A_rest) + (size_t)row * K + k, row < R && k < K);
      }
    }
    wait_all_copies();
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (64 * (first + kWaves * j) >= K) break;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const u32x4_t a = *(lds_u4_ptr)(uintptr_t)((a0 ^ (s << 5)) + j * kPlace);
        if constexpr (B_KC) {
          acc = MOE_MFMA(*(lds_u4_ptr)(uintptr_t)((b0 ^ (s << 5)) + j * kPlace), a, acc);
        } else {
          const uint32_t at = tr0 + j * kPlace + s * 1024;
          const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)at);
          const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)(at + 256));
          acc = MOE_MFMA(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), a, acc);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // read before the next copies go there
  }
  // [wavefront][16][64]; then wavefront w adds up values 2 w and 2 w + 1
  typedef float __attribute__((address_space(3))) * lds_f_ptr;
  auto at = [&](int w, int i) __attribute__((always_inline)) { return (lds_f_ptr)(uintptr_t)(lds0 + ((w * 16 + i) * 64 + lane) * 4); };
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) *at(wave, i) = acc[i];
  __syncthreads();
  const int c = col0 + 8 * (wave / 2) + 4 * hf + 2 * (wave % 2);
  float v[2] = {0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    v[0] += *at(w, 2 * wave);
    v[1] += *at(w, 2 * wave + 1);
  }
  if constexpr (PAIR) {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = pair_sum(v[i], __shfl_xor(v[i], 16, 64));
  }
  if (r < kRows && row0 + r < R && c < N) {
    const uint32_t rounded = pack_bf16x2(v[0], v[1]);
    const size_t to = (size_t)(row0 + r) * N + c;
    *reinterpret_cast<uint32_t*>(C + to) = rounded;
    if (C_rest != nullptr) *reinterpret_cast<uint32_t*>(C_rest + to) = bf16_rest_x2(v[0], v[1], rounded);
  }
}

// fp32 on v_mfma_f32_16x16x4, tiles of 16 x 16: a tile of 32 x 32 would keep its unit's matrix cores busy for 7 us at K 2048 and leave most units
// without one.  Lane (r = lane % 16, q = lane / 16) takes k = 16 g + 4 q + j in step j of a group of 16, so A (and B [N,K], B_KC) comes as 16-byte
// pieces of rows and B [K,N] as 64 bytes of four rows, straight to registers, 128 k of a wavefront at a time.
template <bool B_KC>
__global__ __launch_bounds__(64 * kWaves, 2) void few_rows_f32_kernel(const float* __restrict__ A, const float* __restrict__ B,
                                                                      float* __restrict__ C, int R, int N, int K) {
  constexpr int G = 8;                                         // groups of 16 k
  __shared__ f32x4_t sums[kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const unsigned item = xcd_contiguous(blockIdx.x, gridDim.x), row_tiles = (R + 15) / 16;
  const int col0 = (int)(item / row_tiles) * 16, row0 = (int)(item % row_tiles) * 16;
  const float* const row = A + (size_t)(row0 + r < R ? row0 + r : R - 1) * K + 4 * q;
  const int col = col0 + r < N ? col0 + r : N - 1;
  const float* const bcol = B + (size_t)col * K + 4 * q;       // (B_KC)
  const unsigned boff = (unsigned)(4 * q * N + col);           // (else: from a row that all lanes share)
  f32x4_t acc{};
  for (int k0 = wave * 16 * G; k0 < K; k0 += kWaves * 16 * G) {
    f32x4_t a[G], b[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int k = k0 + 16 * g;
      a[g] = b[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (k + 4 * q < K) {                                     // (K is a multiple of 4)
        a[g] = *reinterpret_cast<const f32x4_t*>(row + k);
        if constexpr (B_KC) b[g] = *reinterpret_cast<const f32x4_t*>(bcol + k);
        else {
#pragma unroll
          for (int j = 0; j < 4; ++j) b[g][j] = (B + (size_t)(k + j) * N)[boff];
        }
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (k0 + 16 * g >= K) break;                             // wavefront-uniform
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(b[g][j], a[g][j], acc, 0, 0, 0);
    }
  }
  sums[wave][lane] = acc;                                      // columns 4 q .. + 3 of row r
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) acc += sums[w][lane];
  const int c = col0 + 4 * q;
  if (row0 + r < R && c < N) *reinterpret_cast<f32x4_t*>(C + (size_t)(row0 + r) * N + c) = acc;
}

}  // namespace

int prepare_few_rows() {
  static LdsLimitOnce once, once_pair, once_kc;
  int rc = ensure_lds_limit(once, reinterpret_cast<const void*>(few_rows_kernel<false, false>), kLds);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_pair, reinterpret_cast<const void*>(few_rows_kernel<true, false>), kLds);
  return rc != MOE_OK ? rc : ensure_lds_limit(once_kc, reinterpret_cast<const void*>(few_rows_kernel<false, true>), kLds);
}

// bf16 blocks fill the device once at most, fp32 blocks, of which several share a unit, three times.  us, gemm_f32.hip / this, fp32: 1024, 2048, 1 16.6 / 4.3;
// 32 16.8 / 5.7; 96 17.2 / 12.5, 128 17.0 / 16.1; 2048, 1024, 4 29.1 / 6.6; 64 29.3 / 9.2; 512, 512, 64 10.2 / 4.0.  bf16, us, the edge kernel of expert_gemm.hip / this; K, N, rows: 1024, 2048, 1 5.7 / 3.4; 64 5.9 / 3.9; 128 6.0 / 4.4,
// 192 6.1 / 7.2; 2048, 1024, 4 9.3 / 4.6; 64 9.4 / 4.7; 256 9.6 / 6.1; 1024, 4096, 64 6.0 / 4.6, 96 6.2 / 7.3; 512, 512, 4 4.0 / 3.0; 2048, 4096, 64 9.7 / 6.5.
bool few_rows_ok(int act_dtype, long long rows, int N) {
  constexpr long long kUnits = 256;
  const long long side = act_dtype == MOE_F32 ? 16 : 32, most = act_dtype == MOE_F32 ? 3 * kUnits : kUnits;
  return rows <= side * most && (rows + side - 1) / side * ((N + side - 1) / side) <= most;
}

int launch_few_rows(int act_dtype, bool b_kc, const void* A, const void* B, void* C, int R, int N, int K, hipStream_t st) {
  if (act_dtype == MOE_F32) {
    const dim3 grid((unsigned)((N + 15) / 16 * ((R + 15) / 16))), threads(64 * kWaves);
    auto a = static_cast<const float*>(A);
    auto b = static_cast<const float*>(B);
    auto c = static_cast<float*>(C);
    if (b_kc) hipLaunchKernelGGL((few_rows_f32_kernel<true>), grid, threads, 0, st, a, b, c, R, N, K);
    else hipLaunchKernelGGL((few_rows_f32_kernel<false>), grid, threads, 0, st, a, b, c, R, N, K);
    return check_launch();
  }
  return b_kc ? MOE_EUNSUPPORTED : launch_few_rows_pair(A, nullptr, B, C, nullptr, R, N, K, st);
}

bool few_rows_pair_ok(long long rows, int N) { return rows <= 16 * 256 && (rows + 15) / 16 * ((N + 31) / 32) <= 256; }

static int launch_bf16(const void* A, const void* A_rest, bool b_kc, const void* B, void* C, void* C_rest, int R, int N, int K, hipStream_t st) {
  if (prepare_few_rows() != MOE_OK) return MOE_EHIP;
  const int rows = A_rest != nullptr ? 16 : 32;
  const dim3 grid((unsigned)((N + 31) / 32 * ((R + rows - 1) / rows))), threads(64 * kWaves);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, threads, kLds, st, static_cast<const bf16_t*>(A), static_cast<const bf16_t*>(A_rest), static_cast<const bf16_t*>(B),
                       static_cast<bf16_t*>(C), static_cast<bf16_t*>(C_rest), R, N, K);
  };
  if (b_kc) run(few_rows_kernel<false, true>);
  else if (A_rest != nullptr) run(few_rows_kernel<true, false>);
  else run(few_rows_kernel<false, false>);
  return check_launch();
}
int launch_few_rows_pair(const void* A, const void* A_rest, const void* B, void* C, void* C_rest, int R, int N, int K, hipStream_t st) {
  return launch_bf16(A, A_rest, false, B, C, C_rest, R, N, K, st);
}
int launch_few_rows_transposed(const void* A, const void* B, void* C, void* C_rest, int R, int N, int K, hipStream_t st) {
  return launch_bf16(A, nullptr, true, B, C, C_rest, R, N, K, st);
}

}  // namespace moe
