// The three large products of a vocabulary's loss in bf16 (vocab_loss.hip has the formulas):
//
//   z  = x . w^T     [rows, M] x [entries, M]^T     both operands K-contiguous; z itself is not stored
//   dx = dz . w      [rows, entries] x [entries, M]
//   dw = dz^T . x    [rows, entries]^T x [rows, M]
//
// v_mfma_f32_32x32x16_bf16 on tiles of 256 x 256, steps of 64 k, one block of eight wavefronts per compute unit.  A SIMD holds
// two of them, wavefront w and w + 4, half a phase apart: while one multiplies, the other fetches its next fragments from LDS
// and starts copies, and a barrier makes them change places.  The matrix pipe is then handed from one to the other instead of
// waiting for the LDS (one wavefront per SIMD with all 256 accumulators, the expert products' persistent kernel, keeps it 60 %
// busy where clocks are not the limit, operands of zeros; 128 x 256 tiles, two blocks per unit, less).
// Bound by power: 31130 rows, M 1024, 32000 entries, z and its statistics 1.54 to 1.6 ms, 1.28 to 1.33 PFLOP/s at 1.5 GHz, the
// matrix pipe 73 % busy; dz 1.04 to 1.13 PFLOP/s, dx 1.27 to 1.33 and dw 1.30 to 1.36 (86 % busy at 1.4 GHz); a library's 8192^3 is at 1.38
// PFLOP/s.  dz's tile end, of 982 us a launch of half the entries: stores 73, the pass through LDS 81, exponentials 40.
//
// A wavefront tile is 2 x 64 rows (of the upper and the lower 128 of the tile) by 2 x 32 columns, so the operands of a step are
// four LDS pieces of 16 KB, A0 A1 B0 B1, and a step has four phases of eight MFMAs:
//     phase   products   fetched meanwhile (by the other phase's turn)    copies started (two steps ahead)
//     1       A0 B0      B0
//     2       A0 B1      B1                                               A1 (one ahead)
//     3       A1 B1      A1                                               B0 B1
//     4       A1 B0      A0 of the tile's next step                       A0
// Of a tile at the end whose second 128 rows, or columns, do not exist the phases that would multiply them only copy and pass the
// barriers (2100 tokens, M 1096, V 32000, backward 513 -> 490 us; 496 tokens, 283 with a target, M 920, V 105770, forward 113 -> 107).
// A piece is copied over as soon as both wavefronts of every SIMD have read it, so two stages (128 KB) give a copy more than a
// step's time.  Copies bypass the registers (global_load_lds_dwordx4) and run on across tiles: a block walks its share of them.
//
// LDS, bank conflicts: a K-contiguous piece is [128 rows][8 chunks of 8 k], chunk c of row r at c ^ ((r >> 1) & 7); a row-of-k
// piece is [64 k][16 chunks of 8 columns], chunk c of row k at c ^ 4 (k & 3), read transposing.
#include <math.h>
#include <type_traits>
#include "common.h"

namespace moe {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr int kXcds = 8;
constexpr uint32_t kPiece = 16384, kStage = 4 * kPiece, kStaging = 2 * kStage;
constexpr uint32_t kRowData = kStaging + 8 * 2048;             // lse2, grad, hit, hit_value of a tile's rows (kLogitGrad)
constexpr uint32_t kSmem = kStaging + 8 * 4096;                // all 160 KB (statistics: 4 KB of staging per wavefront)

static __device__ const u32x4_t vocab_zero_line = {0u, 0u, 0u, 0u};

// kStats: statistics of the logits without the rows' targets, whose logits are stored (cross entropy).  kEntries: of all, and the logits
// at a teacher's entries stored.  (As one kernel for both they hold more than the scalar registers take.)
enum VocabEpi { kStats, kLogitGrad, kSums, kPlain, kEntries };
enum VocabTile { kWhole, kUpper, kLeft };      // of a tile at the end the half that exists, its first 128 rows or columns

struct VocabGemmArgs {
  const bf16_t *A, *B;
  void* C;
  int lda, ldb, ldc;
  int R, N, K;                 // rows and columns of C, length of the sum; R, or K (kPlain), is kept[0], K of a range (kSums) kept[2]
  int k_total, tiles_n, add;
  const int32_t* kept;
  VocabRows v;
};

// The lane's number, found where it is asked for: what the compiler derives from one that it knows is computed before the K loop,
// and takes registers there.
__device__ __forceinline__ int lane_here() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// TAIL: the length of the sums is no multiple of 64.  Asked for in every step it costs 5 % of the time, so the steps before a sum's last
// ones have a loop of their own (6027 tokens, M 1336, V 6322, backward 278 -> 266 us); a branch between two kinds of steps inside
// one loop spills the accumulators.  dw's length, the number of rows with a target, is not known to the host: there both operands
// have rows of zeros up to the next multiple.
template <int EPI, bool TAIL>
__global__ __launch_bounds__(512, 2) void vocab_gemm_kernel(VocabGemmArgs g) {
  constexpr bool A_MNC = EPI == kPlain, B_MNC = EPI == kSums || EPI == kPlain;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  typedef unsigned char __attribute__((address_space(3))) * lds_ptr;
  typedef s16x4_t __attribute__((address_space(3))) * lds_s16x4_ptr;
  typedef bf16x8_t __attribute__((address_space(3))) * lds_bf16x8_ptr;
  typedef u32x2_t __attribute__((address_space(3))) * lds_u2_ptr;
  typedef u32x4_t __attribute__((address_space(3))) * lds_u4_ptr;
  typedef float __attribute__((address_space(3))) * lds_f_ptr;
  typedef int __attribute__((address_space(3))) * lds_i_ptr;
  typedef bf16_t __attribute__((address_space(3))) * lds_bf16_ptr;
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)smem_raw);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int r32 = lane & 31, hh = lane >> 5;

  const int kept = __builtin_amdgcn_readfirstlane(g.kept[0]);
  const int R = EPI == kPlain ? g.R : kept;
  const int tiles_m = (R + 255) >> 8, tiles_n = g.tiles_n;
  const int range = EPI == kSums ? __builtin_amdgcn_readfirstlane(g.kept[2]) : 0;      // (a last piece fills fewer of them)
  const int per_range = tiles_m * tiles_n, ntiles = EPI == kSums ? per_range * ((g.k_total + range - 1) / range) : per_range;
  // k of a range, and its steps
  auto range_k = [&](int e) {
    if (EPI == kPlain) return kept;
    if (EPI != kSums) return g.K;
    const int left = g.k_total - e * range;
    return left < range ? left : range;
  };
  // this block's tiles: a contiguous share of them per XCD, taken in turn by its blocks
  const int xcd = blockIdx.x % kXcds;
  const int xq = ntiles / kXcds, xr = ntiles % kXcds;
  const int t_begin = xcd * xq + (xcd < xr ? xcd : xr), t_end = t_begin + xq + (xcd < xr ? 1 : 0);
  const int stride = ((int)gridDim.x - xcd + kXcds - 1) / kXcds;
  const int first = t_begin + (int)blockIdx.x / kXcds;
  if (first >= t_end) return;
  // tile -> range, row tile, column tile: bands of 8 row tiles, row tile fastest (shared panels in an XCD's L2).  With
  // half tiles a round of them is dealt out nine blocks further on than the one before, so that a block does not get those, or none,
  // of all rounds.
  const bool halves = (R - 1) % 256 < 128 || (B_MNC && (g.N - 1) % 256 < 128);
  auto tile_at = [&](int t, int& e, int& rt, int& ct) {
    if (halves) {
      const int round = (t - t_begin) / stride, from = t_begin + round * stride;
      if (from + stride <= t_end) t = from + (t - from + 9 * round) % stride;
    }
    e = EPI == kSums ? t / per_range : 0;
    t -= e * per_range;
    const int band = t / (8 * tiles_n), rem = t - band * 8 * tiles_n;
    const int left = tiles_m - band * 8, rows = left < 8 ? left : 8;
    ct = rem / rows;
    rt = band * 8 + (rem - ct * rows);
  };

  // ---- copies: two of 1 KB per wavefront and piece
  int p_tile = first, p_kt = 0, p_steps = 0, p_more = 0, p_left = 0;
  uint32_t p_stage = 0;
  const bf16_t *p_a = nullptr, *p_b = nullptr;
  uint32_t a_off[2][2], b_off[2][2];                           // [piece][copy] byte offsets of this lane from p_a, p_b (255 rows of 2^24 bytes at most)
  auto set_sources = [&]() __attribute__((always_inline)) {
    p_more = 0;
    for (; p_tile < t_end; p_tile += stride) {
      int e, rt, ct;
      tile_at(p_tile, e, rt, ct);
      p_left = range_k(e);
      p_steps = (p_left + 63) >> 6;
      if (p_steps == 0) continue;                              // (dw without a single row)
      p_more = 1;
      const int m0 = rt * 256, n0 = ct * 256, lane = lane_here();
      p_a = A_MNC ? g.A + m0 : g.A + (size_t)m0 * g.lda + (EPI == kSums ? (size_t)e * range : 0);
      p_b = B_MNC ? g.B + (EPI == kSums ? (size_t)e * range * g.ldb : 0) : g.B + (size_t)n0 * g.ldb;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int c = 2 * wave + q;
          if (A_MNC || B_MNC) {
            const int kr = 4 * c + (lane >> 4), ch = (lane & 15) ^ (4 * (kr & 3)), col = 128 * h + 8 * ch;
            // (columns of A up to the pitch, a multiple of 256, exist; B's last ones stand in for those behind)
            if (A_MNC) a_off[h][q] = (uint32_t)((kr * g.lda + col) * 2);
            if (B_MNC) b_off[h][q] = (uint32_t)((kr * g.ldb + (n0 + col < g.N ? n0 + col : g.N - 8)) * 2);
          }
          const int pr = 8 * c + (lane >> 3), ch = (lane & 7) ^ ((pr >> 1) & 7);       // row of the piece
          const int row = 128 * h + pr, col = 64 * (pr >> 5) + 32 * h + (pr & 31);
          if (!A_MNC) a_off[h][q] = ((uint32_t)(m0 + row < R ? row : R - 1 - m0) * (uint32_t)g.lda + 8 * ch) * 2;
          if (!B_MNC) b_off[h][q] = ((uint32_t)(n0 + col < g.N ? col : g.N - 1 - n0) * (uint32_t)g.ldb + 8 * ch) * 2;
        }
      break;
    }
    p_more = __builtin_amdgcn_readfirstlane(p_more);
    p_steps = __builtin_amdgcn_readfirstlane(p_steps);
  };
#define MOE_VG_COPY(LDS, VOFF, SBASE)                                                          \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(LDS), "v"(VOFF), "s"(SBASE) : "memory")
#define MOE_VG_COPY_AT(LDS, ADDR)                                                              \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(LDS), "v"(ADDR) : "memory")
  // one piece of an operand; in the last step of a sum, k behind its end comes from a line of zeros
  auto copy_piece = [&](auto tail, bool mnc, uint32_t at, const uint32_t (&off)[2], const bf16_t* base) __attribute__((always_inline)) {
    if (!decltype(tail)::value || p_left >= 64) {
#pragma unroll
      for (int q = 0; q < 2; ++q) MOE_VG_COPY(at + q * 1024, off[q], base);
    } else {
      const int lane = lane_here();
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = 2 * wave + q, pr = 8 * c + (lane >> 3);
        const int k = mnc ? 4 * c + (lane >> 4) : 8 * ((lane & 7) ^ ((pr >> 1) & 7));
        const uint64_t from = k < p_left ? (uint64_t)(uintptr_t)base + off[q] : (uint64_t)(uintptr_t)&vocab_zero_line;
        MOE_VG_COPY_AT(at + q * 1024, from);
      }
    }
  };
  auto copy_a = [&](auto tail, int h) __attribute__((always_inline)) {
    if (p_more) copy_piece(tail, A_MNC, lds0 + p_stage + h * kPiece + wave * 2048, a_off[h], p_a);
  };
  auto copy_b = [&](auto tail) __attribute__((always_inline)) {
    if (!p_more) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) copy_piece(tail, B_MNC, lds0 + p_stage + (2 + h) * kPiece + wave * 2048, b_off[h], p_b);
  };
  auto advance = [&]() __attribute__((always_inline)) {
    if (!p_more) return;
    p_stage ^= kStage;
    p_a += A_MNC ? (size_t)64 * g.lda : 64;
    p_b += B_MNC ? (size_t)64 * g.ldb : 64;
    p_left -= 64;
    if (++p_kt == p_steps) {
      p_kt = 0;
      p_tile += stride;
      set_sources();
    }
  };

#define MOE_VG_WORDS(LDS, P)                                                                   \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(LDS), "v"((uint64_t)(uintptr_t)(P)) : "memory")
  // kLogitGrad: what the tile's epilogue needs of its rows, 64 of them per wavefront.  Started in the tile's first step, when
  // all have left the last tile's epilogue, and landed with what the second step waits for (sums have two steps at least).
  auto copy_row_data = [&](int m0) __attribute__((always_inline)) {
    const int row = m0 + 64 * wn + lane_here(), at = row < R ? row : R - 1;
    const uint32_t to = lds0 + kRowData + wm * 1024 + wn * 256;
    MOE_VG_WORDS(to, (wm == 0 ? g.v.lse2 : g.v.grad) + at);
    if (g.v.hit != nullptr) MOE_VG_WORDS(to + 2048, (wm == 0 ? reinterpret_cast<const float*>(g.v.hit) : g.v.hit_value) + at);
  };

  // kStats: the targets of the wavefront's rows, into its own staging, behind what the wavefronts exchange
  const uint32_t hits = lds0 + kStaging + wave * 4096 + 3 * 1024;
  auto copy_hits = [&](int m0) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = m0 + 128 * h + 64 * wm + lane_here();
      MOE_VG_WORDS(hits + 256 * h, g.v.hit + (row < R ? row : R - 1));
    }
  };

  // ---- fragments
  const int p16 = lane & 15, bb = lane >> 4, bk = 8 * (bb >> 1) + (p16 >> 2);
  // where a wavefront's first fragment of a piece lies: K-contiguous ones of 16 k further on at ^ 32, of 32 rows at + 4096;
  // row-of-k ones of 16 k at + 4096, and those of A's 32 columns further on have a base of their own
  uint32_t a_rd[A_MNC ? 2 : 1], b_rd;
  {
    const uint32_t kc = r32 * 128 + ((hh ^ ((r32 >> 1) & 7)) * 16);
    auto mnc = [&](int chunk) { return (uint32_t)(bk * 256 + (((chunk + 2 * (bb & 1) + ((p16 & 3) >> 1)) ^ (4 * (bk & 3))) * 16) + (p16 & 1) * 8); };
#pragma unroll
    for (int i = 0; i < (A_MNC ? 2 : 1); ++i) a_rd[i] = lds0 + (A_MNC ? mnc(8 * wm + 4 * i) : wm * 64 * 128 + kc);
    b_rd = lds0 + 2 * kPiece + (B_MNC ? mnc(4 * wn) : wn * 32 * 128 + kc);
  }
  auto read_tr = [&](uint32_t at) __attribute__((always_inline)) {
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)at);
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)(at + 4 * 256));
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  bf16x8_t a[2][2][4], b[2][4];                                // [piece][32-row tile][16 k]
  auto read_a = [&](int h) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        a[h][i][kk] = A_MNC ? read_tr(a_rd[A_MNC ? i : 0] + h * kPiece + kk * 16 * 256)
                            : *(lds_bf16x8_ptr)(uintptr_t)((a_rd[0] ^ (32 * kk)) + h * kPiece + i * 32 * 128);
  };
  auto read_b = [&](int h) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      b[h][kk] = B_MNC ? read_tr(b_rd + h * kPiece + kk * 16 * 256)
                       : *(lds_bf16x8_ptr)(uintptr_t)((b_rd ^ (32 * kk)) + h * kPiece);
  };
  uint32_t to_other = kStage;                                  // from the stage being read to the other one
  auto other_stage = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < (A_MNC ? 2 : 1); ++i) a_rd[i] += to_other;
    b_rd += to_other;
    to_other = -to_other;
  };
  f32x16_t acc[4][2];
  // one turn of the matrix pipe: between two barriers, what was fetched before the first of them.  A tile's first step starts
  // from an operand of zeros: 128 registers need no clearing.
  const f32x16_t zeros = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto turn = [&](auto first, int h, int j, bool multiplies) __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (multiplies) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < (multiplies ? 4 : 0); ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        acc[2 * h + i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j][kk], a[h][i][kk],
                                                                    decltype(first)::value && kk == 0 ? zeros : acc[2 * h + i][j], 0, 0, 0);
    if (multiplies) __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // Start: step 0, and B and A0 of step 1, as a step finds them
  int steps_left = 0;                                          // of all this block's tiles, to know which steps exist
  for (int t = first; t < t_end; t += stride) {
    int e, rt, ct;
    tile_at(t, e, rt, ct);
    steps_left += (range_k(e) + 63) >> 6;
  }
  set_sources();
  constexpr auto any = std::integral_constant<bool, TAIL>{};
  copy_b(any); copy_a(any, 0); copy_a(any, 1); advance();
  copy_b(any); copy_a(any, 0);
  if (steps_left > 1) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  if (wm == 1) __builtin_amdgcn_s_barrier();                   // half a phase behind
  asm volatile("" ::: "memory");
  for (int tile = first; tile < t_end; tile += stride) {
    int e, rt, ct;
    tile_at(tile, e, rt, ct);
    const int m0 = rt * 256, n0 = ct * 256;
    const int steps = (range_k(e) + 63) >> 6;
    // kEntries: the teacher's entries among this wavefront's results.  Where they are is fetched in the tile's first step, into the
    // wavefront's staging (as copy_row_data), the first 256 of them are copied to A1's place in the last one (read by all when phase 4
    // begins, free until the next tile's phase 2).
    int entries = 0;
    const uint2* list = nullptr;
    uint32_t list_at = 0;
    auto step = [&](auto first_step, auto tail, auto half, int kt) __attribute__((always_inline)) {
      constexpr bool upper = decltype(half)::value == kUpper, left = decltype(half)::value == kLeft;
      const bool landed = decltype(first_step)::value && tile != first;        // what it waits for: before the last tile's stores
      // phase 1
      read_b(0);
      turn(first_step, 0, 0, true);
      // phase 2; A1 of this step must have landed (younger: B and A0 of the next).  A1 of the next step is started here and not
      // before: its place is where the last tile's results passed through.
      if (!left) read_b(1);
      if (!landed) {
        if (steps_left > 1) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      copy_a(tail, 1);
      advance();
      turn(first_step, 0, 1, !left);
      // phase 3; B and A0 of the next step (younger: its A1)
      if (!upper) read_a(1);
      if (!landed) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
      if (EPI == kLogitGrad && decltype(first_step)::value) copy_row_data(m0);
      if (EPI == kStats && decltype(first_step)::value) copy_hits(m0);
      if (EPI == kEntries && decltype(first_step)::value && g.v.starts != nullptr)
        MOE_VG_WORDS(lds0 + kStaging + wave * 4096, g.v.starts + (size_t)rt * (8 * tiles_n + 1) + 8 * ct + wave + lane_here());
      copy_b(tail);
      turn(first_step, 1, 1, !upper && !left);
      // phase 4
      if (EPI == kEntries && !decltype(first_step)::value && kt + 1 == steps && g.v.starts != nullptr) {
        const u32x2_t start = *(lds_u2_ptr)(uintptr_t)(lds0 + kStaging + wave * 4096);
        const int found = __builtin_amdgcn_readfirstlane((int)start[0]);
        entries = __builtin_amdgcn_readfirstlane((int)start[1]) - found;
        list = g.v.sorted + (size_t)m0 * g.v.K + found;
        list_at = lds0 + (to_other == kStage ? 0 : kStage) + kPiece + wave * 2048;
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(list) + lane_here();
#pragma unroll 1
        for (int c = 0; c < 8 && 32 * c < entries; ++c) MOE_VG_WORDS(list_at + 256 * c, from + 64 * c);
      }
      other_stage();
      if (kt + 1 < steps) read_a(0);
      copy_a(tail, 0);
      turn(first_step, 1, 0, !upper);
      --steps_left;
    };
    if (steps > 0) {
      read_a(0);                                               // (after the last tile's stores: they need the registers)
      step(std::true_type{}, any, std::integral_constant<int, kWhole>{}, 0);
      int kt = 1;
      if (R - m0 <= 128) {
#pragma unroll 1
        for (; kt < steps; ++kt) step(std::false_type{}, any, std::integral_constant<int, kUpper>{}, kt);
      }
      if (B_MNC && g.N - n0 <= 128) {
#pragma unroll 1
        for (; kt < steps; ++kt) step(std::false_type{}, any, std::integral_constant<int, kLeft>{}, kt);
      }
      if (TAIL) {                                              // (what a step copies lies within the next 128 k)
#pragma unroll 1
        for (; kt < steps && p_left >= 128; ++kt) step(std::false_type{}, std::false_type{}, std::integral_constant<int, kWhole>{}, kt);
      }
#pragma unroll 1
      for (; kt < steps; ++kt) step(std::false_type{}, any, std::integral_constant<int, kWhole>{}, kt);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = zeros;
    }

    // acc[2 h + i][j][4 q + r] = C[128 h + 64 wm + 32 i + r32][col(j) + 8 q + 4 hh + r] of the tile.  A wavefront's columns lie
    // together where both are stored as one line (logits); B's pieces are whole lines of a row of k where it is stored so.
    // Every copy started so far is awaited before the first store, so the next tile's first step has nothing to wait for.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int lane = lane_here(), r32 = lane & 31, hh = lane >> 5;
    auto col_of = [&](int j) { return B_MNC ? 128 * j + 32 * wn : 64 * wn + 32 * j; };
    if constexpr (EPI == kEntries) {
      // Logits at a teacher's entries, 256 at a time: each 32 x 32 part of the wavefront's that has any passes through LDS (the
      // register that holds an entry's logit differs from lane to lane).
      for (int done = 0; done < entries; done += 256) {
        const int n = entries - done < 256 ? entries - done : 256;
        if (done > 0)
          for (int at = lane; at < n; at += 64) {
            const uint2 e = list[done + at];
            *(lds_u2_ptr)(uintptr_t)(list_at + 8 * at) = u32x2_t{e.x, e.y};
          }
        __builtin_amdgcn_wave_barrier();
        // the first 64 in registers (there are seldom more), of the others the parts that they lie in
        auto part_of = [](uint32_t x) { return (int)(4 * (x >> 15 & 1) + 2 * (x >> 13 & 1) + (x >> 5 & 1)); };
        const uint32_t st = lds0 + kStaging + wave * 4096;
        auto store = [&](u32x2_t e) __attribute__((always_inline)) {
          const uint32_t row = e[0] >> 8, col = e[0] & 255;
          g.v.entry_logit[e[1]] = *(lds_f_ptr)(uintptr_t)(st + ((col >> 3) & 3) * 1024 +
                                                          ((row & 31) + 32 * ((col >> 2) & 1)) * 16 + (col & 3) * 4);
        };
        u32x2_t entry = {0u, 0u};
        if (lane < n) entry = *(lds_u2_ptr)(uintptr_t)(list_at + 8 * lane);
        const int part = lane < n ? part_of(entry[0]) : -1;
        int more = 0;
#pragma unroll 1
        for (int at = 64; at < n; at += 64) {
          const int p = at + lane < n ? part_of((*(lds_u2_ptr)(uintptr_t)(list_at + 8 * (at + lane)))[0]) : -1;
#pragma unroll
          for (int k = 0; k < 8; ++k) more |= __builtin_amdgcn_ballot_w64(p == k) != 0 ? 1 << k : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const bool here = part == 2 * i + j;
            if (__builtin_amdgcn_ballot_w64(here) == 0 && (more >> (2 * i + j) & 1) == 0) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *(lds_u4_ptr)(uintptr_t)(st + q * 1024 + lane * 16) =
                  u32x4_t{__float_as_uint(acc[i][j][4 * q]), __float_as_uint(acc[i][j][4 * q + 1]),
                          __float_as_uint(acc[i][j][4 * q + 2]), __float_as_uint(acc[i][j][4 * q + 3])};
            __builtin_amdgcn_wave_barrier();
            if (here) store(entry);
#pragma unroll 1
            for (int at = 64 + lane; at < n; at += 64) {
              const u32x2_t e = *(lds_u2_ptr)(uintptr_t)(list_at + 8 * at);
              if (part_of(e[0]) == 2 * i + j) store(e);
            }
            __builtin_amdgcn_wave_barrier();
          }
      }
    }
    if constexpr (EPI == kStats || EPI == kEntries) {
      const float c = g.v.scale;
      const int left = g.N - n0 - 64 * wn - 4 * hh;
      const uint32_t mine = lds0 + kStaging + wave * 4096;     // (maximum, sum) of 128 rows
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= 2 && R - m0 <= 128) continue;                 // (what is met below of these rows is not stored)
        float mx = -INFINITY;
        if constexpr (EPI == kStats) {                         // targets among these columns: few tiles have any
          const int t = *(lds_i_ptr)(uintptr_t)(hits + 256 * (i >> 1) + 4 * (32 * (i & 1) + r32)) - (n0 + 64 * wn) - 4 * hh;
          const bool in = t >= 0 && t < 64 && (t & 4) == 0;    // of this half's columns
          if (__builtin_amdgcn_ballot_w64(in) != 0) {
            float at = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[i][j][r] = take_column(acc[i][j][r], 32 * j + 8 * (r >> 2) + (r & 3), t, &at);
            const int row = m0 + 128 * (i >> 1) + 64 * wm + 32 * (i & 1) + r32;
            if (in && row < R) g.v.hit_value[row] = at;
          }
        }
        if (n0 + 256 > g.N) {
          int here = left;
          if (EPI == kStats) asm volatile("" : "+v"(here));    // (nor are these masks kept from one i to the next)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 32 * j + 8 * (r >> 2) + (r & 3) < here ? acc[i][j][r] : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[i][j][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
        const float m = fabsf(mx) == INFINITY ? 0.f : mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], c, -m));
        sum += __shfl_xor(sum, 32, 64);
        if (hh == 0)
          *(lds_u2_ptr)(uintptr_t)(mine + (32 * i + r32) * 8) =
              u32x2_t{__float_as_uint(mx == INFINITY ? 0.f : mx), __float_as_uint(sum)};
      }
      // the four column parts of the same rows (the wavefronts of one half) meet: each finishes 32 rows
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const uint32_t at = lds0 + kStaging + 4 * wm * 4096 + (32 * wn + r32) * 8;
      float m = -INFINITY, s = 0.f;
      u32x2_t o[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        o[w] = *(lds_u2_ptr)(uintptr_t)(at + w * 4096);
        m = fmaxf(m, __uint_as_float(o[w][0]));
      }
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int w = 0; w < 4; ++w) s += __uint_as_float(o[w][1]) * __builtin_amdgcn_exp2f(__uint_as_float(o[w][0]) - base);
      const int row = m0 + 128 * (wn >> 1) + 64 * wm + 32 * (wn & 1) + r32;
      if (hh == 0 && row < R) g.v.stats[(size_t)ct * g.R + row] = float2{m, s};
    } else if constexpr (EPI == kSums) {
      float* const C = static_cast<float*>(g.C) + (size_t)e * R * g.N;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = m0 + 128 * (i >> 1) + 64 * wm + 32 * (i & 1) + r32;
        if (row >= R) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int col = n0 + col_of(j) + 8 * q + 4 * hh;
            if (col >= g.N) continue;
            f32x4_t* const at = reinterpret_cast<f32x4_t*>(C + (size_t)row * g.N + col);
            f32x4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            if (g.add != 0) v += *at;
            *at = v;
          }
      }
    } else {
      // 32 rows of the 64 columns at a time through 4 KB of LDS into 16-byte stores: 16 rows in the wavefront's staging, 16 in A1
      // of the stage that is free, [rows][8 chunks of 8 columns], chunk c of row r at c ^ ((r >> 1) & 7), its halves swapped in
      // rows 16 .. 31 (each access then meets every bank as often as the others).
      const uint32_t free_a1 = lds0 + (to_other == kStage ? kStage : 0) + kPiece;      // of the step just done
      const uint32_t st = lds0 + kStaging + wave * 2048, st2 = free_a1 + wave * 2048 - 2048;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int in_tile = 128 * (i >> 1) + 64 * wm + 32 * (i & 1), row0 = m0 + in_tile;
        const uint32_t data = lds0 + kRowData + 4 * (in_tile + r32);
        if constexpr (EPI == kLogitGrad) {
          float lse = *(lds_f_ptr)(uintptr_t)data, up = *(lds_f_ptr)(uintptr_t)(data + 1024);
          if (row0 + r32 >= R) { lse = INFINITY; up = 0.f; }    // rows of zeros
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], g.v.scale, -lse)) * up;
          if (n0 + 256 > g.N) {
            const int left = g.N - n0 - 64 * wn - 4 * hh;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[i][j][r] = 32 * j + 8 * (r >> 2) + (r & 3) < left ? acc[i][j][r] : 0.f;
          }
        }
        const uint32_t wr = (r32 < 16 ? st : st2) + r32 * 128;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *(lds_u2_ptr)(uintptr_t)(wr + (((4 * j + q) ^ ((r32 >> 1) & 7)) * 16) + 8 * (hh ^ (r32 >> 4))) =
                u32x2_t{pack_bf16x2(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack_bf16x2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3])};
        if constexpr (EPI == kLogitGrad) {
          if (g.v.hit != nullptr && hh == 0 && row0 + r32 < R) {
            const int t = *(lds_i_ptr)(uintptr_t)(data + 2048) - (g.v.first + n0 + 64 * wn);   // the target's column, in its place
            if (t >= 0 && t < 64)
              *(lds_bf16_ptr)(uintptr_t)(wr + (((t >> 3) ^ ((r32 >> 1) & 7)) * 16) + 8 * (((t >> 2) & 1) ^ (r32 >> 4)) + 2 * (t & 3)) =
                  f32_to_bf16(*(lds_f_ptr)(uintptr_t)(data + 3 * 1024));
          }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int rr = 8 * s + (lane >> 3), c = lane & 7;
          u32x4_t d = *(lds_u4_ptr)(uintptr_t)((s < 2 ? st : st2) + rr * 128 + ((c ^ ((rr >> 1) & 7)) * 16));
          if (s >= 2) d = u32x4_t{d[2], d[3], d[0], d[1]};
          const int col = n0 + col_of(c >> 2) + 8 * (c & 3);
          bf16_t* const C = static_cast<bf16_t*>(g.C) + (size_t)(row0 + rr) * g.ldc + col;
          if ((EPI == kLogitGrad || row0 + rr < R) && col < g.N) {
            *reinterpret_cast<u32x4_t*>(C) = d;
          }
        }
      }
    }
  }
  if (wm == 0) __builtin_amdgcn_s_barrier();                   // the half phase
#undef MOE_VG_COPY
#undef MOE_VG_COPY_AT
#undef MOE_VG_WORDS
}

template <int EPI, bool TAIL>
int prepare_vocab_tiles() {
  static LdsLimitOnce once;
  return ensure_lds_limit(once, reinterpret_cast<const void*>(vocab_gemm_kernel<EPI, TAIL>), (int)kSmem);
}
template <int EPI, bool TAIL>
int launch_tiles(const VocabGemmArgs& g, long long tiles, hipStream_t st) {
  int cus = 0;
  if (prepare_vocab_tiles<EPI, TAIL>() != MOE_OK || compute_units(&cus) != MOE_OK) return MOE_EHIP;
  if (tiles > 0x7fffffffLL) return MOE_EUNSUPPORTED;
  hipLaunchKernelGGL((vocab_gemm_kernel<EPI, TAIL>), dim3((unsigned)(tiles < cus ? tiles : cus)), dim3(512), kSmem, st, g);
  return check_launch();
}
template <int EPI>
int launch_tiles(const VocabGemmArgs& g, long long tiles, bool tail, hipStream_t st) {
  return tail ? launch_tiles<EPI, true>(g, tiles, st) : launch_tiles<EPI, false>(g, tiles, st);
}
VocabGemmArgs args_of(const GemmArgs& a) {
  VocabGemmArgs g{};
  g.A = static_cast<const bf16_t*>(a.A);
  g.B = static_cast<const bf16_t*>(a.B);
  g.C = a.C;
  g.kept = a.kept;
  g.v = a.vocab;
  return g;
}
int tiles_of(int n) { return (n + 255) / 256; }

}  // namespace

int prepare_vocab_gemm() {
  const int rcs[] = {prepare_vocab_tiles<kStats, false>(),     prepare_vocab_tiles<kStats, true>(),
                     prepare_vocab_tiles<kEntries, false>(),   prepare_vocab_tiles<kEntries, true>(),
                     prepare_vocab_tiles<kLogitGrad, false>(), prepare_vocab_tiles<kLogitGrad, true>(),
                     prepare_vocab_tiles<kSums, false>(),      prepare_vocab_tiles<kSums, true>(),
                     prepare_vocab_tiles<kPlain, false>()};
  for (int rc : rcs)
    if (rc != MOE_OK) return rc;
  return MOE_OK;
}

int launch_vocab_tiles_logits(const GemmArgs& a, int rows, int entries, int M, hipStream_t st) {
  VocabGemmArgs g = args_of(a);
  g.lda = g.ldb = g.K = M;
  g.ldc = a.ldc;
  g.R = rows;
  g.N = entries;
  g.tiles_n = tiles_of(entries);
  const long long tiles = (long long)tiles_of(rows) * g.tiles_n;
  if (a.vocab.stats == nullptr) return launch_tiles<kLogitGrad>(g, tiles, M % 64 != 0, st);
  return a.vocab.hit != nullptr ? launch_tiles<kStats>(g, tiles, M % 64 != 0, st) : launch_tiles<kEntries>(g, tiles, M % 64 != 0, st);
}

int launch_vocab_tiles_dx(const GemmArgs& a, int M, hipStream_t st) {
  VocabGemmArgs g = args_of(a);
  g.lda = a.lda;
  g.ldb = g.N = M;
  g.k_total = a.k_total;
  g.add = a.add;
  g.tiles_n = tiles_of(M);
  // (how many tiles there are the device decides)
  return launch_tiles<kSums>(g, 0x7fffffff, a.k_total % 64 != 0, st);
}

int launch_vocab_tiles_dw(const GemmArgs& a, int entries, int M, hipStream_t st) {
  VocabGemmArgs g = args_of(a);
  g.lda = a.lda;
  g.ldb = g.ldc = g.N = M;
  g.R = entries;
  g.tiles_n = tiles_of(M);
  return launch_tiles<kPlain, false>(g, (long long)tiles_of(entries) * g.tiles_n, st);
}

}  // namespace moe
