// Attention of a decoder's tokens to an encoder's states on the matrix cores, forward and backward (bf16, d = 64 or 128).
//
//   ctx = softmax(q K^T / sqrt(d)) V over the states that a source holds;  with p = exp(score - lse), D = rowsum(dctx * ctx):
//   dV = p^T dctx,  ds = p * (dctx V^T - D) / sqrt(d),  dq = ds K,  dK = ds^T q
//
// The arrangement is that of attention_mfma.hip (everything transposed, a lane owns a column of a score tile; steps as lists of units).  What differs:
//
//   columns   Lq tokens times the `share` heads that use one key head: head k share + c % share of token c / share.  Heads that share
//             fill a tile of columns of few tokens, and the gradients of a shared head are one sum, in a fixed order.
//   states    a source's own number of them, read on the device.  Rows past it are staged as zeros and their probabilities are
//             0 (what memory holds there has no part); a source without any gives rows of zeros.
//   lse       is kept in units of log2 (fp32: natural): the exponentials of the backward pass are powers of two.
//   P, dS     are rounded to bf16 in front of the second products, as the self-attention of whole blocks does: three terms of them
//             (attention_mfma.hip, RAGGED) triple those products, and q, ctx and the results are rounded as much anyway.
//   pairs     where tokens are few (generation) q, P and ctx, backward dctx and dS, are pairs of bf16, 16 bits.  A wavefront's tile then has 16
//             columns, first terms in its columns 0 .. 15 and second ones in 16 .. 31: scores are the sums of both halves, P goes into the products as
//             both, ctx is the sum of both again.  That takes no more products or reads than a tile that few tokens do not fill, and as the lanes of
//             a pair share the exponentials, no more instructions.
//
// us (16 heads of 128, 32 x 1024 tokens and states): forward 338, dq 412, dK and dV 550, i.e. 0.81, 1.0 and 1.0 PFLOP/s; in turn with the self-attention's
// on two cards 335 and 349 (320, 328 there), 416 and 431 (392, 406), 572 and 596 (529, 549), 5 to 8 % behind; what bounds them is the same: the
// vector unit forward, the matrix pipes backward, at the 1.7 to 1.9 GHz that power leaves.  One token each of 64 sources of 410 to 2048 states: 141
// (4.7 TB/s).  For dK and dV, staging two blocks
// ahead was within 5 %; two groups of wavefronts with half the blocks each (d 64) made 46 us 54 at 308 blocks, 24 us 21 at 32.
#include <float.h>
#include <math.h>
#include "attention_tiles.h"
#include "cross_attention.h"

namespace moe {
namespace {

// rows of a block of 64 whose first is at `src`; rows from `rows` on are zeros
template <int D>
__device__ __forceinline__ void stage_rows(uint32_t lds, const bf16_t* src, int rows, const uint32_t (&off)[AttGeom<D>::kCopies], int q,
                                           int wave, int lane) {
  using GM = AttGeom<D>;
  lds += (wave * GM::kCopies + q) * 1024;
  if (rows < 64) {
    const int row = GM::kRowsPerCopy * (GM::kCopies * wave + q) + lane / GM::kChunks;
    const uint64_t at = row < rows ? (uint64_t)(uintptr_t)src + off[q] : (uint64_t)(uintptr_t)&att_zero_line;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off[q]), "s"(src) : "memory");
  }
}
// Per-lane byte offsets of this wavefront's copies of 64 columns (share divides 64).
template <int D>
__device__ __forceinline__ void column_offsets(uint32_t (&off)[AttGeom<D>::kCopies], const CrossCols& c, int wave, int lane) {
  using GM = AttGeom<D>;
#pragma unroll
  for (int q = 0; q < GM::kCopies; ++q) {
    const int row = GM::kRowsPerCopy * (GM::kCopies * wave + q) + lane / GM::kChunks;
    off[q] = (uint32_t)(c.offset<D>(row) * 2) + 16 * ((lane % GM::kChunks) ^ att_swizzle<D>(row));
  }
}
// Start the copies of the wavefront's own 32 CT rows to its own LDS block; address(row) is where row `row` is.
template <int D, int CT, typename F>
__device__ __forceinline__ void stage_own_rows(uint32_t lds, int lane, F&& address) {
  using GM = AttGeom<D>;
#pragma unroll
  for (int q = 0; q < 32 * CT * GM::kRow / 1024; ++q) {
    const int row = GM::kRowsPerCopy * q + lane / GM::kChunks;
    const uint64_t src = (uint64_t)(uintptr_t)(address(row) + 8 * ((lane % GM::kChunks) ^ att_swizzle<D>(row)));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + q * 1024), "v"(src) : "memory");
  }
}
// The wavefront's result tiles as whole rows, turned through its own LDS block: packed(c, dt, i) is bf16 of the values 2 i and 2 i + 1 of tile dt of
// the columns 32 c .. + 31; put(row, chunk, 16 bytes).
template <int D, int CT, typename P, typename F>
__device__ __forceinline__ void store_packed(P&& packed, uint32_t lds, int lane, F&& put) {
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
            u32x2_t{packed(c, dt, 2 * g), packed(c, dt, 2 * g + 1)};
#pragma unroll
  for (int q = 0; q < 32 * CT * GM::kRow / 1024; ++q) {
    const int row = GM::kRowsPerCopy * q + lane / GM::kChunks, chunk = lane % GM::kChunks;
    const u32x4_t v = *(lds_u4_ptr)(uintptr_t)(lds + row * GM::kRow + ((chunk ^ att_swizzle<D>(row)) << 4));
    put(row, chunk, v);
  }
}
// The tiles times factor.
template <int D, int CT, typename F>
__device__ __forceinline__ void store_rows(const f32x16_t (&acc)[CT][D / 32], float factor, uint32_t lds, int lane, F&& put) {
  store_packed<D, CT>([&](int c, int dt, int i) __attribute__((always_inline)) { return pack_bf16x2(acc[c][dt][2 * i] * factor, acc[c][dt][2 * i + 1] * factor); },
                      lds, lane, put);
}

// a b, rounded: the difference to a number that was computed so is exact
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
// the block's (source, key head), and the wavefront's first column, of blocks of PER columns, a quarter a wavefront
template <int PER> struct CrossWork {
  long long bk, b;
  int k, block0, col0, range;
  __device__ __forceinline__ CrossWork(int count, int kv_heads, int wave, unsigned ranges = 1) {
    const int blocks = (count + PER - 1) / PER;
    unsigned work = xcd_contiguous(blockIdx.x, gridDim.x);
    range = __builtin_amdgcn_readfirstlane(work % ranges);
    work /= ranges;
    const unsigned pair = work / blocks;
    bk = pair;
    k = __builtin_amdgcn_readfirstlane(pair % kv_heads);
    b = __builtin_amdgcn_readfirstlane(pair / kv_heads);
    block0 = __builtin_amdgcn_readfirstlane((int)(work % blocks) * PER);
    col0 = block0 + wave * (PER / 4);
  }
};

// zeros to the columns first .. first + PER - 1 of a block, 256 threads
template <int D, int PER = 128>
__device__ __forceinline__ void clear_columns(bf16_t* base, const CrossCols& c, int first) {
  for (int i = threadIdx.x; i < PER * (D / 8); i += 256) {
    const int col = first + i / (D / 8);
    if (col < c.count) *reinterpret_cast<u32x4_t*>(base + c.offset<D>(col) + 8 * (i % (D / 8))) = u32x4_t{0u, 0u, 0u, 0u};
  }
}

// Of a pair of columns c and c + 16, which lanes c and c + 16 hold (one row of 16 lanes and the next; a swap exchanges the odd rows of its first operand with
// the even ones of its second): the sums over the pair of two values, a's in the first lane and b's in the second.
__device__ __forceinline__ float pair_fold(float a, float b) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return pair_sum(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
// over the four lanes of a pair of columns
__device__ __forceinline__ float pair_max(float v) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const uint32_t m = __float_as_uint(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])));
  const auto y = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float pair_total(float v) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const uint32_t t = __float_as_uint(__uint_as_float(x[0]) + __uint_as_float(x[1]));
  const auto y = __builtin_amdgcn_permlane32_swap(t, t, false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}
// The way back for two numbers of each lane: those of the first lane (a) and of the second (b), as bf16 terms, first ones in the first lane.
struct PairTerms { uint32_t a, b; };
template <bool FINITE>
__device__ __forceinline__ PairTerms pair_terms(float x, float y) {
  const uint32_t rounded = pack_bf16x2(x, y);
  const uint32_t rest = FINITE ? pack_bf16x2(x - __uint_as_float(rounded << 16), y - __uint_as_float(rounded & 0xffff0000u)) : bf16_rest_x2(x, y, rounded);
  const auto f = __builtin_amdgcn_permlane16_swap(rounded, rest, false, false);
  return {f[0], f[1]};
}

// ---------------------------------------------------------------- forward
// PAIR: q + q_rest, ctx + ctx_rest.
template <int D, bool PAIR>
__global__ __launch_bounds__(256, 2) void cross_forward_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ q_rest,
                                                               const bf16_t* __restrict__ kv, const int32_t* __restrict__ src_len,
                                                               bf16_t* __restrict__ ctx, bf16_t* __restrict__ ctx_rest, float* __restrict__ lse) {
  using GM = AttGeom<D>;
  constexpr int CT = 1, KS = D / 16, DT = D / 32, kOwnBlock = 32 * CT * GM::kRow, kTile = PAIR ? 16 : 32;
  constexpr int kV = 2 * GM::kBlock;                           // LDS: two K blocks, two V blocks
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const bool second = PAIR && r >= 16;
  const CrossCols cols(g, D);
  const CrossWork<4 * kTile> w(cols.count, g.kv_heads, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk);
  if (n == 0) {
    clear_columns<D, 4 * kTile>(ctx + head, cols, w.block0);
    if constexpr (PAIR) clear_columns<D, 4 * kTile>(ctx_rest + head, cols, w.block0);
    if (lse != nullptr && threadIdx.x < 4 * kTile && w.block0 + (int)threadIdx.x < cols.count) lse[(size_t)w.bk * cols.count + w.block0 + threadIdx.x] = 0.f;
    return;
  }
  const int Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const bf16_t* const keys = kv + (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  const bool live = w.col0 < cols.count;

  uint32_t off[GM::kCopies];
  copy_offsets<D>(off, ld, wave, lane);
  const int nkb = (n + 63) / 64;
  // copy x of step j's: K block j + 1 (after the last one, that once more), V block j
  auto start = [&](int j, int x) __attribute__((always_inline)) {
    const int k = j + 1 < nkb ? j + 1 : nkb - 1, v = j;
    if (x < GM::kCopies) stage_rows<D>(lds0 + ((j + 1) & 1) * GM::kBlock, keys + (size_t)64 * k * ld, n - 64 * k, off, x, wave, lane);
    else stage_rows<D>(lds0 + kV + (j & 1) * GM::kBlock, keys + Akv + (size_t)64 * v * ld, n - 64 * v, off, x - GM::kCopies, wave, lane);
  };
  constexpr int COPIES = 2 * GM::kCopies;
  // the wavefront's own rows come (and its results go) through the second places of K and V
  const uint32_t own = GM::kBlock + (wave & 1) * kOwnBlock + (wave >> 1) * kV;
#pragma unroll
  for (int x = 0; x < GM::kCopies; ++x) { start(-1, x); start(0, GM::kCopies + x); }     // K and V block 0
  if (live)
    stage_own_rows<D, CT>(lds0 + own, lane, [&](int row) __attribute__((always_inline)) {
      return (row < kTile ? q : q_rest) + head + cols.offset<D>(cols.within(w.col0 + row % kTile));
    });
  wait_all_copies();

  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  const AttReads<D> rd(lds0, lane);
  u32x4_t qf[KS];                                              // Q^T fragments: lane (r, hf) holds d = 16 s + 8 hf .. + 7
  f32x16_t o[DT];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    qf[s] = rd.row(own, 0, s);
    asm volatile("" : "+v"(qf[s]) :: "memory");
  }
  __syncthreads();
  if (nkb > 1) {
#pragma unroll
    for (int x = 0; x < GM::kCopies; ++x) start(0, x);         // K block 1
  }
  if (!live) {                                                 // a wavefront without columns only stages
    for (int kb = 0; kb + 1 < nkb; ++kb) {
      wait_all_copies();
      __syncthreads();
#pragma unroll
      for (int x = 0; x < COPIES; ++x) start(kb + 1, x);
    }
    wait_all_copies();
    __syncthreads();
    __syncthreads();
    return;
  }
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  // running maximum (in log2 units) and sum; the maximum starts finite, so that a block of states whose scores
  // are all -inf adds nothing
  float m_run = -FLT_MAX, l_run = 0.f, m_new;
  // scores of block kb [32-state tile], and the maximum with them; PAIR: [0] only, of the tile 0 in the first lane of a pair and of 1 in the second
  f32x16_t sacc[2];
  auto mask_end = [&](f32x16_t (&acc)[2], int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < (PAIR ? 1 : 2); ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kb * 64 + 32 * (PAIR ? second : t) + 8 * (i >> 2) + 4 * hf + (i & 3) >= n) acc[t][i] = -INFINITY;
  };
  auto block_max = [&](const f32x16_t (&acc)[2]) __attribute__((always_inline)) {
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < (PAIR ? 1 : 2); ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, acc[t][i]);
    return mx;
  };
  auto fold4 = [&](f32x16_t (&acc)[2], int i4) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 4 * i4; i < 4 * i4 + 4; ++i) acc[0][i] = pair_fold(acc[0][i], acc[1][i]);
  };
  auto new_max = [&](float mx) __attribute__((always_inline)) {
    mx = PAIR ? pair_max(mx) : fmaxf(mx, __shfl_xor(mx, 32, 64));
    m_new = fmaxf(m_run, mx * sl2);                            // sl2 > 0: scaling commutes with max
  };
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < KS; ++s) sacc[t] = MOE_MFMA(rd.row(0, t, s), qf[s], s == 0 ? f32x16_t{} : sacc[t]);
  if constexpr (PAIR) {
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) fold4(sacc, i4);
  }
  if (64 > n) mask_end(sacc, 0);
  new_max(block_max(sacc));

  // One block of states; after the LAST there are no scores to multiply ahead.
  auto step = [&](int kb, auto last) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(last)::value;
    constexpr int FIRST = LAST ? 2 * KS : 0;                   // (units 0 .. 2 KS - 1 are those scores)
    wait_all_copies();                                         // K block kb + 1 and V block kb are there;
    __syncthreads();                                           // K block kb and V block kb - 1 are read, their places free
    const uint32_t kst = ((kb + 1) & 1) * GM::kBlock, vst = kV + (kb & 1) * GM::kBlock;
    // rescale only when some query of the wavefront needs it (alpha == 1 exactly otherwise)
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);   // 0 on the first block
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
    }
    m_run = m_new;
    float psum = 0.f, mx = -INFINITY;
    f32x16_t snext[2];
    constexpr int PF = PAIR ? 4 : 2;
    u32x4_t pf[PF];                                            // P^T, k step % PF
    // probabilities 2 i and 2 i + 1 of both lanes of a pair to the fragments of tile 0 and of tile 1
    auto terms = [&](int i) __attribute__((always_inline)) {
      const PairTerms p = pair_terms<true>(sacc[0][2 * i], sacc[0][2 * i + 1]);
      pf[i / 4][i % 4] = p.a;
      pf[(2 + i / 4) % PF][i % 4] = p.b;
    };
    auto exponentials = [&](int t, int from, int to) __attribute__((always_inline)) {
#pragma unroll
      for (int i = from; i < to; ++i) {
        const float v = __builtin_amdgcn_exp2f(fmaf(sacc[t][i], sl2, -m_run));
        sacc[t][i] = v;
        psum += v;
      }
    };
    if constexpr (LAST) {
      exponentials(0, 0, 16);
      if constexpr (PAIR) {
#pragma unroll
        for (int i = 0; i < 8; ++i) terms(i);
      } else {
        pf[0] = pack8(sacc[0], 0);
        pf[1] = pack8(sacc[0], 8);
      }
    }
    // units 0 .. 2 KS - 1: scores of block kb + 1, under them the first tile's exponentials; then 4 DT units of O^T, under
    // them the second tile's and the next block's maximum
    run_units<FIRST, 2 * KS + 4 * DT, 4>(
        [&](auto) __attribute__((always_inline)) { return std::integral_constant<int, 1>{}; },
        [&](auto U) __attribute__((always_inline)) {
          constexpr int u = decltype(U)::value, v = u - 2 * KS;
          if constexpr (u < 2 * KS) return rd.row(kst, u / KS, u % KS);
          else return rd.transposed(vst, 16 * (v / DT), v % DT);
        },
        [&](auto U, auto, const u32x4_t& f) __attribute__((always_inline)) {
          constexpr int u = decltype(U)::value, v = u - 2 * KS;
          if constexpr (u < 2 * KS) snext[u / KS] = MOE_MFMA(f, qf[u % KS], u % KS == 0 ? f32x16_t{} : snext[u / KS]);
          else o[v % DT] = MOE_MFMA(f, pf[(v / DT) % PF], o[v % DT]);
        },
        [&](auto U, auto, auto) __attribute__((always_inline)) {
          constexpr int u = decltype(U)::value, v = u - 2 * KS;
          if constexpr (!LAST && u < COPIES) start(kb + 1, u);
          if constexpr (u < 2 * KS) {
            exponentials(0, u * 8 / KS, (u + 1) * 8 / KS);
            if constexpr (PAIR) {                              // (two at a time: a swap's operands and results take wait states)
              if constexpr (u > 0 && u % (KS / 2) == 0) { terms(u / (KS / 2) * 2 - 2); terms(u / (KS / 2) * 2 - 1); }
            } else {
              if constexpr (u == KS + 1) pf[0] = pack8(sacc[0], 0);
              if constexpr (u == 2 * KS - 1) pf[1] = pack8(sacc[0], 8);
            }
          } else if constexpr (PAIR) {
            if constexpr (!LAST && v == 0) { terms(6); terms(7); }
            constexpr int gap = 4 * DT / 5, x = v - 1;         // four scores at a time (not right behind their last product), a unit later their maximum
            if constexpr (!LAST && x >= 0 && x % gap == 0 && x / gap < 4) {
              fold4(snext, x / gap);
            }
            if constexpr (!LAST && x >= 1 && (x - 1) % gap == 0 && (x - 1) / gap < 4) {
#pragma unroll
              for (int j = (x - 1) / gap * 4; j < (x - 1) / gap * 4 + 4; ++j) mx = fmaxf(mx, snext[0][j]);
            }
          } else if constexpr (v < 2 * DT) {
            exponentials(1, v * 16 / (2 * DT), (v + 1) * 16 / (2 * DT));
            // the fragment of k step 0 is free after DT units, the second tile's first 8 values done by then
            if constexpr (v == DT) pf[0] = pack8(sacc[1], 0);
          } else {
            if constexpr (v == 2 * DT) pf[1] = pack8(sacc[1], 8);
            constexpr int x = v - 2 * DT - 1, all = 2 * DT - 1;
            if constexpr (!LAST && x >= 0) {
#pragma unroll
              for (int j = x * 32 / all; j < (x + 1) * 32 / all; ++j) mx = fmaxf(mx, snext[j >> 4][j & 15]);
            }
          }
        });
    l_run += PAIR ? psum : psum + __shfl_xor(psum, 32, 64);    // PAIR: each lane's own, added up at the end
    if constexpr (LAST) return;
    if (kb + 2 == nkb && (n & 63) != 0) {                      // the last block comes next: without its rows past the end
      mask_end(snext, kb + 1);
      mx = block_max(snext);
    }
    new_max(mx);
    sacc[0] = snext[0];
    if constexpr (!PAIR) sacc[1] = snext[1];
  };
  for (int kb = 0; kb + 1 < nkb; ++kb) step(kb, std::false_type{});
  step(nkb - 1, std::true_type{});
  __syncthreads();                                             // the other wavefronts have read the last blocks
  const int c = w.col0 + r % kTile;
  // row statistic for the backward pass: log2 sum_k exp(score)
  const float l = PAIR ? pair_total(l_run) : l_run;
  if (lse != nullptr && hf == 0 && !second && c < cols.count) lse[(size_t)w.bk * cols.count + c] = m_run + log2f(l);
  const float inv = 1.0f / l;
  auto put = [&](int row, int chunk, const u32x4_t& v) __attribute__((always_inline)) {
    const int col = w.col0 + row % kTile;
    if (col < cols.count) *reinterpret_cast<u32x4_t*>((row < kTile ? ctx : ctx_rest) + head + cols.offset<D>(col) + 8 * chunk) = v;
  };
  if constexpr (PAIR) {                                        // tiles t and t + 1: the sums of the one in the first lane of a pair, of the other in the second
    uint32_t terms[DT][8];
#pragma unroll
    for (int t = 0; t < DT; t += 2)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const PairTerms p = pair_terms<false>(pair_fold(o[t][2 * i], o[t + 1][2 * i]) * inv, pair_fold(o[t][2 * i + 1], o[t + 1][2 * i + 1]) * inv);
        terms[t][i] = p.a;
        terms[t + 1][i] = p.b;
      }
    store_packed<D, CT>([&](int, int dt, int i) __attribute__((always_inline)) { return terms[dt][i]; }, lds0 + own, lane, put);
  } else {
    store_rows<D, CT>(reinterpret_cast<const f32x16_t (&)[1][DT]>(o), inv, lds0 + own, lane, put);
  }
}

// Start the copies of a wavefront's block of 32 states: rows of K, then of V, zeros from row `rows` on.
template <int D>
__device__ __forceinline__ void stage_few(uint32_t lds, const bf16_t* keys, int Akv, int rows, const uint32_t (&off)[32 * AttGeom<D>::kRow / 1024], int lane) {
  using GM = AttGeom<D>;
  constexpr int COPIES = 32 * GM::kRow / 1024;
#pragma unroll
  for (int x = 0; x < 2 * COPIES; ++x) {
    const bf16_t* const from = x < COPIES ? keys : keys + Akv;
    if (rows < 32) {
      const int i = GM::kRowsPerCopy * (x % COPIES) + lane / GM::kChunks;
      const uint64_t a = i < rows ? (uint64_t)(uintptr_t)from + off[x % COPIES] : (uint64_t)(uintptr_t)&att_zero_line;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + x * 1024), "v"(a) : "memory");
    } else {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds + x * 1024), "v"(off[x % COPIES]), "s"(from) : "memory");
    }
  }
}

// ---------------------------------------------------------------- forward of few columns
// A block's wavefronts share 32 columns and take blocks of 32 states in turn, each through two places of its own in LDS, one on its
// way while the other is used: no barrier, 64 KB (d 128) on their way to a compute unit.  Memory bounds it, so the products are
// not what counts: P keeps its 24 bits as three terms.
constexpr int kFewWaves = 4;
template <int D, bool PAIR>
__global__ __launch_bounds__(64 * kFewWaves, 1) void cross_few_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ q_rest,
                                                           const bf16_t* __restrict__ kv, const int32_t* __restrict__ src_len,
                                                           bf16_t* __restrict__ ctx, bf16_t* __restrict__ ctx_rest, float* __restrict__ lse,
                                                           CrossParts parts) {
  using GM = AttGeom<D>;
  constexpr int W = kFewWaves, KS = D / 16, DT = D / 32, kHalf = 32 * GM::kRow, kPlace = 2 * kHalf, COPIES = kHalf / 1024;      // K rows, V rows
  constexpr int kTile = PAIR ? 16 : 32;
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const bool second = PAIR && r >= 16;
  const CrossCols cols(g, D);
  const int tiles = (cols.count + kTile - 1) / kTile;
  unsigned item = xcd_contiguous(blockIdx.x, gridDim.x);
  const int split = __builtin_amdgcn_readfirstlane(item % parts.splits);
  item /= parts.splits;
  const unsigned pair = item / tiles;
  const int k = __builtin_amdgcn_readfirstlane(pair % g.kv_heads), b = __builtin_amdgcn_readfirstlane(pair / g.kv_heads);
  const int c = (int)(item % tiles) * kTile + r % kTile;
  const size_t row = cols.base(b, k, D) + cols.offset<D>(cols.within(c));
  u32x4_t qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const u32x4_t*>((second ? q_rest : q) + row + 16 * s + 8 * hf);
  const int n = held_states(src_len, b, g.Lk), Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const bf16_t* const keys = kv + (size_t)b * g.Lk * ld + (size_t)k * D;
  const int nkb = (n + 31) / 32, per = (nkb + parts.splits - 1) / parts.splits;
  const int from = split * per + wave, to = (split + 1) * per < nkb ? (split + 1) * per : nkb;

  uint32_t off[COPIES];
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const int at = GM::kRowsPerCopy * x + lane / GM::kChunks;
    off[x] = (uint32_t)(at * ld * 2) + 16 * ((lane % GM::kChunks) ^ att_swizzle<D>(at));
  }
  auto start = [&](int kb, int p) __attribute__((always_inline)) {
    stage_few<D>(lds0 + (2 * wave + p) * kPlace, keys + (size_t)32 * kb * ld, Akv, n - 32 * kb, off, lane);
  };
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  const AttReads<D> rd(lds0, lane);
  f32x16_t o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x16_t{};
  float m_run = -FLT_MAX, l_run = 0.f;                         // (finite: a block whose scores are all -inf adds nothing)
  if (from < to) start(from, 0);
  int p = 0;
  for (int kb = from; kb < to; kb += W, p ^= 1) {
    if (kb + W < to) {
      start(kb + W, p ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * COPIES) : "memory");
    } else {
      wait_all_copies();
    }
    const uint32_t place = (2 * wave + p) * kPlace;
    f32x16_t s;
#pragma unroll
    for (int i = 0; i < KS; ++i) s = MOE_MFMA(rd.row(place, 0, i), qf[i], i == 0 ? f32x16_t{} : s);
    // PAIR: the first lane of a pair has the scores of the block's first 16 states, the second one those of the others
    constexpr int VALUES = PAIR ? 8 : 16;
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = pair_fold(s[i], s[i + 8]);
    }
    float mx = -INFINITY, psum = 0.f;
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
      if (32 * kb + 16 * second + 8 * (i >> 2) + 4 * hf + (i & 3) >= n) s[i] = -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    mx = PAIR ? pair_max(mx) : fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx * sl2);
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
      m_run = m_new;
    }
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -m_run));
      psum += s[i];
    }
    l_run += PAIR ? pair_total(psum) : psum + __shfl_xor(psum, 32, 64);
    u32x4_t both[2];
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const PairTerms p = pair_terms<true>(s[2 * i], s[2 * i + 1]);
        both[0][i] = p.a;
        both[1][i] = p.b;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      constexpr int TERMS = PAIR ? 1 : 3;
      bf16x8_bits_t pf[TERMS];
      if constexpr (PAIR) pf[0] = both[h];
      else split_bf16x8(s, 8 * h, pf);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u32x4_t vt = rd.transposed(place + kHalf, 16 * h, dt);
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) o[dt] = MOE_MFMA(vt, pf[x], o[dt]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the place is read before the next copies go there
  }
  // To the wavefronts' common maximum; then each adds up 32 values of d.  LDS: [wavefront][DT][16][64] and the statistics behind
  typedef float __attribute__((address_space(3))) * lds_f_ptr;
  constexpr uint32_t kStats = W * DT * 16 * 64 * 4;
  __syncthreads();
  auto at = [&](uint32_t byte) __attribute__((always_inline)) { return (lds_f_ptr)(uintptr_t)(lds0 + byte); };
  *at(kStats + (wave * 64 + lane) * 4) = m_run;
  *at(kStats + 256 * W + (wave * 64 + lane) * 4) = l_run;
  __syncthreads();
  float m = m_run, l = 0.f;
#pragma unroll
  for (int x = 0; x < W; ++x) m = fmaxf(m, *at(kStats + (x * 64 + lane) * 4));
#pragma unroll
  for (int x = 0; x < W; ++x) l += *at(kStats + 256 * W + (x * 64 + lane) * 4) * __builtin_amdgcn_exp2f(*at(kStats + (x * 64 + lane) * 4) - m);
  const float alpha = __builtin_amdgcn_exp2f(m_run - m);       // (a wavefront without a block: sums of 0)
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) *at(((wave * DT + t) * 16 + i) * 256 + lane * 4) = o[t][i] * alpha;
  __syncthreads();
  if (c >= cols.count) return;
  const size_t column = ((size_t)b * g.kv_heads + k) * cols.count + c;
  if (wave == 0 && hf == 0 && !second) {
    if (parts.splits > 1) parts.stats[column * parts.splits + split] = float2{m, l};
    else if (lse != nullptr) lse[column] = n == 0 ? 0.f : m + log2f(l);
  }
  const float inv = n == 0 ? 0.f : 1.0f / l;
#pragma unroll
  for (int dt = wave; dt < DT; dt += W) {
    float v[16];                                               // d = 32 dt + 8 (i/4) + 4 hf + i%4 of column c
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int x = 0; x < W; ++x) v[i] += *at(((x * DT + dt) * 16 + i) * 256 + lane * 4);
      if constexpr (PAIR) v[i] = pair_fold(v[i], v[i]);
    }
    if (parts.splits > 1) {
      if (second) continue;
      float* const to_ = parts.sums + (column * parts.splits + split) * D + 32 * dt + 4 * hf;
#pragma unroll
      for (int x = 0; x < 4; ++x) *reinterpret_cast<f32x4_t*>(to_ + 8 * x) = f32x4_t{v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]};
    } else {
      if constexpr (PAIR) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] *= inv;
          v[i] = second ? bf16_rest(v[i], (float)(__bf16)v[i]) : v[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= inv;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<u32x2_t*>((second ? ctx_rest : ctx) + row + 32 * dt + 8 * x + 4 * hf) =
            u32x2_t{pack_bf16x2(v[4 * x], v[4 * x + 1]), pack_bf16x2(v[4 * x + 2], v[4 * x + 3])};
    }
  }
}

// The ranges of a column put together: a wavefront a column, lanes over the ranges (64 at most), then over d.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossGeo g, CrossParts parts, const int32_t* __restrict__ src_len, T* __restrict__ ctx,
                                                         T* __restrict__ ctx_rest, float* __restrict__ lse, long long columns) {
  constexpr bool F32 = sizeof(T) == 4;                         // (units of the maxima)
  const int lane = threadIdx.x & 63;
  const long long column = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (column >= columns) return;
  const CrossCols cols(g, D);
  const long long pair = column / cols.count, b = pair / g.kv_heads;
  const int c = (int)(column - pair * cols.count), k = (int)(pair - b * g.kv_heads);
  const float2 st = lane < parts.splits ? parts.stats[column * parts.splits + lane] : float2{-FLT_MAX, 0.f};
  const float m = wave_max(st.x);
  const float f = F32 ? expf(st.x - m) : __builtin_amdgcn_exp2f(st.x - m);
  const float l = wave_sum(st.y * f);
  float v[D / 64] = {};
  const float* const sums = parts.sums + column * parts.splits * D + lane * (D / 64);
  for (int s = 0; s < parts.splits; s += 8) {                  // eight on their way at a time
    float x[8][D / 64];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < D / 64; ++i) x[j][i] = s + j < parts.splits ? sums[(size_t)(s + j) * D + i] : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < D / 64; ++i) v[i] = fmaf(x[j][i], __shfl(f, s + j, 64), v[i]);
  }
  const bool none = held_states(src_len, b, g.Lk) == 0;
  if (lse != nullptr && lane == 0) lse[column] = none ? 0.f : F32 ? m + logf(l) : m + log2f(l);
  const float inv = none ? 0.f : 1.0f / l;
  const size_t to = cols.base(b, k, D) + cols.offset<D>(c) + lane * (D / 64);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    Elt<T>::store(ctx + to + i, v[i] * inv);
    if constexpr (!F32)
      if (ctx_rest != nullptr) Elt<T>::store(ctx_rest + to + i, bf16_rest(v[i] * inv, (float)(__bf16)(v[i] * inv)));
  }
}

// ---------------------------------------------------------------- dq (and D) of up to 64 states
// D = sum p dP of the probabilities at hand.  Of few states dP - D is a difference of near numbers, of whose error the rounding of the stored ctx, in
// rowsum(dO * ctx), is more than half (two states: dq off by 0.0053 in norm, 0.0038 without it); of one it is 0, as it is here to the last
// bit: p is exactly 1.  What a source holds decides, not what its batch is padded to, so every kernel of dq has this form of its own and padding
// changes no bits.  K and V are two blocks of 32 rows each, zeros from n on: K's first at k0, V's at v0, the second ones `step` behind.
// PAIR: of columns in pairs; dq is rounded by the caller, the sums of both terms in both lanes.
template <int D, bool PAIR = false>
__device__ __forceinline__ void few_states_dq(f32x16_t (&dq)[D / 32], float& dd, const AttReads<D>& rd, uint32_t k0, uint32_t v0, uint32_t step,
                                              const u32x4_t (&qf)[D / 16], const u32x4_t (&dof)[D / 16], int n, int hf, bool second = false) {
  constexpr int KS = D / 16, DT = D / 32, T = PAIR ? 1 : 2;    // PAIR: the first lane has the first 32 states, the second one the others
  const float sl2 = 1.4426950408889634f / sqrtf((float)D);
  f32x16_t sc[2], dp[2];
  float m = -FLT_MAX, sum = 0.f, dsum = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      sc[t] = MOE_MFMA(rd.row(k0 + t * step, 0, x), qf[x], x == 0 ? f32x16_t{} : sc[t]);
      dp[t] = MOE_MFMA(rd.row(v0 + t * step, 0, x), dof[x], x == 0 ? f32x16_t{} : dp[t]);
    }
  if constexpr (PAIR) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[0][i] = pair_fold(sc[0][i], sc[1][i]);
      dp[0][i] = pair_fold(dp[0][i], dp[1][i]);
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[t][i] = 32 * (PAIR ? second : t) + 8 * (i >> 2) + 4 * hf + (i & 3) < n ? rounded_product(sc[t][i], sl2) : -INFINITY;
      m = fmaxf(m, sc[t][i]);
    }
  m = PAIR ? pair_max(m) : fmaxf(m, __shfl_xor(m, 32, 64));
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[t][i] = __builtin_amdgcn_exp2f(sc[t][i] - m);
      sum += sc[t][i];
      dsum += sc[t][i] * dp[t][i];
    }
  sum = PAIR ? pair_total(sum) : sum + __shfl_xor(sum, 32, 64);
  dsum = PAIR ? pair_total(dsum) : dsum + __shfl_xor(dsum, 32, 64);
  const float inv = 1.0f / sum;
  dd = dsum * inv;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dq[dt] = f32x16_t{};
  u32x4_t f[2][2];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[t][i] *= inv * (dp[t][i] - dd);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const PairTerms p = pair_terms<false>(sc[0][8 * x + 2 * i], sc[0][8 * x + 2 * i + 1]);
        f[0][x][i] = p.a;
        f[1][x][i] = p.b;
      }
    } else {
      f[0][x] = pack8(sc[0], 8 * x);
      f[1][x] = pack8(sc[1], 8 * x);
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dq[dt] = MOE_MFMA(rd.transposed(k0 + t * step, 16 * x, dt), f[t][x], dq[dt]);
  if constexpr (PAIR) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) dq[dt][i] = pair_fold(dq[dt][i], dq[dt][i]);
  }
}
// A block of 128 columns of such a source.  K and V lie in LDS whole, the columns' rows come straight from memory.
template <int D>
__device__ __forceinline__ void few_states_block(const CrossCols& cols, const CrossWork<128>& w, size_t head, int n, int Akv,
                                                 const uint32_t (&off)[AttGeom<D>::kCopies], const bf16_t* q, const bf16_t* keys,
                                                 const bf16_t* dctx, bf16_t* dqo, float* dvec, uint32_t lds0, int wave, int lane) {
  using GM = AttGeom<D>;
  constexpr int CT = 1, KS = D / 16, DT = D / 32, kOwnBlock = 32 * CT * GM::kRow, kV = GM::kBlock;
  const int r = lane & 31, hf = lane >> 5;
  const bool live = w.col0 < cols.count;
#pragma unroll
  for (int x = 0; x < GM::kCopies; ++x) {
    stage_rows<D>(lds0, keys, n, off, x, wave, lane);
    stage_rows<D>(lds0 + kV, keys + Akv, n, off, x, wave, lane);
  }
  const size_t row = head + cols.offset<D>(cols.within(w.col0 + r));
  u32x4_t qf[KS], dof[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    qf[s] = *reinterpret_cast<const u32x4_t*>(q + row + 16 * s + 8 * hf);
    dof[s] = *reinterpret_cast<const u32x4_t*>(dctx + row + 16 * s + 8 * hf);
  }
  wait_all_copies();
  __syncthreads();
  f32x16_t dq[CT][DT];
  if (live) {
    float dd;
    few_states_dq<D>(dq[0], dd, AttReads<D>(lds0, lane), 0, kV, kOwnBlock, qf, dof, n, hf);
    if (hf == 0 && w.col0 + r < cols.count) dvec[(size_t)w.bk * cols.count + w.col0 + r] = dd;
  }
  __syncthreads();                                             // K and V are read: the results go through their places
  if (!live) return;
  store_rows<D, CT>(dq, 1.0f / sqrtf((float)D), lds0 + wave * kOwnBlock, lane, [&](int i, int chunk, const u32x4_t& v) __attribute__((always_inline)) {
    if (w.col0 + i < cols.count) *reinterpret_cast<u32x4_t*>(dqo + head + cols.offset<D>(w.col0 + i) + 8 * chunk) = v;
  });
}
// All sources of a call have up to 64 states.
template <int D>
__global__ __launch_bounds__(256, 2) void cross_dq_short_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ kv,
                                                                const int32_t* __restrict__ src_len, const bf16_t* __restrict__ dctx,
                                                                bf16_t* __restrict__ dqo, float* __restrict__ dvec) {
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const CrossCols cols(g, D);
  const CrossWork<128> w(cols.count, g.kv_heads, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk), Akv = g.kv_heads * D;
  if (n == 0) {                                                // (no state asks for D)
    clear_columns<D>(dqo + head, cols, w.block0);
    return;
  }
  uint32_t off[AttGeom<D>::kCopies];
  copy_offsets<D>(off, (size_t)2 * Akv, wave, lane);
  few_states_block<D>(cols, w, head, n, Akv, off, q, kv + (size_t)w.b * g.Lk * 2 * Akv + (size_t)w.k * D, dctx, dqo, dvec, lds0, wave, lane);
}

// ---------------------------------------------------------------- dq (and D)
template <int D>
__global__ __launch_bounds__(256, 2) void cross_dq_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ kv,
                                                          const int32_t* __restrict__ src_len, const bf16_t* __restrict__ ctx,
                                                          const bf16_t* __restrict__ dctx, const float* __restrict__ lse,
                                                          bf16_t* __restrict__ dqo, float* __restrict__ dvec) {
  using GM = AttGeom<D>;
  constexpr int CT = 1, KS = D / 16, DT = D / 32, kOwnBlock = 32 * CT * GM::kRow;
  // LDS: three K blocks, two V blocks; the wavefronts' own rows go through all of their places but the first, so that
  // two blocks share a compute unit
  constexpr int kV = 3 * GM::kBlock, kQ = GM::kBlock, kGrad = kQ + 4 * kOwnBlock;
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const CrossCols cols(g, D);
  const CrossWork<128 * CT> w(cols.count, g.kv_heads, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk);
  if (n == 0) {                                                // (no state asks for D)
    clear_columns<D>(dqo + head, cols, w.block0);
    return;
  }
  const int Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const bf16_t* const keys = kv + (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  const bool live = w.col0 < cols.count;

  uint32_t off[GM::kCopies];
  copy_offsets<D>(off, ld, wave, lane);
  if (n <= 64) {
    few_states_block<D>(cols, w, head, n, Akv, off, q, keys, dctx, dqo, dvec, lds0, wave, lane);
    return;
  }
  const int nkb = (n + 63) / 64;
  // copy x of step j's: K block j + 1 to place `slot`, V block j (after the last ones, those once more)
  auto start = [&](int j, int slot, int x) __attribute__((always_inline)) {
    const int k = j + 1 < nkb ? j + 1 : nkb - 1, v = j < nkb ? j : nkb - 1;
    if (x < GM::kCopies) stage_rows<D>(lds0 + slot * GM::kBlock, keys + (size_t)64 * k * ld, n - 64 * k, off, x, wave, lane);
    else stage_rows<D>(lds0 + kV + (j & 1) * GM::kBlock, keys + Akv + (size_t)64 * v * ld, n - 64 * v, off, x - GM::kCopies, wave, lane);
  };
  constexpr int COPIES = 2 * GM::kCopies;

  // Q^T and dO^T fragments of this wavefront's columns, D and lse of the lane's.  The rows come through LDS: read as
  // fragments from memory, 16 bytes of 32 rows at a time, they take longer (O, one of three, hides behind the others).
  const uint32_t own = kQ + wave * kOwnBlock;
  const float scale = 1.0f / sqrtf((float)D), sl2 = 1.4426950408889634f * scale;
  const AttReads<D> rd(lds0, lane);
  u32x4_t qf[KS], dof[KS], of[KS];
#pragma unroll
  for (int x = 0; x < GM::kCopies; ++x) start(-1, 0, x);       // K block 0
  if (live) {
    auto column = [&](int row) __attribute__((always_inline)) { return head + cols.offset<D>(cols.within(w.col0 + row)); };
    stage_own_rows<D, CT>(lds0 + own, lane, [&](int row) __attribute__((always_inline)) { return q + column(row); });
    stage_own_rows<D, CT>(lds0 + kGrad + wave * kOwnBlock, lane, [&](int row) __attribute__((always_inline)) { return dctx + column(row); });
    const bf16_t* const orow = ctx + column(r);
#pragma unroll
    for (int s = 0; s < KS; ++s) of[s] = *reinterpret_cast<const u32x4_t*>(orow + 16 * s + 8 * hf);
    wait_all_copies();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = rd.row(own, 0, s);
      dof[s] = rd.row(kGrad + wave * kOwnBlock, 0, s);
      asm volatile("" : "+a"(qf[s]), "+a"(dof[s]) :: "memory");
      asm volatile("" : "+v"(of[s]));
    }
  }
  wait_all_copies();
  __syncthreads();
#pragma unroll
  for (int x = 0; x < COPIES; ++x) start(0, 1, x);             // K block 1 and V block 0

  if (!live) {                                                 // a wavefront without columns only stages
    for (int kb = 0, k2 = 2; kb < nkb; ++kb) {
      wait_all_copies();
      __syncthreads();
      if (kb + 1 < nkb) {
#pragma unroll
        for (int x = 0; x < COPIES; ++x) start(kb + 1, k2, x);
      }
      k2 = k2 == 2 ? 0 : k2 + 1;
    }
    wait_all_copies();
    __syncthreads();
    return;
  }
  f32x16_t dq[CT][DT];
  float dd = 0.f, lse2;
  {
    const int c = w.col0 + r;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float gr[8], ov[8];
      Vec16<bf16_t>::unpack(uint4{dof[s][0], dof[s][1], dof[s][2], dof[s][3]}, gr);
      Vec16<bf16_t>::unpack(uint4{of[s][0], of[s][1], of[s][2], of[s][3]}, ov);
#pragma unroll
      for (int i = 0; i < 8; ++i) dd = fmaf(gr[i], ov[i], dd);
    }
    dd += __shfl_xor(dd, 32, 64);
    if (hf == 0 && c < cols.count) dvec[(size_t)w.bk * cols.count + c] = dd;
    lse2 = lse[(size_t)w.bk * cols.count + cols.within(c)];
#pragma unroll
    for (int t = 0; t < DT; ++t) clear_acc(dq[0][t]);
  }
  asm volatile("" : "+v"(lse2));                               // loaded here, not waited for in the loop
  f32x16_t sacc;                                               // scores of 32 states
#pragma unroll
  for (int s = 0; s < KS; ++s) sacc = MOE_MFMA(rd.row(0, 0, s), qf[s], s == 0 ? f32x16_t{} : sacc);

  int k0 = 0;                                                  // place of K block kb
  // One block of states; LAST: nothing follows.
  auto step = [&](int kb, auto last) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(last)::value;
    wait_all_copies();                                         // K block kb + 1 and V block kb are there;
    __syncthreads();                                           // K and V block kb - 1 are read, their places free
    const int k1 = k0 == 2 ? 0 : k0 + 1, k2 = k1 == 2 ? 0 : k1 + 1;
    const uint32_t kst = k0 * GM::kBlock, knext = k1 * GM::kBlock, vst = kV + (kb & 1) * GM::kBlock;
    f32x16_t dpacc, snext;
    u32x4_t dsf[2];                                            // [k step]
    // per 32 states: KS units of dP, under them P; KS of the next 32 states' scores (unless there are none),
    // under them dS; 2 DT of dQ
    constexpr int UNITS = 2 * KS + 2 * DT;
    run_units<0, 2 * UNITS, 4>(
        [&](auto) __attribute__((always_inline)) { return std::integral_constant<int, 1>{}; },
        [&](auto U) __attribute__((always_inline)) {
          constexpr int t = decltype(U)::value / UNITS, u = decltype(U)::value % UNITS, v = u - 2 * KS;
          if constexpr (u < KS) return rd.row(vst, t, u);
          else if constexpr (u < 2 * KS) return rd.row(t == 0 ? kst : knext, 1 - t, u - KS);
          else return rd.transposed(kst, 32 * t + 16 * (v / DT), v % DT);
        },
        [&](auto U, auto, const u32x4_t& f) __attribute__((always_inline)) {
          constexpr int t = decltype(U)::value / UNITS, u = decltype(U)::value % UNITS, v = u - 2 * KS;
          if constexpr (LAST && t == 1 && u >= KS && u < 2 * KS) return;         // (no scores to multiply ahead)
          if constexpr (u < KS) dpacc = MOE_MFMA(f, dof[u], u == 0 ? f32x16_t{} : dpacc);
          else if constexpr (u < 2 * KS) snext = MOE_MFMA(f, qf[u - KS], u == KS ? f32x16_t{} : snext);
          else {
            if constexpr (v % DT == 0) fresh_operand();
            mfma_acc(dq[0][v % DT], f, dsf[v / DT]);
          }
        },
        [&](auto U, auto, auto) __attribute__((always_inline)) {
          constexpr int t = decltype(U)::value / UNITS, u = decltype(U)::value % UNITS;
          if constexpr (!LAST && decltype(U)::value < COPIES) start(kb + 1, k2, decltype(U)::value);
          if constexpr (u < KS) {
#pragma unroll
            for (int j = u * 16 / KS; j < (u + 1) * 16 / KS; ++j) sacc[j] = __builtin_amdgcn_exp2f(fmaf(sacc[j], sl2, -lse2));
            if constexpr (LAST && u == KS - 1) {               // (dP of a row of zeros is 0, D is not)
              if ((n & 63) != 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  if (kb * 64 + 32 * t + 8 * (i >> 2) + 4 * hf + (i & 3) >= n) sacc[i] = 0.f;
              }
            }
          } else if constexpr (u < 2 * KS) {
            constexpr int x = u - KS - 1, all = KS - 1;        // (not right behind dP's last product)
            if constexpr (x >= 0) {
#pragma unroll
              for (int j = x * 16 / all; j < (x + 1) * 16 / all; ++j) sacc[j] = sacc[j] * (dpacc[j] - dd);
            }
            if constexpr (u == KS + KS / 2 + 1) dsf[0] = pack8(sacc, 0);
          } else if constexpr (u == 2 * KS) {
            dsf[1] = pack8(sacc, 8);
          }
          if constexpr (u == UNITS - 1) sacc = snext;
        });
    k0 = k1;
  };
  for (int kb = 0; kb + 1 < nkb; ++kb) step(kb, std::false_type{});
  step(nkb - 1, std::true_type{});
  settle_all(dq);
  __syncthreads();                                             // the other wavefronts have read the last blocks
  store_rows<D, CT>(dq, scale, lds0 + own, lane, [&](int row, int chunk, const u32x4_t& v) __attribute__((always_inline)) {
    if (w.col0 + row < cols.count) *reinterpret_cast<u32x4_t*>(dqo + head + cols.offset<D>(w.col0 + row) + 8 * chunk) = v;
  });
}

// ---------------------------------------------------------------- dq (and D) of few columns
// As the forward pass of few columns: 32 of them a block, whose wavefronts take blocks of 32 states in turn and add up their sums at the end.  A
// wavefront's chain of blocks bounds it (40.5 -> 22.6 us for 1 x 128 tokens of 4 heads of 128, 1500 states: 16 blocks instead of 4, a quarter of the states each).
// PAIR: q, ctx and dctx in pairs, and so dS; rest: their second terms.
struct CrossRest { const bf16_t *q, *ctx, *dctx; };
template <int D, bool PAIR>
__global__ __launch_bounds__(64 * kFewWaves, 1) void cross_dq_few_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ kv,
                                                              const int32_t* __restrict__ src_len, const bf16_t* __restrict__ ctx,
                                                              const bf16_t* __restrict__ dctx, const float* __restrict__ lse,
                                                              bf16_t* __restrict__ dqo, float* __restrict__ dvec, CrossRest rest) {
  using GM = AttGeom<D>;
  constexpr int W = kFewWaves, KS = D / 16, DT = D / 32, kHalf = 32 * GM::kRow, kPlace = 2 * kHalf, COPIES = kHalf / 1024;
  constexpr int kTile = PAIR ? 16 : 32;
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const bool second = PAIR && r >= 16;
  const CrossCols cols(g, D);
  const int tiles = (cols.count + kTile - 1) / kTile;
  const unsigned item = xcd_contiguous(blockIdx.x, gridDim.x), pair = item / tiles;
  const int k = __builtin_amdgcn_readfirstlane(pair % g.kv_heads), b = __builtin_amdgcn_readfirstlane(pair / g.kv_heads);
  const int c = (int)(item % tiles) * kTile + r % kTile;
  const size_t row = cols.base(b, k, D) + cols.offset<D>(cols.within(c));
  const size_t column = ((size_t)b * g.kv_heads + k) * cols.count + cols.within(c);
  const int n = held_states(src_len, b, g.Lk), Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const bf16_t* const keys = kv + (size_t)b * g.Lk * ld + (size_t)k * D;
  const int nkb = (n + 31) / 32;
  uint32_t off[COPIES];
#pragma unroll
  for (int x = 0; x < COPIES; ++x) {
    const int at = GM::kRowsPerCopy * x + lane / GM::kChunks;
    off[x] = (uint32_t)(at * ld * 2) + 16 * ((lane % GM::kChunks) ^ att_swizzle<D>(at));
  }
  auto start = [&](int kb, int p) __attribute__((always_inline)) {
    stage_few<D>(lds0 + (2 * wave + p) * kPlace, keys + (size_t)32 * kb * ld, Akv, n - 32 * kb, off, lane);
  };
  u32x4_t qf[KS], dof[KS];
  float dd = 0.f;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const size_t at = row + 16 * s + 8 * hf;
    qf[s] = *reinterpret_cast<const u32x4_t*>((second ? rest.q : q) + at);
    dof[s] = *reinterpret_cast<const u32x4_t*>((second ? rest.dctx : dctx) + at);
    float gr[8], ov[8];
    Vec16<bf16_t>::unpack(*reinterpret_cast<const uint4*>(ctx + at), ov);
    if constexpr (PAIR) {
      float gr2[8], ov2[8];
      Vec16<bf16_t>::unpack(*reinterpret_cast<const uint4*>(dctx + at), gr);
      Vec16<bf16_t>::unpack(*reinterpret_cast<const uint4*>(rest.dctx + at), gr2);
      Vec16<bf16_t>::unpack(*reinterpret_cast<const uint4*>(rest.ctx + at), ov2);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        gr[i] += gr2[i];
        ov[i] += ov2[i];
      }
    } else {
      Vec16<bf16_t>::unpack(uint4{dof[s][0], dof[s][1], dof[s][2], dof[s][3]}, gr);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) dd = fmaf(gr[i], ov[i], dd);
  }
  dd += __shfl_xor(dd, 32, 64);
  const float scale = 1.0f / sqrtf((float)D), sl2 = 1.4426950408889634f * scale;
  const AttReads<D> rd(lds0, lane);
  f32x16_t dq[DT];
  if (n > 0 && n <= 64) {                                      // block-uniform: one wavefront has both blocks of states
    if (wave > 0) return;
    start(0, 0);
    start(1, 1);
    wait_all_copies();
    few_states_dq<D, PAIR>(dq, dd, rd, 0, kHalf, kPlace, qf, dof, n, hf, second);
    if (c >= cols.count || second) return;
    if (hf == 0) dvec[column] = dd;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<u32x2_t*>(dqo + row + 32 * dt + 8 * x + 4 * hf) =
            u32x2_t{pack_bf16x2(dq[dt][4 * x] * scale, dq[dt][4 * x + 1] * scale), pack_bf16x2(dq[dt][4 * x + 2] * scale, dq[dt][4 * x + 3] * scale)};
    return;
  }
  const float lse2 = lse[column];
#pragma unroll
  for (int t = 0; t < DT; ++t) dq[t] = f32x16_t{};
  if (wave < nkb) start(wave, 0);
  int p = 0;
  for (int kb = wave; kb < nkb; kb += W, p ^= 1) {
    if (kb + W < nkb) {
      start(kb + W, p ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * COPIES) : "memory");
    } else {
      wait_all_copies();
    }
    const uint32_t place = (2 * wave + p) * kPlace;
    f32x16_t s, dp;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = MOE_MFMA(rd.row(place, 0, i), qf[i], i == 0 ? f32x16_t{} : s);
      dp = MOE_MFMA(rd.row(place + kHalf, 0, i), dof[i], i == 0 ? f32x16_t{} : dp);
    }
    if constexpr (PAIR) {                                      // the first lane has the block's first 16 states, the second one the others
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i] = pair_fold(s[i], s[i + 8]);
        dp[i] = pair_fold(dp[i], dp[i + 8]);
      }
    }
#pragma unroll
    for (int i = 0; i < (PAIR ? 8 : 16); ++i) {
      const float e = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -lse2)) * (dp[i] - dd);
      s[i] = 32 * kb + 16 * second + 8 * (i >> 2) + 4 * hf + (i & 3) >= n ? 0.f : e;
    }
    u32x4_t both[2];
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const PairTerms p = pair_terms<false>(s[2 * i], s[2 * i + 1]);
        both[0][i] = p.a;
        both[1][i] = p.b;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4_t dsf = PAIR ? both[h] : pack8(s, 8 * h);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dq[dt] = MOE_MFMA(rd.transposed(place, 16 * h, dt), dsf, dq[dt]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the place is read before the next copies go there
  }
  // LDS: [wavefront][DT][16][64]; each wavefront adds up 32 values of d
  typedef float __attribute__((address_space(3))) * lds_f_ptr;
  auto at = [&](uint32_t byte) __attribute__((always_inline)) { return (lds_f_ptr)(uintptr_t)(lds0 + byte); };
  __syncthreads();
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) *at(((wave * DT + t) * 16 + i) * 256 + lane * 4) = dq[t][i];
  __syncthreads();
  if (c >= cols.count) return;
  if (wave == 0 && hf == 0 && !second) dvec[column] = dd;
#pragma unroll
  for (int dt = wave; dt < DT; dt += W) {
    float v[16];                                               // d = 32 dt + 8 (i/4) + 4 hf + i%4 of column c
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int x = 0; x < W; ++x) v[i] += *at(((x * DT + dt) * 16 + i) * 256 + lane * 4);
      if constexpr (PAIR) v[i] = pair_fold(v[i], v[i]);
      v[i] *= scale;
    }
    if (second) continue;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<u32x2_t*>(dqo + row + 32 * dt + 8 * x + 4 * hf) =
          u32x2_t{pack_bf16x2(v[4 * x], v[4 * x + 1]), pack_bf16x2(v[4 * x + 2], v[4 * x + 3])};
  }
}

// ---------------------------------------------------------------- dK, dV
// RANGES: of a range of the columns, as fp32 sums, which one more launch adds up in order.
struct CrossRanges {
  int count, blocks;         // ranges, and the blocks of 64 columns of each (the last may have fewer, none has none)
  size_t elems;              // of dkv
  float* sums;               // [ranges][dkv]
};
// PAIR: blocks of 32 columns, rows 0 .. 31 of a staged block first terms and 32 .. 63 second ones; P and dS in pairs too.
template <int D, int CT, bool RANGES = false, bool PAIR = false>
__global__ __launch_bounds__(256, 1) void cross_dkv_kernel(CrossGeo g, const bf16_t* __restrict__ q, const bf16_t* __restrict__ kv,
                                                           const int32_t* __restrict__ src_len, const bf16_t* __restrict__ dctx,
                                                           const float* __restrict__ lse, const float* __restrict__ dvec,
                                                           bf16_t* __restrict__ dkv, CrossRanges ranges, CrossRest rest) {
  static_assert(!PAIR || CT == 1, "");
  using GM = AttGeom<D>;
  constexpr int KS = D / 16, DT = D / 32, kOwnBlock = 32 * CT * GM::kRow;
  constexpr int kGrad = GM::kBlock, kStats = 2 * GM::kBlock, kStage = kStats + 512;   // Q rows, dO rows, 64 lse, 64 D
  constexpr int kColumns = PAIR ? 32 : 64;
  constexpr bool kValuesInLds = D == 128 && (CT == 2 || PAIR); // there both operands' fragments and both results are
  constexpr int kOwn = 2 * kStage;                             // 384 registers, too many beside S and dP
  extern __shared__ __attribute__((aligned(256))) unsigned char att_lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_ptr)att_lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const CrossCols cols(g, D);
  const CrossWork<128 * CT> w(g.Lk, g.kv_heads, wave, RANGES ? ranges.count : 1);
  const int n = held_states(src_len, w.b, g.Lk), Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const size_t states = (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  // zeros to the rows first .. first + count - 1 that there are, by `threads` threads of which this is number i0
  using Out = std::conditional_t<RANGES, float, bf16_t>;
  Out* out;
  if constexpr (RANGES) out = ranges.sums + w.range * ranges.elems + states;
  else out = dkv + states;
  auto clear = [&](int first, int count, int i0, int threads) __attribute__((always_inline)) {
    constexpr int E = 16 / sizeof(Out);
    for (int i = i0; i < count * (D / E); i += threads) {
      const int row = first + i / (D / E);
      if (row >= g.Lk) return;
      Out* const at = out + (size_t)row * ld + E * (i % (D / E));
      *reinterpret_cast<u32x4_t*>(at) = u32x4_t{0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4_t*>(at + Akv) = u32x4_t{0u, 0u, 0u, 0u};
    }
  };
  if (w.block0 >= n) {
    clear(w.block0, 128 * CT, threadIdx.x, 256);
    return;
  }
  const size_t head = cols.base(w.b, w.k, D);
  const bool second = PAIR && wave >= 2;
  const bf16_t *const qbase = (second ? rest.q : q) + head, *const gbase = (second ? rest.dctx : dctx) + head;
  const float* const stat = (wave & 1 ? dvec : lse) + (size_t)w.bk * cols.count;      // (two wavefronts copy the same 64 values)
  const bool live = w.col0 < n;

  uint32_t off[GM::kCopies];
  const int row_wave = PAIR ? wave & 1 : wave;                 // whose rows of a block of columns the wavefront copies
  column_offsets<D>(off, cols, row_wave, lane);
  int qb0 = 0, nqb = (cols.count + kColumns - 1) / kColumns;
  if constexpr (RANGES) {
    qb0 = w.range * ranges.blocks;
    nqb = qb0 + ranges.blocks < nqb ? qb0 + ranges.blocks : nqb;
  }
  // copy x of block j: Q rows, dO rows, 64 values of lse and D
  auto start = [&](int j, int x) __attribute__((always_inline)) {
    const uint32_t st = lds0 + (j & 1) * kStage, to = st + (wave - row_wave) * GM::kCopies * 1024;
    const int first = kColumns * j;
    const size_t at = cols.offset<D>(first);
    if (x < GM::kCopies) stage_rows<D>(to, qbase + at, cols.count - first, off, x, row_wave, lane);
    else if (x < 2 * GM::kCopies) stage_rows<D>(to + kGrad, gbase + at, cols.count - first, off, x - GM::kCopies, row_wave, lane);
    else {
      const uint32_t soff = 4 * cols.within(first + lane);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(st + kStats + (wave & 1) * 256),
                   "v"(soff), "s"(stat) : "memory");
    }
  };
  constexpr int COPIES = 2 * GM::kCopies + 1;

  // K and V fragments of this wavefront's states: lane (r, hf) holds d = 16 s + 8 hf .. + 7.  K comes through the places
  // of Q and dO, V through the wavefront's own block.
  const AttReads<D> rd(lds0, lane);
  const uint32_t own = kOwn + wave * kOwnBlock;
  u32x4_t kf[CT][KS], vf[CT][kValuesInLds ? 1 : KS];
  if (live) {
    auto state = [&](int row) __attribute__((always_inline)) {
      const int at = w.col0 + row < n ? w.col0 + row : n - 1;
      return kv + states + (size_t)at * ld;
    };
    stage_own_rows<D, CT>(lds0 + wave * kOwnBlock, lane, [&](int row) __attribute__((always_inline)) { return state(row); });
    stage_own_rows<D, CT>(lds0 + own, lane, [&](int row) __attribute__((always_inline)) { return state(row) + Akv; });
    wait_all_copies();
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        kf[c][s] = rd.row(wave * kOwnBlock, c, s);
        asm volatile("" : "+v"(kf[c][s]) :: "memory");
        if (!kValuesInLds) vf[c][s] = rd.row(own, c, s);
      }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < COPIES; ++x) start(qb0, x);
  if (!live) {                                                 // a wavefront without states that hold stages, and clears its rows
    for (int qb = qb0; qb + 1 < nqb; ++qb) {
      wait_all_copies();
      __syncthreads();
#pragma unroll
      for (int x = 0; x < COPIES; ++x) start(qb + 1, x);
    }
    wait_all_copies();
    __syncthreads();
    clear(w.col0, 32 * CT, lane, 64);
    return;
  }
  f32x16_t dk[CT][DT], dv[CT][DT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      if constexpr (PAIR) dk[c][t] = dv[c][t] = f32x16_t{};
      else { clear_acc(dk[c][t]); clear_acc(dv[c][t]); }
    }
  const float scale = 1.0f / sqrtf((float)D), sl2 = 1.4426950408889634f * scale;
  // value i of a tile belongs to column 32 t + 8 (i/4) + 4 hf + i%4: four consecutive columns per i/4
  auto stat4 = [&](uint32_t block, int t, int i4) __attribute__((always_inline)) {
    return *(lds_f4_ptr)(uintptr_t)(lds0 + block + 4 * (32 * t + 8 * i4 + 4 * hf));
  };
  auto step = [&](int qb, auto last) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(last)::value;
    wait_all_copies();                                         // block qb is there;
    __syncthreads();                                           // block qb - 1 is read, its place free
    const uint32_t qst = (qb & 1) * kStage, gst = qst + kGrad, sst = qst + kStats;
    f32x16_t p[CT], ds[CT];                                    // S, then P; dP, then dS: [query][state]
    u32x4_t pt[2][CT], dst[2][CT];                             // [k step][column tile]
    f32x4_t l4[2], d4[2];
    u32x4_t vcol[3][CT];
    // per 32 queries: KS units of S; KS of dP, under them P; 2 DT of dV, under them dS; 2 DT of dK
    constexpr int UNITS = 2 * KS + 4 * DT;
    auto end_mask = [&](f32x16_t (&v)[CT], int t, int first) __attribute__((always_inline)) {
      if ((cols.count & 63) == 0) return;
#pragma unroll
      for (int i = first; i < first + 8; ++i)
        if (qb * 64 + 32 * t + 8 * (i >> 2) + 4 * hf + (i & 3) >= cols.count) {
#pragma unroll
          for (int c = 0; c < CT; ++c) v[c][i] = 0.f;
        }
    };
    run_units<0, 2 * UNITS, 3>(
        [&](auto) __attribute__((always_inline)) { return std::integral_constant<int, CT>{}; },
        [&](auto U) __attribute__((always_inline)) {
          constexpr int t = decltype(U)::value / UNITS, u = decltype(U)::value % UNITS, v = u - 2 * KS, x = v - 2 * DT;
          if constexpr (u < KS) return rd.row(qst, t, u);
          else if constexpr (u < 2 * KS) return rd.row(gst, t, u - KS);
          else if constexpr (v < 2 * DT) return rd.transposed(gst, 32 * t + 16 * (v / DT), v % DT);
          else return rd.transposed(qst, 32 * t + 16 * (x / DT), x % DT);
        },
        [&](auto U, auto P, const u32x4_t& f) __attribute__((always_inline)) {
          constexpr int u = decltype(U)::value % UNITS, v = u - 2 * KS, x = v - 2 * DT, c = decltype(P)::value;
          if constexpr (kValuesInLds && u >= KS - 2 && u < 2 * KS - 2) vcol[(u - KS + 2) % 3][c] = rd.row(own, c, u - KS + 2);
          if constexpr (u < KS) p[c] = MOE_MFMA(f, kf[c][u], u == 0 ? f32x16_t{} : p[c]);
          else if constexpr (u < 2 * KS) {
            u32x4_t col;                                       // (V from LDS was fetched two units ago)
            if constexpr (kValuesInLds) col = vcol[(u - KS) % 3][c];
            else col = vf[c][u - KS];
            ds[c] = MOE_MFMA(f, col, u == KS ? f32x16_t{} : ds[c]);
          } else {
            if constexpr (v % DT == 0 && c == 0) fresh_operand();
            if constexpr (x < 0) mfma_acc(dv[c][v % DT], f, pt[v / DT][c]);
            else mfma_acc(dk[c][x % DT], f, dst[x / DT][c]);
          }
        },
        [&](auto U, auto P, auto) __attribute__((always_inline)) {
          constexpr int t = decltype(U)::value / UNITS, u = decltype(U)::value % UNITS, v = u - 2 * KS, x = v - 2 * DT;
          constexpr int pc = decltype(P)::value;
          if constexpr (!LAST && decltype(U)::value < COPIES && pc == 0) start(qb + 1, decltype(U)::value);
          if constexpr (u == KS - 1 && pc == 0) l4[0] = stat4(sst, t, 0);
          if constexpr (u >= KS && u < 2 * KS) {               // P
            constexpr int z = CT * (u - KS) + pc, first = z * 16 / KS, to = (z + 1) * 16 / KS;      // value j: row j / CT, column tile j % CT
            if constexpr (first % (4 * CT) == 0 && first + 4 * CT < 16 * CT) l4[(first / (4 * CT) + 1) % 2] = stat4(sst, t, first / (4 * CT) + 1);
#pragma unroll
            for (int j = first; j < to; ++j)
              p[j % CT][j / CT] = __builtin_amdgcn_exp2f(fmaf(p[j % CT][j / CT], sl2, -l4[j / (4 * CT) % 2][j / CT % 4]));
            if constexpr (LAST && to % (8 * CT) == 0) end_mask(p, t, to / CT - 8);
            if constexpr (u == KS + KS / 2 + 1) pt[0][pc] = pack8(p[pc], 0);
            if constexpr (u == 2 * KS - 1 && pc == 0) d4[0] = stat4(sst + 256, t, 0);
          }
          if constexpr (v == 0) pt[1][pc] = pack8(p[pc], 8);
          if constexpr (v >= 0 && x < 0) {                     // dS
            constexpr int z = CT * v + pc, all = 2 * DT * CT, first = z * 16 * CT / all, to = (z + 1) * 16 * CT / all;
            if constexpr (first % (4 * CT) == 0 && first != to && first + 4 * CT < 16 * CT) d4[(first / (4 * CT) + 1) % 2] = stat4(sst + 256, t, first / (4 * CT) + 1);
#pragma unroll
            for (int j = first; j < to; ++j) ds[j % CT][j / CT] = p[j % CT][j / CT] * (ds[j % CT][j / CT] - d4[j / (4 * CT) % 2][j / CT % 4]);
            if constexpr (LAST && first != to && to % (8 * CT) == 0) end_mask(ds, t, to / CT - 8);
            if constexpr (v == DT + 1) dst[0][pc] = pack8(ds[pc], 0);
          }
          if constexpr (x == 0) dst[1][pc] = pack8(ds[pc], 8);
        });
  };
  auto pair_step = [&](int qb) __attribute__((always_inline)) {
    wait_all_copies();                                         // block qb is there;
    __syncthreads();                                           // block qb - 1 is read, its place free
    if (qb + 1 < nqb) {
#pragma unroll
      for (int x = 0; x < COPIES; ++x) start(qb + 1, x);
    }
    const uint32_t qst = (qb & 1) * kStage, gst = qst + kGrad, sst = qst + kStats;
    f32x16_t s[2], dp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        u32x4_t col;
        if constexpr (kValuesInLds) col = rd.row(own, 0, x);
        else col = vf[0][x];
        s[t] = MOE_MFMA(rd.row(qst, t, x), kf[0][x], x == 0 ? f32x16_t{} : s[t]);
        dp[t] = MOE_MFMA(rd.row(gst, t, x), col, x == 0 ? f32x16_t{} : dp[t]);
      }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool there = kColumns * qb + 8 * (i >> 2) + 4 * hf + (i & 3) < cols.count;
      const float p = __builtin_amdgcn_exp2f(fmaf(pair_sum(s[0][i], s[1][i]), sl2, -stat4(sst, 0, i / 4)[i % 4]));
      const float ds = p * (pair_sum(dp[0][i], dp[1][i]) - stat4(sst + 256, 0, i / 4)[i % 4]);
      s[0][i] = there ? p : 0.f;
      dp[0][i] = there ? ds : 0.f;
    }
    auto product = [&](f32x16_t (&acc)[DT], const f32x16_t& v, uint32_t block) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4_t first = pack8(v, 8 * h);
        u32x4_t left;
#pragma unroll
        for (int i = 0; i < 4; ++i) left[i] = bf16_rest_x2(v[8 * h + 2 * i], v[8 * h + 2 * i + 1], first[i]);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const u32x4_t a = rd.transposed(block, 16 * h, dt);
          acc[dt] = MOE_MFMA(rd.transposed(block, 32 + 16 * h, dt), first, acc[dt]);
          acc[dt] = MOE_MFMA(a, left, acc[dt]);
          acc[dt] = MOE_MFMA(a, first, acc[dt]);
        }
      }
    };
    product(dv[0], s[0], gst);
    product(dk[0], dp[0], qst);
  };
  if constexpr (PAIR) {
    for (int qb = qb0; qb < nqb; ++qb) pair_step(qb);
  } else {
    for (int qb = qb0; qb + 1 < nqb; ++qb) step(qb, std::false_type{});
    step(nqb - 1, std::true_type{});
    settle_all(dk);
    settle_all(dv);
  }
  if constexpr (RANGES) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int at = w.col0 + 32 * c + r;
      if (at >= g.Lk) continue;
      float* const to = out + (size_t)at * ld + 4 * hf;
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) {                       // d = 8 i + 4 hf ..
        f32x4_t k4 = {0.f, 0.f, 0.f, 0.f}, v4 = k4;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at < n) {
            k4[j] = dk[c][i / 4][4 * (i % 4) + j] * scale;
            v4[j] = dv[c][i / 4][4 * (i % 4) + j];
          }
        *reinterpret_cast<f32x4_t*>(to + 8 * i) = k4;
        *reinterpret_cast<f32x4_t*>(to + Akv + 8 * i) = v4;
      }
    }
    return;
  }
  auto put = [&](bf16_t* to) __attribute__((always_inline)) {
    return [=](int row, int chunk, const u32x4_t& v) __attribute__((always_inline)) {
      const int at = w.col0 + row;
      if (at < g.Lk) *reinterpret_cast<u32x4_t*>(to + (size_t)at * ld + 8 * chunk) = at < n ? v : u32x4_t{0u, 0u, 0u, 0u};
    };
  };
  store_rows<D, CT>(dk, scale, lds0 + own, lane, put(dkv + states));
  store_rows<D, CT>(dv, 1.f, lds0 + own, lane, put(dkv + states + Akv));
}

template <int D> constexpr int kLdsFew = kFewWaves * 2 * 64 * AttGeom<D>::kRow;
template <int D> constexpr int kLdsForward = 4 * AttGeom<D>::kBlock;
template <int D> constexpr int kLdsQ = 5 * AttGeom<D>::kBlock;
template <int D> constexpr int kLdsQShort = 2 * AttGeom<D>::kBlock;
static_assert(kLdsQShort<128> <= 65536, "without a raised limit");
template <int D, int CT> constexpr int kLdsKV = 2 * (2 * AttGeom<D>::kBlock + 512) + 128 * CT * AttGeom<D>::kRow;

template <int D>
int prepare_kernels() {
  static LdsLimitOnce once, once_pair, once_few, once_few_pair, once_q, once_qfew, once_qpair, once_kvr, once_kv1, once_kvp, once_kvrp, once_kv2;
  static_assert(kLdsFew<D> >= kFewWaves * (128 * D + 512), "the wavefronts' sums and statistics");
  int rc = ensure_lds_limit(once, reinterpret_cast<const void*>(cross_forward_kernel<D, false>), kLdsForward<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_pair, reinterpret_cast<const void*>(cross_forward_kernel<D, true>), kLdsForward<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_few, reinterpret_cast<const void*>(cross_few_kernel<D, false>), kLdsFew<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_few_pair, reinterpret_cast<const void*>(cross_few_kernel<D, true>), kLdsFew<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_q, reinterpret_cast<const void*>(cross_dq_kernel<D>), kLdsQ<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_qfew, reinterpret_cast<const void*>(cross_dq_few_kernel<D, false>), kLdsFew<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_qpair, reinterpret_cast<const void*>(cross_dq_few_kernel<D, true>), kLdsFew<D>);
  if (rc == MOE_OK) rc = ensure_lds_limit(once_kvp, reinterpret_cast<const void*>(cross_dkv_kernel<D, 1, false, true>), (kLdsKV<D, 1>));
  if (rc == MOE_OK) rc = ensure_lds_limit(once_kvrp, reinterpret_cast<const void*>(cross_dkv_kernel<D, 1, true, true>), (kLdsKV<D, 1>));
  if (rc == MOE_OK) rc = ensure_lds_limit(once_kv1, reinterpret_cast<const void*>(cross_dkv_kernel<D, 1>), (kLdsKV<D, 1>));
  if (rc == MOE_OK) rc = ensure_lds_limit(once_kvr, reinterpret_cast<const void*>(cross_dkv_kernel<D, 1, true>), (kLdsKV<D, 1>));
  if constexpr (D == 128)
    if (rc == MOE_OK) rc = ensure_lds_limit(once_kv2, reinterpret_cast<const void*>(cross_dkv_kernel<D, 2>), (kLdsKV<D, 2>));
  return rc;
}

// what a forward call has besides the shape; q_rest: in pairs
struct CrossForward {
  const bf16_t *q, *q_rest, *kv;
  const int32_t* src_len;
  bf16_t *ctx, *ctx_rest;
  float* lse;
};
template <int D>
int forward(const CrossShape& s, const CrossPlan& plan, const CrossForward& f, const CrossParts& parts, hipStream_t st) {
  if (prepare_kernels<D>() != MOE_OK) return MOE_EHIP;
  const bool pair = f.q_rest != nullptr;
  const int per = (plan.few ? 32 : 128) / (pair ? 2 : 1);
  const long long blocks = s.B * s.kv_heads * ((s.columns() + per - 1) / per) * plan.splits;
  const CrossGeo g(s);
  const dim3 grid((unsigned)blocks), threads(256);
  static_assert(64 * kFewWaves == 256, "threads of both kernels");
  auto run = [&](auto kernel, int lds, auto... last) {
    hipLaunchKernelGGL(kernel, grid, threads, lds, st, g, f.q, f.q_rest, f.kv, f.src_len, f.ctx, f.ctx_rest, f.lse, last...);
  };
  if (plan.few && pair) run(cross_few_kernel<D, true>, kLdsFew<D>, parts);
  else if (plan.few) run(cross_few_kernel<D, false>, kLdsFew<D>, parts);
  else if (pair) run(cross_forward_kernel<D, true>, kLdsForward<D>);
  else run(cross_forward_kernel<D, false>, kLdsForward<D>);
  return check_launch();
}
template <typename T>
int join(const CrossShape& s, const CrossParts& parts, const int32_t* src_len, T* ctx, T* ctx_rest, float* lse, hipStream_t st) {
  const long long columns = s.B * s.kv_heads * s.columns();
  const dim3 grid((unsigned)((columns + 3) / 4)), threads(256);
  if (s.d == 64) hipLaunchKernelGGL((cross_join_kernel<T, 64>), grid, threads, 0, st, CrossGeo(s), parts, src_len, ctx, ctx_rest, lse, columns);
  else hipLaunchKernelGGL((cross_join_kernel<T, 128>), grid, threads, 0, st, CrossGeo(s), parts, src_len, ctx, ctx_rest, lse, columns);
  return check_launch();
}
template <int D>
int backward(const CrossShape& s, const bf16_t* q, const bf16_t* kv, const int32_t* src_len, const bf16_t* ctx, const bf16_t* dctx,
             const float* lse, bf16_t* dq, bf16_t* dkv, float* dvec, float* sums, const CrossRest& rest, hipStream_t st) {
  const bool pair = rest.q != nullptr;
  int cus = 0;
  if (prepare_kernels<D>() != MOE_OK || compute_units(&cus) != MOE_OK) return MOE_EHIP;
  const long long blocks = s.B * s.kv_heads * ((s.columns() + 127) / 128), blocks1 = s.B * s.kv_heads * ((s.Lk + 127) / 128),
                  blocks2 = s.B * s.kv_heads * ((s.Lk + 255) / 256);
  const CrossGeo g(s);
  // dq of few columns where its blocks run all at once: one a unit, two at d 64 if the other kernel's blocks leave half of the units idle.  us, blocks of
  // 128 / 32 columns, on 256 units:  d 64  1 x 20 tokens, 1862 states, 2 key heads 19.4 / 11.4; 2 x 300, 2000 34.8 / 20.4; 2 x 1000, 1000 (512 blocks of 32)
  // 21.9 / 17.6; 31 x 40, 200 (186 blocks of 128, 372 of 32) 7.3 / 8.0; 11 x 333, 777 25.6 / 44.2;  d 128  4 x 64, 1000 29.2 / 17.8; 16 x 64, 256 (256 of
  // 32) 12.8 / 9.7; 3 x 700, 700 (264 of 32) 22.3 / 25.9; 4 x 400, 1000 32.5 / 36.6
  const long long blocks32 = s.B * s.kv_heads * ((s.columns() + 31) / 32);
  const bool few_dq = blocks32 <= cus || (D == 64 && blocks32 <= 2LL * cus && 2 * blocks <= cus);
  const long long blocks16 = s.B * s.kv_heads * ((s.columns() + 15) / 16);
  if (pair) hipLaunchKernelGGL((cross_dq_few_kernel<D, true>), dim3((unsigned)blocks16), dim3(64 * kFewWaves), kLdsFew<D>, st, g, q, kv, src_len, ctx, dctx, lse, dq, dvec, rest);
  else if (s.Lk <= 64) hipLaunchKernelGGL((cross_dq_short_kernel<D>), dim3((unsigned)blocks), dim3(256), kLdsQShort<D>, st, g, q, kv, src_len, dctx, dq, dvec);
  else if (few_dq) hipLaunchKernelGGL((cross_dq_few_kernel<D, false>), dim3((unsigned)blocks32), dim3(64 * kFewWaves), kLdsFew<D>, st, g, q, kv, src_len, ctx, dctx, lse, dq, dvec, rest);
  else hipLaunchKernelGGL((cross_dq_kernel<D>), dim3((unsigned)blocks), dim3(256), kLdsQ<D>, st, g, q, kv, src_len, ctx, dctx, lse, dq, dvec);
  const int each = pair ? cross_pair_dkv_blocks(s) : cross_dkv_blocks(s), blocks64 = (int)((s.columns() + 63) / 64);
  const CrossRanges ranges{(blocks64 + each - 1) / each, pair ? 2 * each : each, (size_t)s.B * s.Lk * 2 * s.kv_heads * D, sums};
  if (ranges.count > 1) {
    const dim3 grid((unsigned)(blocks1 * ranges.count));
    if (pair) hipLaunchKernelGGL((cross_dkv_kernel<D, 1, true, true>), grid, dim3(256), (kLdsKV<D, 1>), st, g, q, kv, src_len, dctx, lse, dvec, dkv, ranges, rest);
    else hipLaunchKernelGGL((cross_dkv_kernel<D, 1, true>), grid, dim3(256), (kLdsKV<D, 1>), st, g, q, kv, src_len, dctx, lse, dvec, dkv, ranges, rest);
    const int rc = check_launch();
    return rc != MOE_OK ? rc : launch_add_ranges(sums, ranges.count, (long long)ranges.elems, dkv, st);
  }
  if (pair) {
    hipLaunchKernelGGL((cross_dkv_kernel<D, 1, false, true>), dim3((unsigned)blocks1), dim3(256), (kLdsKV<D, 1>), st, g, q, kv, src_len, dctx, lse, dvec, dkv, ranges, rest);
    return check_launch();
  }
  // two tiles of 32 states per wavefront where that takes fewer rounds of blocks (1.46 times as long each: attention_dkv_wide)
  if constexpr (D == 128)
    if (1.46 * (double)((blocks2 + cus - 1) / cus) < (double)((blocks1 + cus - 1) / cus)) {
      hipLaunchKernelGGL((cross_dkv_kernel<D, 2>), dim3((unsigned)blocks2), dim3(256), (kLdsKV<D, 2>), st, g, q, kv, src_len, dctx, lse, dvec, dkv, ranges, rest);
      return check_launch();
    }
  hipLaunchKernelGGL((cross_dkv_kernel<D, 1>), dim3((unsigned)blocks1), dim3(256), (kLdsKV<D, 1>), st, g, q, kv, src_len, dctx, lse, dvec, dkv, ranges, rest);
  return check_launch();
}

// 16 bytes at a time: rows of states that hold, zeros for the others
__global__ __launch_bounds__(256) void held_rows_kernel(const uint4* __restrict__ mem, const int32_t* __restrict__ src_len,
                                                        uint4* __restrict__ out, int Lk, int vecs, long long total) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = i / vecs, b = row / Lk;
    const int n = src_len[b];
    out[i] = (int)(row - b * Lk) < n ? mem[i] : uint4{0u, 0u, 0u, 0u};
  }
}

}  // namespace

int prepare_cross_attention() {
  const int rc = prepare_kernels<64>();
  return rc != MOE_OK ? rc : prepare_kernels<128>();
}

// Which form a forward call takes, by what both are expected to take (us).  A block of 128 columns walks its states in steps, two blocks on a unit
// (fp32: one at a time multiplies); one of 32 columns shares them among its wavefronts and `splits` blocks, which cost a launch to join and
// bring only as much memory as they have units.  What the ranges leave of each column is written and read once more, 0.5 to 0.8 us a MB, and so there are no more
// blocks in ranges than four rounds of the device: without that, a rounded number of rounds asked for up to 64 ranges of many columns.  us of calls in 1 / 4 /
// 64 ranges, bf16, heads of 64: 10 x 1162 tokens, 8161 states, 1 head 111 / 93 / 197; 19 x 83, 8174, 8 on 4 114 / 117 / 251; 19 x 15, 8100, 24 on 3
// 94 / 70 / 130; fp32, 19 x 83, 8174, 8 on 4 381 / 382 / 571.
// us, 128 / 32 columns in the best number of ranges, bf16, heads of 128: 64 x 1 tokens, 410 to 2048
// states, 16 heads 120 / 128; 1 x 4, 53 5.0 / 6.1; 1 x 1, 1000 23.7 / 10.1 (8); 1 x 1, 8000 155 / 23 (16); 8 x 1, 1000 23.2 / 19.1 (2); 4 x 8, 4000, 2 key
// heads of 16 82 / 13.7 (16); 4 x 64, 1000, 8 heads 26.9 / 14.2 (4); 3 x 700, up to 700, 4 heads 20.4 / 29; of 64: 16 x 1, 2000, 8 heads 28.2 / 16.9 (4);
// 2 x 300, 2000 34.5 / 23.0 (2); 27 x 834, up to 100 18.9 / 47; fp32, of 64: 5 x 187, up to 411, 8 heads 40.8 / 16.3; 8 x 500, 500 59 / 64; 27 x 834, up to
// 100 56 / 95.
// In pairs, blocks have half the columns.  us of the kernels, 64 / 16 columns in the best number of ranges: heads of 128: 55 x 4 tokens, 131 states, 8 heads 9.3 / 14.3;
// 47 x 1, 267, 16 26.0 / 34.4; 1 x 2, 23, 3 5.1 / 7.0; 1 x 16, 115, 4 7.3 / 6.2; 5 x 1, 935, 8 23.7 / 13.3 (4); 8 x 12, 2761, 4 63.1 / 17.7 (8); 3 x 4, 5147, 3
// 108.5 / 14.6 (16); of 64: 4 x 1, 55, 3 4.1 / 4.9; 106 x 1, 633, 2 12.8 / 9.6; 83 x 4, 2954, 2 46.9 / 27.9 (2); 7 x 1, 5269, 8 on 4 77.2 / 15.0 (16).
static CrossPlan plan_of(int act_dtype, const CrossShape& s, bool pair) {
  constexpr double kUnits = 256;                               // of a whole device: the choice sizes a workspace
  const bool f32 = act_dtype == MOE_F32;
  const double pairs = (double)s.B * s.kv_heads, mb = pairs * s.Lk * 2 * s.d * (f32 ? 4 : 2) / 1e6;
  const double step128 = f32 ? (s.d == 64 ? 3.5 : 7.0) : pair ? (s.d == 64 ? 0.8 : 1.3) : s.d == 64 ? 0.75 : 1.2;
  const double step32 = f32 ? step128 : pair ? (s.d == 64 ? 1.1 : 1.9) : s.d == 64 ? 1.1 : 1.7, ends = f32 ? 1 : 0;
  const double base128 = pair ? 5 : 4, base32 = pair ? 5 : 6, join = pair ? 7 : 4, rate = pair ? 8 : 5;         // us, us, us, MB/us
  const int blocks = (s.Lk + 31) / 32, wide = pair ? 64 : 128, narrow = pair ? 16 : 32;
  auto rounds = [](double n, double at_once) { return ceil(n / at_once); };
  auto longer = [](double a, double b) { return a > b ? a : b; };
  CrossPlan best{false, 1};
  double least = base128 + longer(step128 * (f32 ? blocks : (blocks + 1) / 2) * rounds(pairs * ((s.columns() + wide - 1) / wide), f32 ? kUnits : 2 * kUnits), mb / rate);
  for (int splits = 1; splits <= 64 && splits <= (blocks + 3) / 4; splits *= 2) {
    const double items = pairs * ((s.columns() + narrow - 1) / narrow) * splits, at_once = !f32 && s.d == 64 ? 2 * kUnits : kUnits;
    if (splits > 1 && items > 4 * at_once) break;
    const double joined = splits > 1 ? join + 0.55 * pairs * s.columns() * splits * (4 * s.d + 8) / 1e6 : 0;
    const double us = base32 + joined + longer((step32 * ((blocks + 4 * splits - 1) / (4 * splits)) + ends) * rounds(items, at_once),
                                           mb / rate * (items < kUnits ? kUnits / items : 1.0));
    if (us < least) {
      least = us;
      best = {true, splits};
    }
  }
  return best;
}

CrossPlan cross_plan(int act_dtype, const CrossShape& s) { return plan_of(act_dtype, s, false); }
CrossPlan cross_pair_plan(const CrossShape& s) { return plan_of(MOE_BF16, s, true); }

static size_t scratch_of(const CrossShape& s, const CrossPlan& p) {
  const size_t columns = (size_t)s.B * s.kv_heads * s.columns();
  return p.splits > 1 ? align_up(columns * p.splits * sizeof(float2), 256) + columns * p.splits * s.d * sizeof(float) : 0;
}

size_t cross_scratch_bytes(int act_dtype, const CrossShape& s) { return scratch_of(s, cross_plan(act_dtype, s)); }
size_t cross_pair_scratch_bytes(const CrossShape& s) { return scratch_of(s, cross_pair_plan(s)); }

// in pairs a step has 32 columns, of as many products and more vector work
static int dkv_blocks_of(const CrossShape& s, bool pair) {
  constexpr double kUnits = 256;                               // of a whole device: the choice sizes a workspace
  const double blocks = (double)s.B * s.kv_heads * ((s.Lk + 127) / 128), at_once = s.d == 64 ? 2 * kUnits : kUnits;
  const double step = pair ? (s.d == 64 ? 3.8 : 4.6) : s.d == 64 ? 1.18 : 1.8, mb = blocks * 128 * 2 * s.d * sizeof(float) / 1e6;
  const int all = (int)((s.columns() + 63) / 64);
  int best = all;
  double least = 5 + step * all;
  for (int ranges : {2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    if (ranges > all || blocks * ranges > at_once) break;
    const int each = (all + ranges - 1) / ranges;
    const double us = 9 + step * each + 0.5 * mb * ranges;
    if (us < least) {
      least = us;
      best = each;
    }
  }
  return best;
}

int cross_dkv_blocks(const CrossShape& s) { return dkv_blocks_of(s, false); }
int cross_pair_dkv_blocks(const CrossShape& s) { return dkv_blocks_of(s, true); }

size_t cross_bwd_scratch_bytes(int act_dtype, const CrossShape& s, bool pair) {
  if (act_dtype == MOE_F32) return 0;
  const long long all = (s.columns() + 63) / 64, each = dkv_blocks_of(s, pair), ranges = (all + each - 1) / each;
  return ranges > 1 ? (size_t)ranges * s.B * s.Lk * 2 * s.kv_heads * s.d * sizeof(float) : 0;
}

static CrossParts parts_of(const CrossShape& s, const CrossPlan& plan, void* scratch) {
  const size_t columns = (size_t)s.B * s.kv_heads * s.columns();
  return {plan.splits, static_cast<float2*>(scratch), reinterpret_cast<float*>(static_cast<char*>(scratch) + align_up(columns * plan.splits * sizeof(float2), 256))};
}
static int launch_bf16(const CrossShape& s, const CrossPlan& plan, const CrossForward& f, void* scratch, hipStream_t st) {
  const CrossParts parts = parts_of(s, plan, scratch);
  const int rc = s.d == 64 ? forward<64>(s, plan, f, parts, st) : forward<128>(s, plan, f, parts, st);
  return rc != MOE_OK || plan.splits == 1 ? rc : join(s, parts, f.src_len, f.ctx, f.ctx_rest, f.lse, st);
}

int launch_cross_attention(int act_dtype, const CrossShape& s, const void* q, const void* kv, const int32_t* src_len, void* ctx,
                           float* lse, void* scratch, hipStream_t st) {
  const CrossPlan plan = cross_plan(act_dtype, s);
  if (act_dtype == MOE_F32) {
    const CrossParts parts = parts_of(s, plan, scratch);
    float* const c = static_cast<float*>(ctx);
    const int rc = launch_cross_attention_f32(s, plan, static_cast<const float*>(q), static_cast<const float*>(kv), src_len, c, lse, parts, st);
    return rc != MOE_OK || plan.splits == 1 ? rc : join<float>(s, parts, src_len, c, nullptr, lse, st);
  }
  return launch_bf16(s, plan, {static_cast<const bf16_t*>(q), nullptr, static_cast<const bf16_t*>(kv), src_len, static_cast<bf16_t*>(ctx), nullptr, lse}, scratch, st);
}

int launch_cross_attention_pair(const CrossShape& s, const void* q, const void* q_rest, const void* kv, const int32_t* src_len, void* ctx, void* ctx_rest,
                                float* lse, void* scratch, hipStream_t st) {
  return launch_bf16(s, cross_pair_plan(s), {static_cast<const bf16_t*>(q), static_cast<const bf16_t*>(q_rest), static_cast<const bf16_t*>(kv), src_len,
                     static_cast<bf16_t*>(ctx), static_cast<bf16_t*>(ctx_rest), lse}, scratch, st);
}

static int launch_bf16_bwd(const CrossShape& s, const void* q, const void* kv, const int32_t* src_len, const void* ctx, const void* dctx, const float* lse,
                           void* dq, void* dkv, float* dvec, float* sums, const CrossRest& rest, hipStream_t st) {
  auto qb = static_cast<const bf16_t*>(q);
  auto kb = static_cast<const bf16_t*>(kv);
  auto c = static_cast<const bf16_t*>(ctx);
  auto gb = static_cast<const bf16_t*>(dctx);
  auto dqb = static_cast<bf16_t*>(dq);
  auto dkb = static_cast<bf16_t*>(dkv);
  return s.d == 64 ? backward<64>(s, qb, kb, src_len, c, gb, lse, dqb, dkb, dvec, sums, rest, st)
                   : backward<128>(s, qb, kb, src_len, c, gb, lse, dqb, dkb, dvec, sums, rest, st);
}

int launch_cross_attention_bwd(int act_dtype, const CrossShape& s, const void* q, const void* kv, const int32_t* src_len,
                               const void* ctx, const void* dctx, const float* lse, void* dq, void* dkv, float* dvec, float* sums, hipStream_t st) {
  if (act_dtype == MOE_F32)
    return launch_cross_attention_f32_bwd(s, static_cast<const float*>(q), static_cast<const float*>(kv), src_len, static_cast<const float*>(ctx),
                                          static_cast<const float*>(dctx), lse, static_cast<float*>(dq), static_cast<float*>(dkv), dvec, st);
  return launch_bf16_bwd(s, q, kv, src_len, ctx, dctx, lse, dq, dkv, dvec, sums, CrossRest{}, st);
}

int launch_cross_attention_pair_bwd(const CrossShape& s, const CrossPair& q, const void* kv, const int32_t* src_len, const CrossPair& ctx, const CrossPair& dctx,
                                    const float* lse, void* dq, void* dkv, float* dvec, float* sums, hipStream_t st) {
  const CrossRest rest{static_cast<const bf16_t*>(q.rest), static_cast<const bf16_t*>(ctx.rest), static_cast<const bf16_t*>(dctx.rest)};
  return launch_bf16_bwd(s, q.first, kv, src_len, ctx.first, dctx.first, lse, dq, dkv, dvec, sums, rest, st);
}

int launch_held_rows(int act_dtype, const void* mem, const int32_t* src_len, void* out, long long B, int Lk, int M, hipStream_t st) {
  const int vecs = M / (act_dtype == MOE_F32 ? 4 : 8);
  const long long total = B * Lk * vecs;
  const long long blocks = (total + 255) / 256, most = 1 << 16;
  hipLaunchKernelGGL(held_rows_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, static_cast<const uint4*>(mem), src_len,
                     static_cast<uint4*>(out), Lk, vecs, total);
  return check_launch();
}

}  // namespace moe
