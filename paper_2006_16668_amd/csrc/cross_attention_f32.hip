// Attention of a decoder's tokens to an encoder's states in fp32 on the matrix cores (d = 64 or 128): the sums of attention_f32.hip
// (full fp32 products, a lane owns a column, four wavefronts with 32 columns each or all on the same 32), with columns,
// states that hold and empty sources as in cross_attention.hip.
//
// Few columns: the wavefronts share 32 columns and the states' blocks are cut into `splits` ranges besides, a block each, which
// cross_join_kernel puts together; K and V come straight from memory, a block ahead.
#include <float.h>
#include <math.h>
#include "attention_f32_tiles.h"
#include "cross_attention.h"

namespace moe {
namespace {

// What a wavefront does: 32 columns from col0 on, blocks of 32 rows from `first` to `last`, `step` apart.
struct CrossWorkF32 {
  long long bk, b;
  int k, block0, col0, split;
};
template <bool SPLIT>
__device__ __forceinline__ CrossWorkF32 work_of(int count, int kv_heads, int splits, int wave) {
  const int columns = SPLIT ? 32 : 32 * kWaves, per = (count + columns - 1) / columns;
  unsigned item = blockIdx.x;                                  // XCDs get contiguous ranges: a head's blocks share an L2
  const unsigned per_xcd = gridDim.x / 8;
  if (item < per_xcd * 8) item = (item % 8) * per_xcd + item / 8;
  CrossWorkF32 w;
  w.split = 0;
  if (SPLIT) {
    w.split = item % splits;
    item /= splits;
  }
  const unsigned pair = item / per;
  w.bk = pair;
  w.b = pair / kv_heads;
  w.k = (int)(pair % kv_heads);
  w.block0 = (int)(item % per) * columns;
  w.col0 = w.block0 + (SPLIT ? 0 : 32 * wave);
  return w;
}

template <int D, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 2 : 1) void cross_f32_kernel(CrossGeo g, const float* __restrict__ q,
                                                                                 const float* __restrict__ kv, const int32_t* __restrict__ src_len,
                                                                                 float* __restrict__ ctx, float* __restrict__ lse,
                                                                                 CrossParts parts) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const CrossCols cols(g, D);
  const CrossWorkF32 w = work_of<SPLIT>(cols.count, g.kv_heads, parts.splits, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk), Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const float* const keys = kv + (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  const int nkb = (n + 31) / 32, per = (nkb + parts.splits - 1) / parts.splits;
  const int from = SPLIT ? w.split * per : 0, to = SPLIT ? (from + per < nkb ? from + per : nkb) : nkb;
  const int c = w.col0 + r;
  Pieces<D> qf, kf;
  qf.load(q + head + cols.offset<D>(cols.within(c)), hf);
  auto load_keys = [&](int kb) __attribute__((always_inline)) {          // (past the end: the last state)
    const int key = 32 * kb + r;
    kf.load(keys + (size_t)(key < n ? key : n - 1) * ld, hf);
  };
  f32x16_t o[D / 32];
  clear<D>(o);
  const float scale = 1.0f / sqrtf((float)D);
  // (the maximum starts finite: a block of states whose scores are all -inf adds nothing)
  float m_run = -FLT_MAX, l_run = 0.f;
  auto softmax_block = [&](int kb, f32x16_t& p) __attribute__((always_inline)) {     // scores to probabilities
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] *= scale;
      if (32 * kb + 8 * (i >> 2) + 4 * hf + (i & 3) >= n) p[i] = -INFINITY;
      mx = fmaxf(mx, p[i]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m_run, mx);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) { p[i] = expf(p[i] - m_new); sum += p[i]; }
    sum += __shfl_xor(sum, 32, 64);
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
      const float alpha = expf(m_run - m_new);                 // 0 on the first block
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
    }
    l_run += sum;
    m_run = m_new;
  };
  if constexpr (SPLIT) {
    if (from + wave < to) load_keys(from + wave);
    for (int kb = from + wave; kb < to; kb += kWaves) {
      Rows<D> vf;
      vf.load(keys + Akv, ld, 32 * kb, n, r, hf);
      f32x16_t p = over_d<D>(kf, qf);
      load_keys(kb + kWaves);
      softmax_block(kb, p);
      if (32 * kb + 32 > n) vf.clear_past(32 * kb, n, hf);     // wavefront-uniform
      over_rows<D>(o, vf, p);
    }
  } else if (nkb > 0) {                                        // block-uniform
    __shared__ __attribute__((aligned(16))) float ks[Staged<D>::kFloats], vs[Staged<D>::kFloats];
    Transit<D> next;
    next.fetch(keys, ld, keys + Akv, ld, 0, n);
    for (int kb = 0; kb < nkb; ++kb) {
      __syncthreads();                                         // the block before has been read by everyone
      next.put(ks, vs, kb, n);
      __syncthreads();
      if (kb + 1 < nkb) next.fetch(keys, ld, keys + Akv, ld, kb + 1, n);
      f32x16_t p = over_d<D>(Staged<D>{ks, r, hf}, qf);
      softmax_block(kb, p);
      over_rows<D>(o, Staged<D>{vs, r, hf}, p);
    }
  }
  if constexpr (SPLIT) {                                       // to the columns' common maximum, then add up
    __shared__ float stats[2][kWaves][64], sums[kWaves - 1][D / 32][16][64];
    stats[0][wave][lane] = m_run;
    stats[1][wave][lane] = l_run;
    __syncthreads();
    float m = m_run;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) m = fmaxf(m, stats[0][k][lane]);
    const float alpha = expf(m_run - m);                       // (a wavefront without a block of states: 0 x 0)
    l_run = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) l_run += stats[1][k][lane] * expf(stats[0][k][lane] - m);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
    m_run = m;
    add_up<D>(o, sums, wave, lane);
    if (wave > 0) return;
  }
  if (c >= cols.count) return;
  const size_t column = (size_t)w.bk * cols.count + c;
  if (SPLIT && parts.splits > 1) {
    if (hf == 0) parts.stats[column * parts.splits + w.split] = float2{m_run, l_run};
    store_column<D>(parts.sums + (column * parts.splits + w.split) * D, o, 1.0f, hf);
    return;
  }
  if (lse != nullptr && hf == 0) lse[column] = n == 0 ? 0.f : m_run + logf(l_run);
  store_column<D>(ctx + head + cols.offset<D>(c), o, n == 0 ? 0.f : 1.0f / l_run, hf);
}

// dq, and D = rowsum(dctx * ctx)
template <int D, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves, 1) void cross_f32_dq_kernel(CrossGeo g, const float* __restrict__ q, const float* __restrict__ kv,
                                                                      const int32_t* __restrict__ src_len, const float* __restrict__ ctx,
                                                                      const float* __restrict__ dctx, const float* __restrict__ lse,
                                                                      float* __restrict__ dqo, float* __restrict__ dvec) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const CrossCols cols(g, D);
  const CrossWorkF32 w = work_of<SPLIT>(cols.count, g.kv_heads, 1, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk), Akv = g.kv_heads * D;
  const size_t ld = (size_t)2 * Akv;
  const float* const keys = kv + (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  const int c = w.col0 + r;
  const size_t row = head + cols.offset<D>(cols.within(c)), column = (size_t)w.bk * cols.count + cols.within(c);
  Pieces<D> qf, gf, kf, vf;
  qf.load(q + row, hf);
  gf.load(dctx + row, hf);
  kf.load(ctx + row, hf);
  float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) part[j] = fmaf(gf.v[i][j], kf.v[i][j], part[j]);
  float dd = (part[0] + part[1]) + (part[2] + part[3]);
  dd += __shfl_xor(dd, 32, 64);
  const int nkb = (n + 31) / 32;
  // (one block of states: see score_gradients)
  if (nkb > 1 && hf == 0 && c < cols.count && (!SPLIT || wave == 0)) dvec[column] = dd;
  const float ls = lse[column];
  const float scale = 1.0f / sqrtf((float)D);
  auto load_keys = [&](int kb) __attribute__((always_inline)) {
    const int key = 32 * kb + r;
    const float* const at = keys + (size_t)(key < n ? key : n - 1) * ld;
    kf.load(at, hf);
    vf.load(at + Akv, hf);
  };
  f32x16_t dq[D / 32];
  clear<D>(dq);
  // Up to 32 states: D = sum p dP of the probabilities at hand, without the rounding of ctx: of one state p is exactly 1, and dP - D is 0.
  auto score_gradients = [&](int kb, f32x16_t& s, f32x16_t& ds) __attribute__((always_inline)) {
#pragma clang fp contract(off)
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = 32 * kb + 8 * (i >> 2) + 4 * hf + (i & 3) < n ? expf(s[i] * scale - ls) : 0.f;
      sum += s[i] * ds[i];
    }
    if (nkb == 1) {                                            // uniform
      dd = sum + __shfl_xor(sum, 32, 64);
      if (hf == 0 && c < cols.count) dvec[column] = dd;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) ds[i] = s[i] == 0.f ? 0.f : s[i] * (ds[i] - dd) * scale;
  };
  if constexpr (SPLIT) {
    if (wave < nkb) load_keys(wave);
    for (int kb = wave; kb < nkb; kb += kWaves) {
      Rows<D> kr;
      kr.load(keys, ld, 32 * kb, n, r, hf);
      f32x16_t s = over_d<D>(kf, qf);
      f32x16_t ds = over_d<D>(vf, gf);
      load_keys(kb + kWaves);
      score_gradients(kb, s, ds);
      over_rows<D>(dq, kr, ds);
    }
  } else if (nkb > 0) {
    __shared__ __attribute__((aligned(16))) float ks[Staged<D>::kFloats], vs[Staged<D>::kFloats];
    Transit<D> next;
    next.fetch(keys, ld, keys + Akv, ld, 0, n);
    for (int kb = 0; kb < nkb; ++kb) {
      __syncthreads();
      next.put(ks, vs, kb, n);
      __syncthreads();
      if (kb + 1 < nkb) next.fetch(keys, ld, keys + Akv, ld, kb + 1, n);
      f32x16_t s = over_d<D>(Staged<D>{ks, r, hf}, qf);
      f32x16_t ds = over_d<D>(Staged<D>{vs, r, hf}, gf);
      score_gradients(kb, s, ds);
      over_rows<D>(dq, Staged<D>{ks, r, hf}, ds);
    }
  }
  if constexpr (SPLIT) {
    __shared__ float sums[kWaves - 1][D / 32][16][64];
    add_up<D>(dq, sums, wave, lane);
    if (wave > 0) return;
  }
  if (c >= cols.count) return;
  store_column<D>(dqo + row, dq, 1.0f, hf);
}

// dK and dV; needs lse and D of every column of the key head.  The rows of states that do not hold get zeros.
template <int D, bool SPLIT>
__global__ __launch_bounds__(64 * kWaves, 1) void cross_f32_dkv_kernel(CrossGeo g, const float* __restrict__ q, const float* __restrict__ kv,
                                                                       const int32_t* __restrict__ src_len, const float* __restrict__ dctx,
                                                                       const float* __restrict__ lse, const float* __restrict__ dvec,
                                                                       float* __restrict__ dkv) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, hf = lane >> 5;
  const CrossCols cols(g, D);
  const CrossWorkF32 w = work_of<SPLIT>(g.Lk, g.kv_heads, 1, wave);
  const size_t head = cols.base(w.b, w.k, D);
  const int n = held_states(src_len, w.b, g.Lk), Akv = g.kv_heads * D, L = cols.count;
  const size_t ld = (size_t)2 * Akv;
  const size_t states = (size_t)w.b * g.Lk * ld + (size_t)w.k * D;
  const float *const lrow = lse + (size_t)w.bk * L, *const drow = dvec + (size_t)w.bk * L;
  auto query = [&](int c) __attribute__((always_inline)) { return q + head + cols.offset<D>(c); };
  auto grad = [&](int c) __attribute__((always_inline)) { return dctx + head + cols.offset<D>(c); };
  const int key = w.col0 + r, nqb = w.block0 < n ? (L + 31) / 32 : 0;          // (without a state that holds: no blocks, zeros)
  Pieces<D> kf, vf, qf, gf;
  if (nqb > 0) {
    const float* const at = kv + states + (size_t)(key < n ? key : n - 1) * ld;
    kf.load(at, hf);
    vf.load(at + Akv, hf);
  }
  auto load_queries = [&](int qb) __attribute__((always_inline)) {
    const int c = cols.within(32 * qb + r);
    qf.load(query(c), hf);
    gf.load(grad(c), hf);
  };
  const float scale = 1.0f / sqrtf((float)D);
  f32x16_t dk[D / 32], dv[D / 32];
  clear<D>(dk);
  clear<D>(dv);
  // scores to p, dctx v^T to ds; ls, dd: lse and D of the columns.  A column past the end has lse = inf: p = ds = 0
  auto probabilities = [&](f32x16_t& p, f32x16_t& ds, const float (&ls)[16], const float (&dd)[16]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = expf(p[i] * scale - ls[i]);
      ds[i] = p[i] * (ds[i] - dd[i]) * scale;
      if (ls[i] == INFINITY) p[i] = ds[i] = 0.f;               // (also where a copied row's products are not finite)
    }
  };
  float ls[16], dd[16];
  if constexpr (SPLIT) {
    constexpr bool kAhead = D == 64;                           // (registers do not hold a block more at d = 128)
    if (kAhead && nqb > 0) load_queries(wave);
    for (int qb = wave; qb < nqb; qb += kWaves) {
      if (!kAhead) load_queries(qb);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 32 * qb + 8 * (i >> 2) + 4 * hf + (i & 3), rc = cols.within(row);
        ls[i] = row < L ? lrow[rc] : INFINITY;
        dd[i] = row < L ? drow[rc] : 0.f;
      }
      Rows<D> rows;
      if (kAhead) rows.load_at(grad, 32 * qb, L, r, hf);
      f32x16_t p = over_d<D>(qf, kf);
      f32x16_t ds = over_d<D>(gf, vf);
      if (kAhead) load_queries(qb + kWaves);
      else rows.load_at(grad, 32 * qb, L, r, hf);
      probabilities(p, ds, ls, dd);
      rows.clear_past(32 * qb, L, hf);
      over_rows<D>(dv, rows, p);
      rows.load_at(query, 32 * qb, L, r, hf);
      over_rows<D>(dk, rows, ds);
    }
  } else if (nqb > 0) {                                        // block-uniform
    __shared__ __attribute__((aligned(16))) float qs[Staged<D>::kFloats], gs[Staged<D>::kFloats], stats[2][32];
    Transit<D> next;
    float next_stat = 0.f;                                     // threads 0..31: lse, 32..63: D
    auto fetch = [&](int qb) __attribute__((always_inline)) {
      next.fetch_at(query, grad, qb, L);
      const int row = 32 * qb + (threadIdx.x & 31);
      if (threadIdx.x < 32) next_stat = row < L ? lrow[row] : INFINITY;
      else if (threadIdx.x < 64) next_stat = row < L ? drow[row] : 0.f;
    };
    fetch(0);
    for (int qb = 0; qb < nqb; ++qb) {
      __syncthreads();
      next.put(qs, gs, qb, L);
      if (threadIdx.x < 64) stats[threadIdx.x >> 5][threadIdx.x & 31] = next_stat;
      __syncthreads();
      if (qb + 1 < nqb) fetch(qb + 1);
      f32x16_t p = over_d<D>(Staged<D>{qs, r, hf}, kf);
      f32x16_t ds = over_d<D>(Staged<D>{gs, r, hf}, vf);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ls[i] = stats[0][8 * (i >> 2) + 4 * hf + (i & 3)];
        dd[i] = stats[1][8 * (i >> 2) + 4 * hf + (i & 3)];
      }
      probabilities(p, ds, ls, dd);
      over_rows<D>(dv, Staged<D>{gs, r, hf}, p);
      over_rows<D>(dk, Staged<D>{qs, r, hf}, ds);
    }
  }
  if constexpr (SPLIT) {
    __shared__ float sums[kWaves - 1][D / 32][16][64];
    add_up<D>(dk, sums, wave, lane);
    add_up<D>(dv, sums, wave, lane);
    if (wave > 0) return;
  }
  if (key >= g.Lk) return;
  if (key >= n) {
    clear<D>(dk);
    clear<D>(dv);
  }
  float* const out = dkv + states + (size_t)key * ld;
  store_column<D>(out, dk, 1.0f, hf);
  store_column<D>(out + Akv, dv, 1.0f, hf);
}

// (figures at share_columns of attention_f32.hip)
inline bool share_columns(long long columns, int L, double ends) {
  const int blocks = (L + 31) / 32;
  return columns <= 1024 && (double)((columns + 255) / 256) * ((blocks + 3) / 4 + ends) < blocks;
}

}  // namespace

#define MOE_CROSS_F32(KERNEL, SPLIT, COUNT, SPLITS, ...)                                                            \
  {                                                                                                                \
    const int per = SPLIT ? 32 : 32 * kWaves;                                                                      \
    const long long blocks = s.B * s.kv_heads * ((COUNT + per - 1) / per) * (SPLITS);                              \
    const dim3 grid((unsigned)blocks), threads(64 * kWaves);                                                       \
    if (s.d == 64) {                                                                                               \
      if (SPLIT) hipLaunchKernelGGL((KERNEL<64, true>), grid, threads, 0, st, g, __VA_ARGS__);                     \
      else hipLaunchKernelGGL((KERNEL<64, false>), grid, threads, 0, st, g, __VA_ARGS__);                          \
    } else {                                                                                                       \
      if (SPLIT) hipLaunchKernelGGL((KERNEL<128, true>), grid, threads, 0, st, g, __VA_ARGS__);                    \
      else hipLaunchKernelGGL((KERNEL<128, false>), grid, threads, 0, st, g, __VA_ARGS__);                         \
    }                                                                                                              \
  }

int launch_cross_attention_f32(const CrossShape& s, const CrossPlan& plan, const float* q, const float* kv, const int32_t* src_len,
                               float* ctx, float* lse, const CrossParts& parts, hipStream_t st) {
  const CrossGeo g(s);
  MOE_CROSS_F32(cross_f32_kernel, plan.few, s.columns(), plan.splits, q, kv, src_len, ctx, lse, parts)
  return check_launch();
}

int launch_cross_attention_f32_bwd(const CrossShape& s, const float* q, const float* kv, const int32_t* src_len, const float* ctx,
                                   const float* dctx, const float* lse, float* dq, float* dkv, float* dvec, hipStream_t st) {
  const CrossGeo g(s);
  const bool few = share_columns(s.B * s.kv_heads * ((s.columns() + 31) / 32), s.Lk, 1.0);
  const bool few_states = share_columns(s.B * s.kv_heads * ((s.Lk + 31) / 32), s.columns(), 1.0);
  MOE_CROSS_F32(cross_f32_dq_kernel, few, s.columns(), 1, q, kv, src_len, ctx, dctx, lse, dq, dvec)
  MOE_CROSS_F32(cross_f32_dkv_kernel, few_states, s.Lk, 1, q, kv, src_len, dctx, lse, dvec, dkv)
  return check_launch();
}

}  // namespace moe
