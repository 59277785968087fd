// The loss at the end of a model (the paper trains its models on the cross entropy of the next word, over vocabularies of 32k
// and 64k entries): x [N,M] are the last hidden states, w [V,M] one row per vocabulary entry, z = x . w^T the logits.
//
//   cross entropy   loss_n = lse_n - z[n,target_n],  lse_n = log sum_v exp z[n,v]
//                          = log(1 + exp d_n),  d_n = log sum_{v != target_n} exp z[n,v]  -  z[n,target_n]
//                   dz[n,v] = g_n (exp(z[n,v] - lse_n) - [v = target_n]),  exp(-loss_n) - 1 at the target
//   distillation    q = softmax(t_n / T) over a teacher's K entries,  lse_n = log sum_v exp(z[n,v] / T)
//                   loss_n = sum_k q_k (log q_k - z[n,i_k] / T + lse_n)
//                   dz[n,v] = g_n / T (exp(z[n,v] / T - lse_n) - sum_{k: i_k = v} q_k)
//   both            dx = dz . w,  dw = dz^T . x
//
// The logits are never kept: the forward product leaves of every row and wavefront tile the maximum and the sum of exponentials
// (8 bytes for 32 to 256 logits), a target's logit left out of them and by itself, so that the loss of a token that is nearly sure is
// no difference of near numbers (of lse and a logit, 16 each, 1e-6 would be left of 1e-4); the backward pass multiplies again and keeps one piece of the vocabulary's dz for the two
// products that read it, in bf16 rounded once, as the upstream gradients of the expert layers are.
//
// The passes over rows take 36 of 1600 us forward, 65 of 5100 backward (32768 tokens, M 1024, V 32000): bound by memory.
//
// Tokens without a target (padding, prompts) are left out of every product: the rows that have one are numbered first
// (vocab_rows_kernel), so neither their work nor what their x holds, NaN included, reaches anything.
//
// This file holds the passes over rows; the products are in expert_gemm.hip and gemm_f32.hip.
#include <math.h>
#include "common.h"

namespace moe {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// ---------------------------------------------------------------- rows with a target
// perm[p] = the p-th token with a target, pos[n] = its p or -1, kept[0] their number.  A block of 1024 threads numbers its
// tokens and counts those before them by itself: no order of blocks, one launch.
struct VocabRowArgs {
  const int32_t* has;          // targets (a target is 0 .. entries - 1), or with entries 0: flags
  int entries;
  long long N;
  int32_t *perm, *pos, *kept;
  // forward: zeros for the tokens without a target
  float *loss, *lse;
  int32_t* hit;                      // NULL, or the packed rows' targets
  // backward: what the products read per packed row
  const float *loss_in, *lse_in, *dloss;
  float inv_t, *lse2, *grad, *hit_value;
  // backward with dx on 256 x 256 tiles: its ranges are chosen here, for the rows that there are
  int dx_entries, dx_tiles_n, M;     // dx_entries 0: no
  long long dx_rows;                 // rows of sums that there is room for
  VocabTileCost dx_cost;
};
constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / 64;
// kept[1] ranges of kept[2] entries: the fastest by tiles_time of vocab_dx_plan, one candidate per lane
__device__ void vocab_dx_ranges(const VocabRowArgs& a, int rows) {
  const int lane = threadIdx.x & 63, want = lane + 1, tiles = (rows + 255) / 256 * a.dx_tiles_n;
  const int k = ((a.dx_entries + want - 1) / want + 63) / 64 * 64, n = (a.dx_entries + k - 1) / k;
  float us = 3e38f;
  if (want == 1 || (k >= 256 && n == want && (long long)n * rows <= a.dx_rows))
    us = (float)(vocab_tiles_time(a.dx_cost, (long long)n * tiles, k, 2.0 * rows * a.dx_entries) +
                 1.6e-6 * n * rows * a.M);
  float best = us;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = fminf(best, __shfl_xor(best, o, 64));
  if (lane == __builtin_ctzll(__builtin_amdgcn_ballot_w64(us == best))) { a.kept[1] = n; a.kept[2] = k; }
}
// token n, whose target is `target`, is packed row p
struct TokenData { float lse, loss, dloss; };
__device__ TokenData vocab_token_data(const VocabRowArgs& a, long long n) {
  return TokenData{a.lse_in[n], a.hit != nullptr ? a.loss_in[n] : 0.f, a.dloss[n]};
}
__device__ void vocab_row_data(const VocabRowArgs& a, int p, long long n, int32_t target, const TokenData& d) {
  a.perm[p] = (int32_t)n;
  if (a.hit != nullptr) a.hit[p] = target;
  if (a.lse_in == nullptr) return;
  const float g = d.dloss * a.inv_t;
  a.lse2[p] = d.lse * kLog2e;
  a.grad[p] = g;
  if (a.hit != nullptr) a.hit_value[p] = expm1f(-d.loss) * g;  // exp(z - lse) - 1 at the target, where z - lse = -loss
}
// PER neighbouring tokens a thread.  One, for whole lines of all that is written, as long as counting the tokens before takes few
// fetches (8336 tokens, all that a backward pass needs: four 9.5 us, one 4.8; 32768: 15.8 and 7.2); four where blocks are many.
template <int PER>
__global__ __launch_bounds__(kRowThreads) void vocab_rows_kernel(VocabRowArgs a) {
  const long long first = (long long)blockIdx.x * (PER * kRowThreads);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto valid = [&](int32_t v) { return a.entries != 0 ? (uint32_t)v < (uint32_t)a.entries : v != 0; };
  const long long n0 = first + PER * tid;
  int32_t v[PER];
  TokenData data[PER] = {};
  int own = 0, before = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const long long n = n0 + i < a.N ? n0 + i : a.N - 1;
    v[i] = a.has[n];
    if (a.lse_in != nullptr) data[i] = vocab_token_data(a, n);
  }
#pragma unroll 8
  for (long long i = 4 * tid; i < first; i += 4 * kRowThreads) {
    const int4 u = *reinterpret_cast<const int4*>(a.has + i);
    before += (int)valid(u.x) + (int)valid(u.y) + (int)valid(u.z) + (int)valid(u.w);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) own += (int)(n0 + i < a.N && valid(v[i]));
  int incl = own;                                              // within the wavefront, then of the wavefronts before
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
    before += __shfl_xor(before, o, 64);
  }
  __shared__ int sums[2 * kRowWaves];
  if (lane == 63) { sums[wave] = incl; sums[kRowWaves + wave] = before; }
  __syncthreads();
  int p = incl - own, total = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    p += sums[kRowWaves + w] + (w < wave ? sums[w] : 0);
    total += sums[kRowWaves + w] + sums[w];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const long long n = n0 + i;
    if (n >= a.N) break;
    const bool ok = valid(v[i]);
    if (a.pos != nullptr) a.pos[n] = ok ? p : -1;
    if (!ok) {
      if (a.loss != nullptr) { a.loss[n] = 0.f; a.lse[n] = 0.f; }
      continue;
    }
    vocab_row_data(a, p, n, v[i], data[i]);
    ++p;
  }
  if (blockIdx.x == gridDim.x - 1 && wave == kRowWaves - 1) {  // (the wavefront with the fewest tokens)
    if (lane == 0) a.kept[0] = total;
    if (a.dx_entries != 0) vocab_dx_ranges(a, total);
  }
}

// ---------------------------------------------------------------- single logits
// The dot product of two rows of M by the 16 lanes l of a group, in all of them; rows in pieces of 16 bytes.
template <typename T>
__device__ __forceinline__ float row_dot(const uint4* __restrict__ x, const uint4* __restrict__ w, int pieces, int l) {
  constexpr int K = Vec16<T>::kElts;
  float acc = 0.f;
#pragma unroll 4
  for (int i = l; i < pieces; i += 16) {
    float a[K], b[K];
    Vec16<T>::unpack(x[i], a);
    Vec16<T>::unpack(w[i], b);
#pragma unroll
    for (int k = 0; k < K; ++k) acc = fmaf(a[k], b[k], acc);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) acc += __shfl_xor(acc, o, 64);
  return acc;
}

// ---------------------------------------------------------------- the teacher's entries
// An entry is there if its index is one of the vocabulary's and its logit is not -inf.
struct TeacherArgs {
  const int32_t* idx;          // [N,K]
  const float* logit;          // [N,K]
  int K, entries;
  float inv_t;
};
__device__ __forceinline__ bool teacher_has(const TeacherArgs& t, int32_t i, float l) {
  return (uint32_t)i < (uint32_t)t.entries && l != -INFINITY;
}
// A wavefront's look at one token: maximum of its teacher's logits and the sum of exponentials, and whether there is any entry
__device__ __forceinline__ bool teacher_stat(const TeacherArgs& t, long long n, float2* stat) {
  const int lane = threadIdx.x & 63;
  const int32_t* idx = t.idx + n * t.K;
  const float* logit = t.logit + n * t.K;
  float mx = -INFINITY;
  bool any = false;
  for (int k = lane; k < t.K; k += 64)
    if (teacher_has(t, idx[k], logit[k])) { mx = fmaxf(mx, logit[k]); any = true; }
  mx = wave_max(mx);
  float sum = 0.f;
  for (int k = lane; k < t.K; k += 64)
    if (teacher_has(t, idx[k], logit[k])) sum += expf((logit[k] - mx) * t.inv_t);
  *stat = float2{mx, wave_sum(sum)};
  return __builtin_amdgcn_ballot_w64(any) != 0;
}
// The student's logits z at the entries of token n, 0 where there is none: a group of 16 lanes per entry, of 16 groups `at` .. by
// `groups` (a wavefront's four stay together: row_dot's shuffles)
template <typename T>
__device__ __forceinline__ void entry_logits(const TeacherArgs& t, long long n, const uint4* __restrict__ x,
                                             const uint4* __restrict__ w, int pieces, float* __restrict__ z, int at, int groups) {
  const int l = threadIdx.x & 15, first = at & ~3;
  for (int k0 = first; k0 < t.K; k0 += groups) {
    const int k = k0 + (at & 3);
    const bool ok = k < t.K && teacher_has(t, t.idx[n * t.K + k], t.logit[n * t.K + k]);
    const float d = row_dot<T>(x + (size_t)n * pieces, w + (size_t)(ok ? t.idx[n * t.K + k] : 0) * pieces, ok ? pieces : 0, l);
    if (l == 0 && k < t.K) z[n * t.K + k] = ok ? d : 0.f;
  }
}
// one wavefront per token; z may be NULL.  SORTED: the logits of the entries that are there come from the product (vocab_sort_kernel)
template <typename T, bool SORTED>
__global__ __launch_bounds__(256) void vocab_teacher_kernel(TeacherArgs t, const uint4* __restrict__ x,
                                                            const uint4* __restrict__ w, int pieces, long long N,
                                                            float2* __restrict__ stat, int32_t* __restrict__ has,
                                                            float* __restrict__ z) {
  const long long n = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= N) return;
  float2 s;
  const bool any = teacher_stat(t, n, &s);
  if ((threadIdx.x & 63) == 0) { stat[n] = s; has[n] = any; }
  if (SORTED) {
    for (int k = threadIdx.x & 63; k < t.K; k += 64)
      if (!teacher_has(t, t.idx[n * t.K + k], t.logit[n * t.K + k])) z[n * t.K + k] = 0.f;
  } else if (z != nullptr) {
    entry_logits<T>(t, n, x, w, pieces, z, (threadIdx.x >> 4) & 3, 4);
  }
}
// The entries of the packed rows in the order of the product's 256 x 256 tiles and their eight wavefronts, so that each finds its
// own (a handful, where their dot products one by one would read a row of w each: 8192 tokens, M 1024, 32 entries 86 us).  A block
// per row tile; the entries of a wavefront come in no fixed order, which no result depends on.
__global__ __launch_bounds__(1024) void vocab_sort_kernel(TeacherArgs t, const int32_t* __restrict__ perm,
                                                          const int32_t* __restrict__ kept, int lists,
                                                          int32_t* __restrict__ starts, uint2* __restrict__ sorted) {
  extern __shared__ int place[];                               // [lists] counts, then where the next entry goes
  __shared__ int sums[16];
  const int p0 = blockIdx.x * 256, rows = kept[0], tid = threadIdx.x, lane = tid & 63;
  if (p0 >= rows) return;
  const int entries = (rows - p0 < 256 ? rows - p0 : 256) * t.K;
  for (int i = tid; i < lists; i += 1024) place[i] = 0;
  __syncthreads();
  auto list_of = [](int r, int i) { return 8 * (i >> 8) + 4 * (r >> 6 & 1) + (i >> 6 & 3); };      // tile, wavefront
  auto each = [&](auto take) {
    for (int e = tid; e < entries; e += 1024) {
      const int r = e / t.K, k = e - r * t.K;
      const long long at = (long long)perm[p0 + r] * t.K + k;
      const int32_t i = t.idx[at];
      if (teacher_has(t, i, t.logit[at])) take(r, i, (uint32_t)at);
    }
  };
  each([&](int r, int i, uint32_t) { atomicAdd(&place[list_of(r, i)], 1); });
  __syncthreads();
  // running counts: a thread's stretch of lists, the stretches in a wavefront, the wavefronts
  const int per = (lists + 1023) / 1024, b0 = tid * per;
  int own = 0;
  for (int i = b0; i < b0 + per && i < lists; ++i) own += place[i];
  int incl = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  if (lane == 63) sums[tid >> 6] = incl;
  __syncthreads();
  int run = incl - own;
  for (int w = 0; w < (tid >> 6); ++w) run += sums[w];
  int32_t* const mine = starts + (size_t)blockIdx.x * (lists + 1);
  for (int i = b0; i < b0 + per && i < lists; ++i) {
    const int n = place[i];
    place[i] = mine[i] = run;
    run += n;
  }
  if (tid == 1023) mine[lists] = run;                          // (of all: its stretch is the last, empty or not)
  __syncthreads();
  each([&](int r, int i, uint32_t at) {
    sorted[(size_t)p0 * t.K + atomicAdd(&place[list_of(r, i)], 1)] = uint2{(uint32_t)(r << 8 | (i & 255)), at};
  });
}
constexpr int kSortTiles = 2000;                               // column tiles whose counts fit 64 KB of LDS

// Up to 1024 tokens, a block each: what vocab_rows_kernel and vocab_pack_kernel do, in one launch, and up to 64 what
// vocab_teacher_kernel does too (with t.K).  Every block looks at all tokens to number its own.  A backward pass of 200 tokens, M 512,
// V 2000 29.4 -> 26.6 us.
constexpr int kFewTokens = 64, kBlockTokens = 1024;
template <typename T>
__global__ __launch_bounds__(256) void vocab_few_kernel(VocabRowArgs a, TeacherArgs t, const uint4* __restrict__ x,
                                                        const uint4* __restrict__ w, int pieces, float2* __restrict__ stat,
                                                        float* __restrict__ z, uint4* __restrict__ packed) {
  const int n = blockIdx.x, N = (int)a.N, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __shared__ int has[kFewTokens];
  __shared__ int2 counts[4];                                   // tokens with a target: before this one, all
  const TokenData data = threadIdx.x == 0 && a.lse_in != nullptr ? vocab_token_data(a, n) : TokenData{0.f, 0.f, 0.f};
  if (t.K != 0) {
    if (threadIdx.x < kFewTokens) has[threadIdx.x] = 0;
    __syncthreads();
    for (int e = threadIdx.x; e < N * t.K; e += 256)
      if (teacher_has(t, t.idx[e], t.logit[e])) has[e / t.K] = 1;
    if (wave == 0) {
      float2 s;
      teacher_stat(t, n, &s);
      if (lane == 0) stat[n] = s;
    }
    if (z != nullptr) entry_logits<T>(t, n, x, w, pieces, z, threadIdx.x >> 4, 16);
    __syncthreads();
  }
  auto counts_in = [&](int i) { return t.K != 0 ? has[i] != 0 : a.entries != 0 ? (uint32_t)a.has[i] < (uint32_t)a.entries : a.has[i] != 0; };
  int2 c = {0, 0};
  for (int i0 = 64 * wave; i0 < N; i0 += 256) {
    const uint64_t which = __builtin_amdgcn_ballot_w64(i0 + lane < N && counts_in(i0 + lane));
    c.x += __builtin_popcountll(n >= i0 + 64 ? which : n > i0 ? which & ((1ull << (n - i0)) - 1) : 0);
    c.y += __builtin_popcountll(which);
  }
  if (lane == 0) counts[wave] = c;
  __syncthreads();
  const int p = counts[0].x + counts[1].x + counts[2].x + counts[3].x, rows = counts[0].y + counts[1].y + counts[2].y + counts[3].y;
  const bool ok = counts_in(n);
  if (threadIdx.x == 0) {
    if (n == 0) a.kept[0] = rows;
    if (a.pos != nullptr) a.pos[n] = ok ? p : -1;
    if (ok) vocab_row_data(a, p, n, t.K == 0 ? a.has[n] : 0, data);
    else if (a.loss != nullptr) { a.loss[n] = 0.f; a.lse[n] = 0.f; }
  }
  if (n == 0 && wave == 0 && a.dx_entries != 0) vocab_dx_ranges(a, rows);
  if (packed == nullptr) return;
  if (ok)
    for (int i = threadIdx.x; i < pieces; i += 256) packed[(size_t)p * pieces + i] = x[(size_t)n * pieces + i];
  // rows of zeros up to whole 64: the p-th block without a target writes the one behind the last that many on
  else
    for (int i = threadIdx.x; i < pieces; i += 256) packed[(size_t)(rows + n - p) * pieces + i] = uint4{0u, 0u, 0u, 0u};
  if (n == N - 1)
    for (int r = N; r < (N + 63) / 64 * 64; ++r)
      for (int i = threadIdx.x; i < pieces; i += 256) packed[(size_t)r * pieces + i] = uint4{0u, 0u, 0u, 0u};
}

// ---------------------------------------------------------------- loss of the packed rows
// ROWS rows a block: the 256 / ROWS threads of a row meet the slots' maxima and sums, then the 16 lanes of a group finish one row:
// the loss and log-sum from those of the other entries and the target's logit (cross entropy), or the sum over the teacher's entries.
// 16 rows read whole lines of the statistics; a row by itself is done sooner where there are few.  kept NULL: no rows were numbered,
// row n is token n.
template <bool TEACHER, int ROWS>
__global__ __launch_bounds__(256) void vocab_finish_kernel(const float2* __restrict__ stats, int slots, long long N,
                                                           const int32_t* __restrict__ perm, const int32_t* __restrict__ kept,
                                                           const int32_t* __restrict__ target, const int32_t* __restrict__ flags,
                                                           const float* __restrict__ hit_logit, TeacherArgs t,
                                                           const float2* __restrict__ tstat, const float* __restrict__ z,
                                                           float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 part[16][17];
  __shared__ float2 sum_of[16];                                // 2^(x + y) is the sum
  const long long p0 = (long long)blockIdx.x * ROWS;
  const int rows = kept != nullptr ? kept[0] : (int)N;
  if (p0 >= rows) return;
  const int r = threadIdx.x & 15, sl = threadIdx.x >> 4;
  const long long p = ROWS == 1 ? p0 : p0 + r < rows ? p0 + r : rows - 1;
  float m = -INFINITY, s = 0.f;
  auto meet = [](float& m, float& s, const float2 o) {
    const float up = fmaxf(m, o.x), at = up == -INFINITY ? 0.f : up;
    s = s * __builtin_amdgcn_exp2f(m - at) + o.y * __builtin_amdgcn_exp2f(o.x - at);
    m = up;
  };
#pragma unroll 4
  for (int i = ROWS == 1 ? threadIdx.x : sl; i < slots; i += 256 / ROWS) meet(m, s, stats[(size_t)i * N + p]);
  part[r][sl] = float2{m, s};
  __syncthreads();
  if (threadIdx.x < 16) {
#pragma unroll
    for (int i = 1; i < 16; ++i) meet(m, s, part[r][i]);
    if (ROWS == 1) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) meet(m, s, float2{__shfl_xor(m, o, 64), __shfl_xor(s, o, 64)});
    }
    sum_of[r] = float2{m, log2f(s)};
  }
  __syncthreads();
  if (sl >= ROWS || p0 + sl >= rows) return;                   // (whole groups of 16 lanes)
  if (kept == nullptr && (TEACHER ? flags[p0 + sl] == 0 : (uint32_t)target[p0 + sl] >= (uint32_t)t.entries)) {
    if (r == 0) { loss[p0 + sl] = 0.f; lse[p0 + sl] = 0.f; }
    return;
  }
  const long long n = kept != nullptr ? perm[p0 + sl] : p0 + sl;
  const float2 q2 = sum_of[sl];
  float l = (q2.x + q2.y) * kLn2, out;
  if (!TEACHER) {
    // d: what is added to the fma's difference is small where that is; the larger of the two logits stands outside the logarithm
    const float zt = hit_logit[p0 + sl], d = (fmaf(-kLog2e, zt, q2.x) + q2.y) * kLn2, more = log1pf(expf(-fabsf(d)));
    out = zt == INFINITY ? NAN : (d > 0.f ? d : 0.f) + more;
    l = (d > 0.f ? l : zt) + more;
  } else {
    const float2 ts = tstat[n];
    const float inv = 1.f / ts.y, log_sum = logf(ts.y);
    out = 0.f;
    for (int k = r; k < t.K; k += 16) {
      const float tl = t.logit[n * t.K + k];
      if (!teacher_has(t, t.idx[n * t.K + k], tl)) continue;
      const float a = (tl - ts.x) * t.inv_t, q = expf(a) * inv;
      if (!(q == 0.f)) out += q * (a - log_sum - z[n * t.K + k] * t.inv_t + l);     // (0 log 0 = 0; NaN stays)
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) out += __shfl_xor(out, o, 64);
  }
  if (r == 0) { loss[n] = out; lse[n] = l; }
}

// ---------------------------------------------------------------- dz at the teacher's entries
// One wavefront per packed row: (exp(z/T - lse) - the q of all its entries with that index) g/T, at the entries of this piece.
template <typename T>
__global__ __launch_bounds__(256) void vocab_entry_grad_kernel(TeacherArgs t, const float2* __restrict__ tstat,
                                                               const float* __restrict__ z, VocabRows a,
                                                               const int32_t* __restrict__ perm,
                                                               const int32_t* __restrict__ kept, T* __restrict__ dz, int ld,
                                                               int entries) {
  extern __shared__ float2 entry_smem[];                       // [4 wavefronts][K]: index (its bits) and q
  const long long p = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (p >= kept[0]) return;
  const int lane = threadIdx.x & 63;
  float2* const e = entry_smem + (threadIdx.x >> 6) * t.K;
  const long long n = perm[p];
  const float2 ts = tstat[n];
  const float inv = 1.f / ts.y;
  for (int k = lane; k < t.K; k += 64) {
    const int32_t i = t.idx[n * t.K + k];
    const float l = t.logit[n * t.K + k];
    const bool ok = teacher_has(t, i, l);
    e[k] = float2{__int_as_float(ok ? i : -1), ok ? expf((l - ts.x) * t.inv_t) * inv : 0.f};
  }
  __builtin_amdgcn_wave_barrier();
  for (int k = lane; k < t.K; k += 64) {
    const int i = __float_as_int(e[k].x), at = i - a.first;
    if (i < 0 || at < 0 || at >= entries) continue;
    float q = 0.f;
    for (int j = 0; j < t.K; ++j) q += __float_as_int(e[j].x) == i ? e[j].y : 0.f;
    const float d = __builtin_amdgcn_exp2f(fmaf(z[n * t.K + k], a.scale, -a.lse2[p])) - q;
    Elt<T>::store(dz + (size_t)p * ld + at, d * a.grad[p]);
  }
}

// ---------------------------------------------------------------- rows in and out
// packed[p] = x[perm[p]], 16 bytes a thread: dw sums over rows that lie together, in whole 64 (zeros behind the last)
__global__ __launch_bounds__(256) void vocab_pack_kernel(const uint4* __restrict__ x, uint4* __restrict__ packed,
                                                         const int32_t* __restrict__ perm, const int32_t* __restrict__ kept,
                                                         int pieces, long long total) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const long long p = i / pieces;
  const int rows = kept[0];
  if (p >= (rows + 63) / 64 * 64) return;
  packed[i] = p < rows ? x[(size_t)perm[p] * pieces + (i - p * pieces)] : uint4{0u, 0u, 0u, 0u};
}
// dx[n] = the sum of the ranges' sums of its packed row, zeros without one; kept not NULL: as many ranges as kept[1], of as many rows
// PARTS neighbouring threads share the ranges of a piece (few rows: more loads on their way at once).
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void vocab_dx_kernel(const float4* __restrict__ sums, int splits, long long N,
                                                       const int32_t* __restrict__ kept, const int32_t* __restrict__ pos,
                                                       uint4* __restrict__ dx, int pieces) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x, i = id / PARTS;
  const int part = (int)(id % PARTS);
  if (i >= N * pieces) return;                                 // (a piece's threads together)
  constexpr int K = Vec16<T>::kElts;
  const long long n = i / pieces;
  const int p = pos[n];
  float v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.f;
  if (p >= 0) {
    const size_t at = ((size_t)p * pieces + (i - n * pieces)) * (K / 4);
    const size_t next = (size_t)(kept != nullptr ? kept[0] : N) * pieces * (K / 4);
    if (kept != nullptr) splits = kept[1];
#pragma unroll 4
    for (int s = part; s < splits; s += PARTS)
#pragma unroll
      for (int k = 0; k < K; k += 4) {
        const float4 f = sums[s * next + at + k / 4];
        v[k] += f.x; v[k + 1] += f.y; v[k + 2] += f.z; v[k + 3] += f.w;
      }
  }
#pragma unroll
  for (int o = 1; o < PARTS; o <<= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, 64);
  if (part == 0) dx[i] = Vec16<T>::pack(v);
}

// dw = the sum over ranges of rows, 16 bytes a thread
template <typename T>
__global__ __launch_bounds__(256) void vocab_dw_kernel(const float4* __restrict__ sums, int splits, long long total,
                                                       uint4* __restrict__ dw) {
  constexpr int K = Vec16<T>::kElts;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  float v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.f;
#pragma unroll 4
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int k = 0; k < K; k += 4) {
      const float4 f = sums[(s * total + i) * (K / 4) + k / 4];
      v[k] += f.x; v[k + 1] += f.y; v[k + 2] += f.z; v[k + 3] += f.w;
    }
  dw[i] = Vec16<T>::pack(v);
}

unsigned blocks_of(long long threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace

// Pieces of the vocabulary: as many entries as keep a piece of [N, entries] within 1 GiB, 4096 at least (a sum of dx over
// fewer would spend its time on adding to dx), all alike; in whole 256.
VocabPieces vocab_pieces(const moe_config& c, const moe_vocab_dims& d) {
  const long long N = (long long)c.G * c.S, elt = c.act_dtype == MOE_F32 ? 4 : 2;
  long long most = d.piece;
  if (most == 0) {
    most = (1LL << 30) / (N * elt);
    if (most < 4096) most = 4096;
  }
  if (most > d.V) most = d.V;
  const long long n = (d.V + most - 1) / most;
  VocabPieces p;
  p.entries = (int)(((d.V + n - 1) / n + 255) / 256 * 256);
  p.count = (d.V + p.entries - 1) / p.entries;
  return p;
}

// The product of the logits on tiles leaves those at the teacher's entries too.  Asked one by one they read as many rows of w, 6 GB a
// ms; the sort and the tiles' looks at it take about 16 us: worth it for more than 100 MB (8192 tokens, M 1024, V 64000, 32 entries
// 952 -> 911 us), and then also a reason for tiles (13384 tokens, M 1256, V 1630, 25 entries 148 -> 98 us).  us saved, or 0: not sorted.
static double vocab_sort_saves(const moe_config& c, const moe_vocab_dims& d) {
  const double bytes = 2.0 * c.G * c.S * d.K * c.M;
  return (d.V + 255) / 256 <= kSortTiles && bytes > 1e8 ? bytes / 6e6 - 16.0 : 0.0;
}
// How the forward pass goes about the logits.  all: those of tokens without a target too, which are not read later, where that takes no
// longer than to number the others: one row tile, or a product expected within 12 us (200 tokens, M 512, V 8000 19.5 -> 16.2 us, whether
// 5 or 60 of 100 have none)
struct VocabForwardPlan { bool packs, sorts, all; int slots; };
static VocabForwardPlan forward_plan(const moe_config& c, const moe_vocab_dims& d, bool teacher) {
  const int N = c.G * c.S;
  if (c.act_dtype == MOE_F32) return {false, false, false, vocab_stat_slots_f32(N, d.V, c.M)};
  const double saved = teacher ? vocab_sort_saves(c, d) : 0.0;
  const bool packs = vocab_logits_on_tiles(N, d.V, c.M, true, saved);
  return {packs, packs && saved > 0, !packs && (N <= kFewTokens || vocab_logits_edge_us(N, d.V, c.M) < 12.0),
          vocab_stat_slots(N, d.V, c.M, saved)};
}

VocabWs carve_vocab(const moe_config& c, const moe_vocab_dims& d, bool teacher, bool backward) {
  const size_t N = (size_t)c.G * c.S, elt = c.act_dtype == MOE_F32 ? 4 : 2;
  const VocabPieces p = vocab_pieces(c, d);
  VocabWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes, 256); return o; };
  const size_t whole = align_up(N, 256);                       // rows in whole tiles
  w.kept = take(12);
  w.perm = take(N * 4);
  w.tstat = take(teacher ? N * 8 : 0);
  w.has = take(teacher ? N * 4 : 0);
  if (!backward) {
    const VocabForwardPlan f = forward_plan(c, d, teacher);
    w.slots = f.slots;
    w.packed = take(f.packs ? whole * c.M * elt : 0);
    w.starts = take(f.sorts ? (whole / 256 * ((size_t)8 * ((d.V + 255) / 256) + 1) + 64) * 4 : 0);      // (a wavefront fetches 64)
    w.sorted = take(f.sorts ? (N * d.K + 64) * 8 : 0);             // (a wavefront fetches whole 32)
    w.stats = take((size_t)w.slots * N * 8);
    w.hit = take(teacher ? 0 : N * 4);
    w.hit_logit = take(teacher ? 0 : N * 4);
  } else {
    w.pos = take(N * 4);
    w.lse2 = take(N * 4);
    w.grad = take(N * 4);
    w.hit = take(N * 4);
    w.hit_value = take(N * 4);
    const int entries = p.entries < d.V ? p.entries : d.V;
    w.dx_plan = c.act_dtype == MOE_F32 ? vocab_dx_plan_f32((int)N, entries, c.M) : vocab_dx_plan((int)N, entries, c.M);
    w.packed = take(whole * c.M * elt);
    w.dz = take(whole * p.entries * elt);
    w.sums = take((size_t)w.dx_plan.splits * N * c.M * 4);
    w.dw_splits = c.act_dtype == MOE_F32 ? vocab_dw_splits_f32((int)N, entries, c.M)
                                         : vocab_dw_splits((int)N, entries, c.M, w.dx_plan);
    w.dw_sums = take(w.dw_splits > 1 ? (size_t)w.dw_splits * entries * c.M * 4 : 0);
  }
  w.total = off;
  return w;
}

// sorted: not the logits of the entries that are there
static int launch_teacher(const moe_config& c, const TeacherArgs& t, const void* x, const void* w, char* base, const VocabWs& ws,
                          float* z, bool sorted, hipStream_t st) {
  const long long N = (long long)c.G * c.S;
  const int pieces = c.M * (c.act_dtype == MOE_F32 ? 4 : 2) / 16;
  auto args = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((N + 3) / 4)), dim3(256), 0, st, t, static_cast<const uint4*>(x),
                       static_cast<const uint4*>(w), pieces, N, reinterpret_cast<float2*>(base + ws.tstat),
                       reinterpret_cast<int32_t*>(base + ws.has), z);
  };
  if (sorted) args(vocab_teacher_kernel<bf16_t, true>);
  else if (c.act_dtype == MOE_F32) args(vocab_teacher_kernel<float, false>);
  else args(vocab_teacher_kernel<bf16_t, false>);
  return check_launch();
}

static VocabRowArgs row_args(const moe_config& c, const moe_vocab_dims& d, const VocabCall& a, char* base, const VocabWs& ws) {
  VocabRowArgs r{};
  r.has = a.target != nullptr ? a.target : reinterpret_cast<const int32_t*>(base + ws.has);
  r.entries = a.target != nullptr ? d.V : 0;
  r.N = (long long)c.G * c.S;
  r.perm = reinterpret_cast<int32_t*>(base + ws.perm);
  r.kept = reinterpret_cast<int32_t*>(base + ws.kept);
  return r;
}
// up to 1024 tokens, with a teacher 64; packed and z may be NULL
static int launch_few(const moe_config& c, const VocabRowArgs& r, const TeacherArgs& t, const VocabCall& a, char* base,
                      const VocabWs& ws, float* z, void* packed, hipStream_t st) {
  const int pieces = c.M * (c.act_dtype == MOE_F32 ? 4 : 2) / 16;
  auto args = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)r.N), dim3(256), 0, st, r, t, static_cast<const uint4*>(a.x),
                       static_cast<const uint4*>(a.w), pieces, reinterpret_cast<float2*>(base + ws.tstat), z,
                       static_cast<uint4*>(packed));
  };
  if (c.act_dtype == MOE_F32) args(vocab_few_kernel<float>); else args(vocab_few_kernel<bf16_t>);
  return check_launch();
}
static int launch_rows(const VocabRowArgs& r, hipStream_t st) {
  const int per = r.N <= 64 * kRowThreads ? 1 : 4, tokens = per * kRowThreads;
  hipLaunchKernelGGL(per == 1 ? vocab_rows_kernel<1> : vocab_rows_kernel<4>, dim3((unsigned)((r.N + tokens - 1) / tokens)),
                     dim3(kRowThreads), 0, st, r);
  return check_launch();
}

static int launch_pack(const moe_config& c, const void* x, void* packed, const VocabRowArgs& r, hipStream_t st) {
  const int pieces = c.M * (c.act_dtype == MOE_F32 ? 4 : 2) / 16;
  const long long total = (r.N + 63) / 64 * 64 * pieces;
  hipLaunchKernelGGL(vocab_pack_kernel, dim3(blocks_of(total)), dim3(256), 0, st, static_cast<const uint4*>(x),
                     static_cast<uint4*>(packed), r.perm, r.kept, pieces, total);
  return check_launch();
}

// the rows numbered from targets or flags, and x packed if packed is not NULL
static int launch_numbered(const moe_config& c, const VocabRowArgs& r, const VocabCall& a, char* base, const VocabWs& ws, void* packed,
                           hipStream_t st) {
  if (packed != nullptr && r.N <= kBlockTokens) return launch_few(c, r, TeacherArgs{}, a, base, ws, nullptr, packed, st);
  const int rc = launch_rows(r, st);
  return rc != MOE_OK || packed == nullptr ? rc : launch_pack(c, a.x, packed, r, st);
}

int launch_vocab_forward(const moe_config& c, const moe_vocab_dims& d, const VocabCall& a, void* base_, const VocabWs& ws,
                         hipStream_t st) {
  char* const base = static_cast<char*>(base_);
  const long long N = (long long)c.G * c.S;
  const bool f32 = c.act_dtype == MOE_F32;
  const float inv_t = a.target != nullptr ? 1.f : 1.f / d.temperature;
  const TeacherArgs t{a.idx, a.logit, a.target != nullptr ? 0 : d.K, d.V, inv_t};
  int rc = MOE_OK;
  VocabRowArgs r = row_args(c, d, a, base, ws);
  r.loss = a.loss;
  r.lse = a.lse;
  if (a.target != nullptr) r.hit = reinterpret_cast<int32_t*>(base + ws.hit);
  const VocabForwardPlan plan = forward_plan(c, d, a.target == nullptr);
  const bool packs = plan.packs, sorts = plan.sorts;
  const bool few = N <= kFewTokens && !packs, all = plan.all && !(few && a.target == nullptr);
  if (few) {
    if (!all) rc = launch_few(c, r, t, a, base, ws, a.entry_logit, nullptr, st);
  } else {
    if (a.target == nullptr) rc = launch_teacher(c, t, a.x, a.w, base, ws, a.entry_logit, sorts, st);
    if (rc == MOE_OK && !all) rc = launch_numbered(c, r, a, base, ws, packs ? base + ws.packed : nullptr, st);
    if (rc == MOE_OK && sorts) {
      const int lists = 8 * ((d.V + 255) / 256);
      hipLaunchKernelGGL(vocab_sort_kernel, dim3((unsigned)((N + 255) / 256)), dim3(1024), (size_t)lists * sizeof(int), st, t,
                         r.perm, r.kept, lists, reinterpret_cast<int32_t*>(base + ws.starts),
                         reinterpret_cast<uint2*>(base + ws.sorted));
      rc = check_launch();
    }
  }
  if (rc != MOE_OK) return rc;
  float2* const stats = reinterpret_cast<float2*>(base + ws.stats);
  GemmArgs g{packs ? base + ws.packed : a.x, a.w, nullptr};
  g.gather = packs || all ? nullptr : r.perm;
  g.kept = all ? nullptr : r.kept;
  g.vocab.scale = kLog2e * inv_t;
  g.vocab.stats = stats;
  float* const hit_logit = reinterpret_cast<float*>(base + ws.hit_logit);
  if (a.target != nullptr) {
    g.vocab.hit = all ? a.target : r.hit;                      // (one outside the vocabulary is in no column)
    g.vocab.hit_value = hit_logit;
  }
  if (sorts) {
    g.vocab.starts = reinterpret_cast<const int32_t*>(base + ws.starts);
    g.vocab.sorted = reinterpret_cast<const uint2*>(base + ws.sorted);
    g.vocab.entry_logit = a.entry_logit;
    g.vocab.K = d.K;
  }
  rc = f32 ? launch_gemm_f32(kDataGrad, g, 1, (int)N, d.V, c.M, st) : launch_vocab_logits(g, (int)N, d.V, c.M, st);
  if (rc != MOE_OK) return rc;
  const bool single = N <= 1024;                               // a block per row where 16 rows each would not fill the units
  auto finish = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(single ? N : (N + 15) / 16)), dim3(256), 0, st, stats, ws.slots, N, r.perm, g.kept,
                       a.target, r.has, hit_logit, t, reinterpret_cast<const float2*>(base + ws.tstat), a.entry_logit, a.loss, a.lse);
  };
  if (a.target != nullptr) finish(single ? vocab_finish_kernel<false, 1> : vocab_finish_kernel<false, 16>);
  else finish(single ? vocab_finish_kernel<true, 1> : vocab_finish_kernel<true, 16>);
  return check_launch();
}

int launch_vocab_backward(const moe_config& c, const moe_vocab_dims& d, const VocabCall& a, void* base_, const VocabWs& ws,
                          hipStream_t st) {
  char* const base = static_cast<char*>(base_);
  const VocabPieces pc = vocab_pieces(c, d);
  const long long N = (long long)c.G * c.S;
  const bool f32 = c.act_dtype == MOE_F32;
  const size_t elt = f32 ? 4 : 2;
  const int pieces = (int)(c.M * elt / 16);
  const float inv_t = a.target != nullptr ? 1.f : 1.f / d.temperature;
  const TeacherArgs t{a.idx, a.logit, a.target != nullptr ? 0 : d.K, d.V, inv_t};
  int rc = MOE_OK;
  VocabRowArgs r = row_args(c, d, a, base, ws);
  r.pos = reinterpret_cast<int32_t*>(base + ws.pos);
  r.lse_in = a.lse;
  r.loss_in = a.loss;
  r.dloss = a.dloss;
  r.inv_t = inv_t;
  r.lse2 = reinterpret_cast<float*>(base + ws.lse2);
  r.grad = reinterpret_cast<float*>(base + ws.grad);
  if (a.target != nullptr) {
    r.hit = reinterpret_cast<int32_t*>(base + ws.hit);
    r.hit_value = reinterpret_cast<float*>(base + ws.hit_value);
  }
  const bool ranges = ws.dx_plan.tiles;                        // chosen by the rows kernel
  if (ranges) {
    r.dx_entries = pc.entries < d.V ? pc.entries : d.V;
    r.dx_tiles_n = (c.M + 255) / 256;
    r.M = c.M;
    r.dx_rows = (long long)ws.dx_plan.splits * N;
    r.dx_cost = kTilesDx;
  }
  if (N <= kFewTokens) {
    rc = launch_few(c, r, t, a, base, ws, nullptr, base + ws.packed, st);
  } else {
    if (a.target == nullptr) rc = launch_teacher(c, t, a.x, a.w, base, ws, nullptr, false, st);
    if (rc == MOE_OK) rc = launch_numbered(c, r, a, base, ws, base + ws.packed, st);
  }
  if (rc != MOE_OK) return rc;
  for (int i = 0; i < pc.count; ++i) {
    const int first = i * pc.entries, n = d.V - first < pc.entries ? d.V - first : pc.entries;
    const char* const w = static_cast<const char*>(a.w) + (size_t)first * c.M * elt;
    GemmArgs z{base + ws.packed, w, base + ws.dz};
    z.kept = r.kept;
    z.ldc = pc.entries;
    z.vocab.scale = kLog2e * inv_t;
    z.vocab.lse2 = r.lse2;
    z.vocab.grad = r.grad;
    z.vocab.hit = r.hit;
    z.vocab.hit_value = r.hit_value;
    z.vocab.first = first;
    rc = f32 ? launch_gemm_f32(kDataGrad, z, 1, (int)N, n, c.M, st) : launch_vocab_logits(z, (int)N, n, c.M, st);
    if (rc != MOE_OK) return rc;
    if (a.target == nullptr) {
      auto entries = [&](auto kernel, auto* dz) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((N + 3) / 4)), dim3(256), (size_t)4 * d.K * sizeof(float2), st, t,
                           reinterpret_cast<const float2*>(base + ws.tstat), a.entry_logit, z.vocab, r.perm, r.kept, dz,
                           pc.entries, n);
      };
      if (f32) entries(vocab_entry_grad_kernel<float>, static_cast<float*>(z.C));
      else entries(vocab_entry_grad_kernel<bf16_t>, static_cast<bf16_t*>(z.C));
      if ((rc = check_launch()) != MOE_OK) return rc;
    }
    GemmArgs gx{z.C, w, base + ws.sums};
    gx.kept = r.kept;
    gx.lda = pc.entries;
    gx.k_total = n;
    gx.add = i > 0;
    const VocabDxPlan plan{(n + ws.dx_plan.k - 1) / ws.dx_plan.k, ws.dx_plan.k, ws.dx_plan.tiles};      // (a last piece fills fewer ranges)
    GemmArgs gw{z.C, base + ws.packed, static_cast<char*>(a.dw) + (size_t)first * c.M * elt};
    gw.kept = r.kept;
    gw.lda = pc.entries;
    if (ws.dw_splits > 1) { gw.C = base + ws.dw_sums; gw.k_total = ws.dw_splits; }
    bool done = false;
    if (!f32) rc = launch_vocab_grads_pair(gx, plan, gw, (int)N, n, c.M, st, &done);
    if (rc != MOE_OK) return rc;
    if (done) continue;
    rc = f32 ? launch_gemm_f32(kForward, gx, plan.splits, (int)N, c.M, plan.k, st) : launch_vocab_dx(gx, plan, (int)N, c.M, st);
    if (rc != MOE_OK) return rc;
    rc = f32 ? launch_gemm_f32(kWeightGrad, gw, ws.dw_splits, n, c.M, row_range((int)N, ws.dw_splits), st)
             : launch_vocab_dw(gw, (int)N, n, c.M, st);
    if (rc != MOE_OK) return rc;
    if (ws.dw_splits > 1) {
      uint4* const dw = reinterpret_cast<uint4*>(static_cast<char*>(a.dw) + (size_t)first * c.M * elt);
      const long long total = (long long)n * pieces;
      hipLaunchKernelGGL(f32 ? vocab_dw_kernel<float> : vocab_dw_kernel<bf16_t>, dim3(blocks_of(total)), dim3(256), 0, st,
                         reinterpret_cast<const float4*>(base + ws.dw_sums), ws.dw_splits, total, dw);
      if ((rc = check_launch()) != MOE_OK) return rc;
    }
  }
  const int parts = N * pieces < 65536 ? 8 : 1;
  auto out = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(N * pieces * parts)), dim3(256), 0, st, reinterpret_cast<const float4*>(base + ws.sums),
                       ws.dx_plan.splits, N, ranges ? r.kept : nullptr, r.pos, static_cast<uint4*>(a.dx), pieces);
  };
  if (f32) { if (parts == 1) out(vocab_dx_kernel<float, 1>); else out(vocab_dx_kernel<float, 8>); }
  else { if (parts == 1) out(vocab_dx_kernel<bf16_t, 1>); else out(vocab_dx_kernel<bf16_t, 8>); }
  return check_launch();
}

}  // namespace moe
