// Backward pass of the encoder sub-layers around the MoE layer (Section 2.1 of the paper names
// the sub-layers; the paper trains them by automatic differentiation, the derivatives below are
// the chain rule written out).  The pieces that are not GEMMs:
//
//   layer norm     n = gamma * xhat + beta, xhat = (s - mean) * rstd:
//                  ds = rstd * (g - mean(g) - xhat * mean(g * xhat)),  g = gamma * dn
//                  dgamma = sum_rows dn * xhat,  dbeta = sum_rows dn      (two kernels)
//   attention core with p = softmax(q k^T / sqrt(d)), ctx = p v and D = rowsum(dctx * ctx):
//                  dv = p^T dctx,  ds = p * (dctx v^T - D) / sqrt(d),  dq = ds k,  dk = ds^T q
//                  The probabilities are recomputed from q, k and the row statistic
//                  lse = log sum_k exp(score) that the forward kernels store.
//
// The attention core has a plain form here (one wavefront per query row for dq, one per key row
// for dk and dv, any dtype and shape whose rows fit in LDS); the MFMA form lives in
// attention_mfma.hip.
#include <math.h>
#include "common.h"

namespace moe {
namespace {

// ---------------------------------------------------------------- layer normalisation
// One wavefront per row, a wavefront walks rows wave, wave + waves, ...; its column sums of
// dn * xhat and dn stay in registers; the WAVES wavefronts of a block add theirs in LDS (fixed
// order) and the block leaves one partial row.  The sums of dn start `pitch` floats behind the others: M, or, with one
// block whose sums are dgamma and dbeta themselves, what lies between those.
template <typename T, int VPL, int WAVES = 4>
__global__ __launch_bounds__(64 * WAVES) void layer_norm_bwd_kernel(
    const uint4* __restrict__ s, const uint4* __restrict__ dn, const float* __restrict__ gamma,
    const uint4* dres, uint4* dx, float* __restrict__ partial, long long pitch, int M, int vec_per_row,
    long long rows, float eps) {
  const int lane = threadIdx.x & 63;
  const long long wave_id = (long long)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const long long waves = (long long)gridDim.x * WAVES;
  constexpr int K = Vec16<T>::kElts;
  float ag[VPL][K], ab[VPL][K], gam[VPL][K];
#pragma unroll
  for (int j = 0; j < VPL; ++j)
#pragma unroll
    for (int i = 0; i < K; i += 4) {
      const int col = (lane + 64 * j) * K + i;                 // (M is a multiple of K)
      const float4 g4 = col < M ? *reinterpret_cast<const float4*>(gamma + col) : float4{0.f, 0.f, 0.f, 0.f};
      gam[j][i] = g4.x; gam[j][i + 1] = g4.y; gam[j][i + 2] = g4.z; gam[j][i + 3] = g4.w;
#pragma unroll
      for (int k = 0; k < 4; ++k) ag[j][i + k] = ab[j][i + k] = 0.f;
    }
  const float inv_m = 1.0f / (float)M;
  for (long long row = wave_id; row < rows; row += waves) {
    float v[VPL][K], g[VPL][K];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int vi = lane + 64 * j;
#pragma unroll
      for (int i = 0; i < K; ++i) { v[j][i] = 0.f; g[j][i] = 0.f; }
      if (vi < vec_per_row) {
        Vec16<T>::unpack(s[row * vec_per_row + vi], v[j]);
        Vec16<T>::unpack(dn[row * vec_per_row + vi], g[j]);
#pragma unroll
        for (int i = 0; i < K; ++i) sum += v[j][i];
      }
    }
    const float mean = wave_sum(sum) * inv_m;
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < VPL; ++j)
      if (lane + 64 * j < vec_per_row)
#pragma unroll
        for (int i = 0; i < K; ++i) q += (v[j][i] - mean) * (v[j][i] - mean);
    const float rstd = 1.0f / sqrtf(wave_sum(q) * inv_m + eps);
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int j = 0; j < VPL; ++j)
      if (lane + 64 * j < vec_per_row)
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const float xh = (v[j][i] - mean) * rstd;
          v[j][i] = xh;
          ag[j][i] += g[j][i] * xh;                 // g still holds dn
          ab[j][i] += g[j][i];
          g[j][i] *= gam[j][i];
          sg += g[j][i];
          sgx += g[j][i] * xh;
        }
    sg = wave_sum(sg) * inv_m;
    sgx = wave_sum(sgx) * inv_m;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int vi = lane + 64 * j;
      if (vi < vec_per_row) {
        float o[K];
#pragma unroll
        for (int i = 0; i < K; ++i) o[i] = rstd * (g[j][i] - sg - v[j][i] * sgx);
        if (dres != nullptr) {
          float r[K];
          Vec16<T>::unpack(dres[row * vec_per_row + vi], r);
#pragma unroll
          for (int i = 0; i < K; ++i) o[i] += r[i];
        }
        dx[row * vec_per_row + vi] = Vec16<T>::pack(o);
      }
    }
  }
  extern __shared__ float ln_bwd_smem[];              // [wavefronts][M], used twice
  float* mine = ln_bwd_smem + (size_t)(threadIdx.x >> 6) * M;
  float* pg = partial + (size_t)blockIdx.x * 2 * M;
#pragma unroll
  for (int which = 0; which < 2; ++which) {           // 0: dgamma sums, 1: dbeta sums
#pragma unroll
    for (int j = 0; j < VPL; ++j)
#pragma unroll
      for (int i = 0; i < K; i += 4) {
        const int col = (lane + 64 * j) * K + i;
        const float* a = which == 0 ? &ag[j][i] : &ab[j][i];
        if (col < M) *reinterpret_cast<float4*>(mine + col) = float4{a[0], a[1], a[2], a[3]};
      }
    __syncthreads();
    for (int i = threadIdx.x * 4; i < M; i += 256 * WAVES) {
      float4 t = *reinterpret_cast<const float4*>(ln_bwd_smem + i);
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        const float4 o = *reinterpret_cast<const float4*>(ln_bwd_smem + w * M + i);
        t.x += o.x; t.y += o.y; t.z += o.z; t.w += o.w;
      }
      *reinterpret_cast<float4*>(pg + which * pitch + i) = t;
    }
    __syncthreads();
  }
}

// Wide rows (layer_norm_bwd_plan says from where): one block per row, which walks rows block, block + blocks, ... with the parameters' column sums in
// registers (VPT vectors of 16 bytes per thread) and fetches the next row while the sums of one meet.  4096 rows of 8192 bf16 with a
// residual's gradient, 256 blocks of 1024 threads 67 us, of 512 61 (4.4 TB/s), of 256 64, 512 blocks of 512 71 (more sums).
template <typename T, int TH, int VPT>
__global__ __launch_bounds__(TH) void layer_norm_bwd_wide_kernel(
    const uint4* __restrict__ s, const uint4* __restrict__ dn, const float* __restrict__ gamma, const uint4* dres, uint4* dx,
    float* __restrict__ partial, int M, int vec_per_row, long long rows, float eps) {
  constexpr int K = Vec16<T>::kElts, W = TH / 64;
  __shared__ float4 red[2][W];
  const int tid = threadIdx.x;
  float ag[VPT][K], ab[VPT][K], gam[VPT][K];
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < K; i += 4) {
      const int col = (tid + TH * j) * K + i;
      const float4 g4 = col < M ? *reinterpret_cast<const float4*>(gamma + col) : float4{0.f, 0.f, 0.f, 0.f};
      gam[j][i] = g4.x; gam[j][i + 1] = g4.y; gam[j][i + 2] = g4.z; gam[j][i + 3] = g4.w;
#pragma unroll
      for (int k = 0; k < 4; ++k) ag[j][i + k] = ab[j][i + k] = 0.f;
    }
  const float inv_m = 1.0f / (float)M;
  uint4 sv[VPT], dv[VPT], rv[VPT];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int vi = tid + TH * j;
      sv[j] = dv[j] = rv[j] = uint4{0u, 0u, 0u, 0u};
      if (vi < vec_per_row) {
        sv[j] = s[row * vec_per_row + vi];
        dv[j] = dn[row * vec_per_row + vi];
        if (dres != nullptr) rv[j] = dres[row * vec_per_row + vi];
      }
    }
  };
  if ((long long)blockIdx.x < rows) fetch(blockIdx.x);
  for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
    // (the row stays packed, three uses unpack it: as floats it would not fit beside the next one and the columns' sums)
    uint4 cs[VPT], cd[VPT], cr[VPT];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      cs[j] = sv[j]; cd[j] = dv[j]; cr[j] = rv[j];
      float v[K];
      Vec16<T>::unpack(cs[j], v);
#pragma unroll
      for (int i = 0; i < K; ++i) sum += v[i];
    }
    if (row + gridDim.x < rows) fetch(row + gridDim.x);
    auto keep_packed = [&]() {                                 // (the compiler would keep what it unpacked)
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        asm volatile("" : "+v"(cs[j].x), "+v"(cs[j].y), "+v"(cs[j].z), "+v"(cs[j].w), "+v"(cd[j].x), "+v"(cd[j].y), "+v"(cd[j].z), "+v"(cd[j].w));
    };
    auto meet = [&](float4 a, int which) {                     // three sums of the block
      a.x = wave_sum(a.x); a.y = wave_sum(a.y); a.z = wave_sum(a.z);
      if ((tid & 63) == 0) red[which][tid >> 6] = a;
      __syncthreads();
      float4 t = red[which][0];
#pragma unroll
      for (int w = 1; w < W; ++w) { t.x += red[which][w].x; t.y += red[which][w].y; t.z += red[which][w].z; }
      return t;
    };
    const float mean = meet(float4{sum, 0.f, 0.f, 0.f}, 0).x * inv_m;
    keep_packed();
    // sums of (v - mean)^2, g and g (v - mean): of the last two the factor rstd is left out until it is known
    float q = 0.f, sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      float v[K], g[K];
      Vec16<T>::unpack(cs[j], v);
      Vec16<T>::unpack(cd[j], g);
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const float c = tid + TH * j < vec_per_row ? v[i] - mean : 0.f, up = g[i] * gam[j][i];
        q += c * c;
        sg += up;
        sgx += up * c;
      }
    }
    const float4 t = meet(float4{q, sg, sgx, 0.f}, 1);
    const float rstd = 1.0f / sqrtf(t.x * inv_m + eps);
    keep_packed();
    const float mg = t.y * inv_m, mgx = t.z * rstd * inv_m;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int vi = tid + TH * j;
      if (vi < vec_per_row) {
        float v[K], g[K], o[K];
        Vec16<T>::unpack(cs[j], v);
        Vec16<T>::unpack(cd[j], g);
        Vec16<T>::unpack(cr[j], o);
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const float xh = (v[i] - mean) * rstd;
          ag[j][i] += g[i] * xh;
          ab[j][i] += g[i];
          o[i] += rstd * (g[i] * gam[j][i] - mg - xh * mgx);
        }
        dx[row * vec_per_row + vi] = Vec16<T>::pack(o);
      }
    }
    // (the next row's first sums go to red[0], which all have read before they met in red[1])
  }
  float* const pg = partial + (size_t)blockIdx.x * 2 * M;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int vi = tid + TH * j;
    if (vi < vec_per_row)
#pragma unroll
      for (int i = 0; i < K; i += 4) {
        *reinterpret_cast<float4*>(pg + vi * K + i) = float4{ag[j][i], ag[j][i + 1], ag[j][i + 2], ag[j][i + 3]};
        *reinterpret_cast<float4*>(pg + M + vi * K + i) = float4{ab[j][i], ab[j][i + 1], ab[j][i + 2], ab[j][i + 3]};
      }
  }
}
// Rows of any width: a block of 1024 threads per row, every pass reads the row again, and its mean and rstd are left for the
// columns' sums.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_bwd_any_kernel(
    const uint4* __restrict__ s, const uint4* __restrict__ dn, const float* __restrict__ gamma, const uint4* dres, uint4* dx,
    float2* __restrict__ stats, int M, int vec_per_row, float eps) {
  constexpr int K = Vec16<T>::kElts;
  __shared__ float red[4][16];
  const size_t base = (size_t)blockIdx.x * vec_per_row;
  const int tid = threadIdx.x;
  const float inv_m = 1.0f / (float)M;
  auto block_sum = [&](float a, int which) {
    a = wave_sum(a);
    if ((tid & 63) == 0) red[which][tid >> 6] = a;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += red[which][w];
    return t;
  };
  float f[K], g[K];
  float sum = 0.f;
  for (int vi = tid; vi < vec_per_row; vi += 1024) {
    Vec16<T>::unpack(s[base + vi], f);
#pragma unroll
    for (int i = 0; i < K; ++i) sum += f[i];
  }
  const float mean = block_sum(sum, 0) * inv_m;
  float q = 0.f, sg = 0.f, sgx = 0.f;
  for (int vi = tid; vi < vec_per_row; vi += 1024) {
    Vec16<T>::unpack(s[base + vi], f);
    Vec16<T>::unpack(dn[base + vi], g);
#pragma unroll
    for (int i = 0; i < K; ++i) {
      f[i] -= mean;
      g[i] *= gamma[vi * K + i];
      q += f[i] * f[i];
      sg += g[i];
      sgx += g[i] * f[i];
    }
  }
  const float rstd = 1.0f / sqrtf(block_sum(q, 1) * inv_m + eps);
  const float mg = block_sum(sg, 2) * inv_m, mgx = block_sum(sgx, 3) * rstd * inv_m;
  if (tid == 0) stats[blockIdx.x] = float2{mean, rstd};
  for (int vi = tid; vi < vec_per_row; vi += 1024) {
    Vec16<T>::unpack(s[base + vi], f);
    Vec16<T>::unpack(dn[base + vi], g);
    float o[K], r[K];
#pragma unroll
    for (int i = 0; i < K; ++i) r[i] = 0.f;
    if (dres != nullptr) Vec16<T>::unpack(dres[base + vi], r);
#pragma unroll
    for (int i = 0; i < K; ++i) o[i] = rstd * (g[i] * gamma[vi * K + i] - mg - (f[i] - mean) * rstd * mgx) + r[i];
    dx[base + vi] = Vec16<T>::pack(o);
  }
}
// partial sums of dn xhat and dn over rows part, part + parts, ...: a thread per 16 bytes of the columns
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_param_any_kernel(
    const uint4* __restrict__ s, const uint4* __restrict__ dn, const float2* __restrict__ stats, float* __restrict__ partial,
    int M, int vec_per_row, long long rows) {
  constexpr int K = Vec16<T>::kElts;
  const int vi = blockIdx.x * 256 + threadIdx.x;
  if (vi >= vec_per_row) return;
  float ag[K], ab[K];
#pragma unroll
  for (int i = 0; i < K; ++i) ag[i] = ab[i] = 0.f;
  for (long long row = blockIdx.y; row < rows; row += gridDim.y) {
    float f[K], g[K];
    Vec16<T>::unpack(s[row * vec_per_row + vi], f);
    Vec16<T>::unpack(dn[row * vec_per_row + vi], g);
    const float2 st = stats[row];
#pragma unroll
    for (int i = 0; i < K; ++i) { ag[i] += g[i] * ((f[i] - st.x) * st.y); ab[i] += g[i]; }
  }
  float* const pg = partial + (size_t)blockIdx.y * 2 * M + vi * K;
#pragma unroll
  for (int i = 0; i < K; ++i) { pg[i] = ag[i]; pg[M + i] = ab[i]; }
}

// dgamma[m] = sum_p partial[p][0][m], dbeta[m] = sum_p partial[p][1][m]: a block owns 16 of the
// 2 M columns, its 64 groups of 16 threads each sum every 64th partial row, LDS adds the groups
// in a fixed order (bit-reproducible).  Bound by the latency of a thread's dependent loads, so many short
// chains with the loads of eight rows in flight: 1024 partial rows, M 1024 20.6 -> 5.2 us (16 groups before).
constexpr int kReduceGroups = 64;
__global__ __launch_bounds__(16 * kReduceGroups) void layer_norm_param_reduce_kernel(
    const float* __restrict__ partial, int parts, int M, float* __restrict__ dgamma,
    float* __restrict__ dbeta) {
  __shared__ float red[kReduceGroups][17];
  const int c = threadIdx.x & 15, pl = threadIdx.x >> 4;
  const int i = blockIdx.x * 16 + c;
  float acc = 0.f;
  if (i < 2 * M) {
#pragma unroll 8
    for (int p = pl; p < parts; p += kReduceGroups) acc += partial[(size_t)p * 2 * M + i];
  }
  red[pl][c] = acc;
  __syncthreads();
  if (pl < 8) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < kReduceGroups / 8; ++k) t += red[pl * (kReduceGroups / 8) + k][c];
    red[pl * (kReduceGroups / 8)][c] = t;                      // (its own rows only)
  }
  __syncthreads();
  if (pl == 0 && i < 2 * M) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t += red[k * (kReduceGroups / 8)][c];
    if (i < M) dgamma[i] = t; else dbeta[i - M] = t;
  }
}

// ---------------------------------------------------------------- attention core, plain form
// dq: one wavefront per (sequence, head, query).  Also writes D = rowsum(dctx * ctx) of its row.
template <typename T>
__global__ __launch_bounds__(256) void attention_bwd_dq_rows_kernel(
    const T* __restrict__ qkv, const T* __restrict__ ctx, const T* __restrict__ dctx,
    const float* __restrict__ lse, T* __restrict__ dqkv, float* __restrict__ dvec, int L, int heads,
    int d, long long queries) {
  extern __shared__ float att_bwd_smem[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* sc = att_bwd_smem + (size_t)wave * (L + 2 * d);   // [L] ds of the row, [d] q, [d] dctx
  float* qs = sc + L;
  float* dos = qs + d;
  const long long id = (long long)blockIdx.x * 4 + wave;   // (b * heads + h) * L + l
  if (id >= queries) return;
  const int l = (int)(id % L);
  const long long bh = id / L;
  const int h = (int)(bh % heads);
  const long long b = bh / heads;
  const int A = heads * d;
  const size_t ld = (size_t)3 * A;
  const T* qrow = qkv + ((size_t)b * L + l) * ld + (size_t)h * d;
  const T* kbase = qkv + (size_t)b * L * ld + A + (size_t)h * d;
  const T* vbase = kbase + A;
  const size_t crow = ((size_t)b * L + l) * A + (size_t)h * d;
  float dd = 0.f;
  for (int i = lane; i < d; i += 64) {
    qs[i] = Elt<T>::load(qrow + i);
    const float g = Elt<T>::load(dctx + crow + i);
    dos[i] = g;
    dd += g * Elt<T>::load(ctx + crow + i);
  }
  dd = wave_sum(dd);
  if (lane == 0) dvec[id] = dd;
  __builtin_amdgcn_wave_barrier();
  const float scale = 1.0f / sqrtf((float)d);
  const float ls = lse[id];
  for (int k0 = 0; k0 < L; k0 += 64) {
    const int key = k0 + lane;
    if (key < L) {
      const T* kr = kbase + (size_t)key * ld;
      const T* vr = vbase + (size_t)key * ld;
      float dot = 0.f, dp = 0.f;
      for (int i = 0; i < d; ++i) {
        dot = fmaf(qs[i], Elt<T>::load(kr + i), dot);
        dp = fmaf(dos[i], Elt<T>::load(vr + i), dp);
      }
      const float p = expf(dot * scale - ls);
      sc[key] = p * (dp - dd) * scale;
    }
  }
  __builtin_amdgcn_wave_barrier();
  T* out = dqkv + ((size_t)b * L + l) * ld + (size_t)h * d;
  for (int i = lane; i < d; i += 64) {
    float acc = 0.f;
    for (int key = 0; key < L; ++key) acc = fmaf(sc[key], Elt<T>::load(kbase + (size_t)key * ld + i), acc);
    Elt<T>::store(out + i, acc);
  }
}

// dk, dv: one wavefront per (sequence, head, key); needs lse and D of every query of the head.
template <typename T>
__global__ __launch_bounds__(256) void attention_bwd_dkv_rows_kernel(
    const T* __restrict__ qkv, const T* __restrict__ dctx, const float* __restrict__ lse,
    const float* __restrict__ dvec, T* __restrict__ dqkv, int L, int heads, int d, long long keys) {
  extern __shared__ float att_bwd_smem[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* pp = att_bwd_smem + (size_t)wave * (2 * L + 2 * d);   // [L] p, [L] ds, [d] k, [d] v
  float* sd = pp + L;
  float* ks = sd + L;
  float* vs = ks + d;
  const long long id = (long long)blockIdx.x * 4 + wave;       // (b * heads + h) * L + key
  if (id >= keys) return;
  const int key = (int)(id % L);
  const long long bh = id / L;
  const int h = (int)(bh % heads);
  const long long b = bh / heads;
  const int A = heads * d;
  const size_t ld = (size_t)3 * A;
  const T* qbase = qkv + (size_t)b * L * ld + (size_t)h * d;
  const T* krow = qbase + (size_t)key * ld + A;
  const T* gbase = dctx + (size_t)b * L * A + (size_t)h * d;
  for (int i = lane; i < d; i += 64) {
    ks[i] = Elt<T>::load(krow + i);
    vs[i] = Elt<T>::load(krow + A + i);
  }
  __builtin_amdgcn_wave_barrier();
  const float scale = 1.0f / sqrtf((float)d);
  for (int q0 = 0; q0 < L; q0 += 64) {
    const int q = q0 + lane;
    if (q < L) {
      const T* qr = qbase + (size_t)q * ld;
      const T* gr = gbase + (size_t)q * A;
      float dot = 0.f, dp = 0.f;
      for (int i = 0; i < d; ++i) {
        dot = fmaf(Elt<T>::load(qr + i), ks[i], dot);
        dp = fmaf(Elt<T>::load(gr + i), vs[i], dp);
      }
      const float p = expf(dot * scale - lse[bh * L + q]);
      pp[q] = p;
      sd[q] = p * (dp - dvec[bh * L + q]) * scale;
    }
  }
  __builtin_amdgcn_wave_barrier();
  T* out = dqkv + ((size_t)b * L + key) * ld + A + (size_t)h * d;
  for (int i = lane; i < d; i += 64) {
    float dk = 0.f, dv = 0.f;
    for (int q = 0; q < L; ++q) {
      dk = fmaf(sd[q], Elt<T>::load(qbase + (size_t)q * ld + i), dk);
      dv = fmaf(pp[q], Elt<T>::load(gbase + (size_t)q * A + i), dv);
    }
    Elt<T>::store(out + i, dk);
    Elt<T>::store(out + A + i, dv);
  }
}

// out[i] = sum_s partial[s][i] (fixed order), rounded once to bf16; 8 elements per thread
__global__ __launch_bounds__(256) void splitk_reduce_kernel(const float* __restrict__ partial,
                                                            int splits, long long elems,
                                                            uint4* __restrict__ out) {
  const long long v = (long long)blockIdx.x * 256 + threadIdx.x;
  if (v * 8 >= elems) return;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int sp = 0; sp < splits; ++sp) {
    const float4* p = reinterpret_cast<const float4*>(partial + (size_t)sp * elems + v * 8);
    const float4 a = p[0], b = p[1];
    acc[0] += a.x; acc[1] += a.y; acc[2] += a.z; acc[3] += a.w;
    acc[4] += b.x; acc[5] += b.y; acc[6] += b.z; acc[7] += b.w;
  }
  out[v] = Vec16<bf16_t>::pack(acc);
}

}  // namespace

int launch_add_ranges(const float* partial, int ranges, long long elems, void* out, hipStream_t st) {
  hipLaunchKernelGGL(splitk_reduce_kernel, dim3((unsigned)((elems / 8 + 255) / 256)), dim3(256), 0, st, partial, ranges, elems,
                     static_cast<uint4*>(out));
  return check_launch();
}

// Weight gradient of a dense layer, dW [in,out] = X^T dY over `rows` tokens.  Its output has few tiles but a very
// long K (the tokens), so one product alone would leave most compute units idle: the tokens are cut into ranges
// (dense_wgrad_plan) that run as a batch with fp32 results, and one pass adds the ranges in order and rounds once.
size_t dense_wgrad_partial_bytes(int act_dtype, long long rows, int in, int out) {
  if (act_dtype != MOE_BF16 || rows > 0x7fffffffLL) return 0;
  const int sp = dense_wgrad_plan(rows, in, out).splits;
  return sp > 1 ? (size_t)sp * in * out * sizeof(float) : 0;
}

int launch_dense_grads(const moe_config& c, long long rows, int in, int out, const void* X, const void* dY, const void* W,
                       const void* mask, void* dX, void* dW, float* partial, hipStream_t st) {
  if (rows > 0x7fffffffLL) return MOE_EUNSUPPORTED;
  DenseWgradPlan plan{1, (int)rows};
  if (c.act_dtype == MOE_BF16 && partial != nullptr) plan = dense_wgrad_plan(rows, in, out);
  bool done = false;
  int rc = MOE_OK;
  if (c.act_dtype == MOE_BF16)
    rc = launch_dense_grads_pair(plan, rows, in, out, X, dY, W, mask, dX, dW, partial, st, &done);
  if (rc != MOE_OK) return rc;
  if (!done) {
    moe_config g = c;
    g.E = 1; g.G = 1; g.C = (int)rows; g.M = in; g.H = out;
    rc = plan.splits > 1 ? launch_dense_wgrad_ranges(plan, rows, in, out, X, dY, partial, st)
                         : launch_expert_wgrad1(g, X, dY, dW, nullptr, st);
  }
  if (rc != MOE_OK) return rc;
  if (plan.splits > 1) {
    if ((rc = launch_add_ranges(partial, plan.splits, (long long)in * out, dW, st)) != MOE_OK) return rc;
  }
  if (done) return MOE_OK;
  // (the second product of a feed-forward layer is its transpose in the expert's naming)
  moe_config g = c;
  g.E = 1; g.G = 1; g.S = g.C = (int)rows;
  g.M = mask != nullptr ? out : in;
  g.H = mask != nullptr ? in : out;
  return mask != nullptr ? launch_expert_dgrad2(g, dY, W, mask, nullptr, dX, nullptr, st)
                         : launch_expert_dgrad1(g, dY, W, dX, nullptr, st);
}

// How the rows are walked: by wavefronts up to 3 KB bf16, 5 KB fp32 (with fewer than 1024 rows 8 KB and 4096 columns), by blocks up
// to 32 KB, wider ones in any number of passes, which keep every row's mean and rstd.  A wavefront's column sums take three
// registers for every 64 columns of its row and leave too few others on the unit: us by wavefronts / by blocks, bf16 with a residual's
// gradient 6421 x 1600 33 / 25, 16000 x 2048 70 / 52, 8192 x 2400 68 / 49, 16000 x 4096 268 / 112 (105 is one pass over all), without
// 16000 x 1400 40 / 41; fp32 without 6421 x 1196 29 / 36, with 8192 x 1500 48 / 44, 3000 x 2048 32 / 24.  As many blocks as units hold:
// four, two or one per unit with one, one or more vectors a thread (the sums that a block leaves are as long as four rows; 8192 x 2400
// 256 blocks 67, 512 49, 768 53).
enum LayerNormBwdForm { kLnWavefronts, kLnBlocks, kLnAny };
static LayerNormBwdForm layer_norm_bwd_plan(int act_dtype, long long rows, int M, bool by_wavefronts, int* parts) {
  const int vec = M * (act_dtype == MOE_F32 ? 4 : 2) / 16;
  const int waves = by_wavefronts || rows < 1024 ? 512 : act_dtype == MOE_F32 ? 320 : 192;
  const LayerNormBwdForm form = vec <= waves && M <= 4096 ? kLnWavefronts : vec <= 2048 ? kLnBlocks : kLnAny;
  const long long most = form == kLnWavefronts || (form == kLnBlocks && vec <= 256) ? 1024
                         : form == kLnBlocks ? (vec <= 512 ? 512 : 256) : 64, blocks = (rows + 3) / 4;
  *parts = (int)(blocks < most ? blocks : most);
  return form;
}
size_t layer_norm_bwd_bytes(int act_dtype, long long rows, int M, bool by_wavefronts) {
  int parts;
  const LayerNormBwdForm form = layer_norm_bwd_plan(act_dtype, rows, M, by_wavefronts, &parts);
  return (size_t)parts * 2 * M * sizeof(float) + (form == kLnAny ? (size_t)rows * sizeof(float2) : 0);
}

int launch_layer_norm_bwd(int act_dtype, const void* s, const void* dn, const float* gamma,
                          const void* dres, void* dx, float* partial, float* dgamma, float* dbeta,
                          long long rows, int M, bool by_wavefronts, hipStream_t st) {
  const int elt = act_dtype == MOE_F32 ? 4 : 2;
  const int vec_per_row = M * elt / 16;
  const int vpl = (vec_per_row + 63) / 64;
  if (!by_wavefronts && rows <= 64 && M <= 1024) {
    // One block of 16 wavefronts, whose sums are the parameters' gradients: one launch (37 rows of 520 fp32, with the call from Python
    // 17.6 -> 12.5 us).
    auto one = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(1), dim3(1024), (size_t)16 * M * sizeof(float), st, static_cast<const uint4*>(s),
                         static_cast<const uint4*>(dn), gamma, static_cast<const uint4*>(dres), static_cast<uint4*>(dx), dgamma,
                         ((intptr_t)dbeta - (intptr_t)dgamma) / (long long)sizeof(float), M, vec_per_row, rows, 1e-6f);
    };
    if (act_dtype == MOE_F32) {
      if (vpl <= 1) one(layer_norm_bwd_kernel<float, 1, 16>);
      else if (vpl <= 2) one(layer_norm_bwd_kernel<float, 2, 16>);
      else one(layer_norm_bwd_kernel<float, 4, 16>);
    } else {
      if (vpl <= 1) one(layer_norm_bwd_kernel<bf16_t, 1, 16>); else one(layer_norm_bwd_kernel<bf16_t, 2, 16>);
    }
    return check_launch();
  }
  const size_t lds = (size_t)4 * M * sizeof(float);
  const float eps = 1e-6f;
  int parts;
  const LayerNormBwdForm form = layer_norm_bwd_plan(act_dtype, rows, M, by_wavefronts, &parts);
  auto reduce = [&]() {
    hipLaunchKernelGGL(layer_norm_param_reduce_kernel, dim3((unsigned)((2 * M + 15) / 16)), dim3(16 * kReduceGroups), 0, st,
                       partial, parts, M, dgamma, dbeta);
    return check_launch();
  };
  if (form != kLnWavefronts) {
    if (form == kLnAny && rows >= 1 << 22) return MOE_EUNSUPPORTED;      // (a launch has less than 2^32 threads)
    auto wide = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)parts), dim3(threads), 0, st, static_cast<const uint4*>(s),
                         static_cast<const uint4*>(dn), gamma, static_cast<const uint4*>(dres), static_cast<uint4*>(dx), partial,
                         M, vec_per_row, rows, eps);
    };
    auto any = [&](auto rows_kernel, auto columns_kernel) {
      float2* const stats = reinterpret_cast<float2*>(partial + (size_t)parts * 2 * M);
      hipLaunchKernelGGL(rows_kernel, dim3((unsigned)rows), dim3(1024), 0, st, static_cast<const uint4*>(s),
                         static_cast<const uint4*>(dn), gamma, static_cast<const uint4*>(dres), static_cast<uint4*>(dx), stats, M,
                         vec_per_row, eps);
      hipLaunchKernelGGL(columns_kernel, dim3((unsigned)((vec_per_row + 255) / 256), (unsigned)parts), dim3(256), 0, st,
                         static_cast<const uint4*>(s), static_cast<const uint4*>(dn), stats, partial, M, vec_per_row, rows);
    };
#define MOE_LNB_WIDE(T)                                                                       \
  if (form == kLnBlocks && vec_per_row <= 256) wide(layer_norm_bwd_wide_kernel<T, 256, 1>, 256);  \
  else if (form == kLnBlocks && vec_per_row <= 512) wide(layer_norm_bwd_wide_kernel<T, 512, 1>, 512); \
  else if (form == kLnBlocks && vec_per_row <= 1024) wide(layer_norm_bwd_wide_kernel<T, 512, 2>, 512); \
  else if (form == kLnBlocks && vec_per_row <= 1536) wide(layer_norm_bwd_wide_kernel<T, 512, 3>, 512); \
  else if (form == kLnBlocks) wide(layer_norm_bwd_wide_kernel<T, 512, 4>, 512);               \
  else any(layer_norm_bwd_any_kernel<T>, layer_norm_param_any_kernel<T>);
    if (act_dtype == MOE_F32) { MOE_LNB_WIDE(float) } else { MOE_LNB_WIDE(bf16_t) }
#undef MOE_LNB_WIDE
    const int rc = check_launch();
    return rc != MOE_OK ? rc : reduce();
  }
  const unsigned grid = (unsigned)parts;
#define MOE_LNB_CASE(T, V)                                                                    \
  hipLaunchKernelGGL((layer_norm_bwd_kernel<T, V>), dim3(grid), dim3(256), lds, st,           \
                     static_cast<const uint4*>(s), static_cast<const uint4*>(dn), gamma,      \
                     static_cast<const uint4*>(dres), static_cast<uint4*>(dx), partial, M, M, \
                     vec_per_row, rows, eps)
#define MOE_LNB_VPL(T)                                                                        \
  if (vpl <= 1) MOE_LNB_CASE(T, 1); else if (vpl <= 2) MOE_LNB_CASE(T, 2);                    \
  else if (vpl <= 4) MOE_LNB_CASE(T, 4);                                                      \
  else if (vpl <= 5) MOE_LNB_CASE(T, 5); else if (vpl <= 6) MOE_LNB_CASE(T, 6); else MOE_LNB_CASE(T, 8)
  if (act_dtype == MOE_F32) { MOE_LNB_VPL(float); } else { MOE_LNB_VPL(bf16_t); }
#undef MOE_LNB_VPL
#undef MOE_LNB_CASE
  const int rc = check_launch();
  return rc != MOE_OK ? rc : reduce();
}

// dqkv [B*L, 3*heads*d] from qkv, ctx, dctx [B*L, heads*d], lse [B*heads*L]; dvec [B*heads*L] scratch
int launch_attention_core_bwd(int act_dtype, const void* qkv, const void* ctx, const void* dctx,
                              const float* lse, void* dqkv, float* dvec, long long B, int L,
                              int heads, int d, hipStream_t st) {
  if (attention_mfma_ok(act_dtype, L, heads, d))
    return launch_attention_bwd_mfma(qkv, ctx, dctx, lse, dqkv, dvec, B, L, heads, d, st);
  const long long rows = B * heads * L;
  const size_t lds = (size_t)4 * (2 * L + 2 * d) * sizeof(float);
  if (lds > 64 * 1024 || (rows + 3) / 4 > 0x7fffffffLL) return MOE_EUNSUPPORTED;
  if (attention_f32_ok(act_dtype, d, B * heads * L))
    return launch_attention_f32_bwd(qkv, ctx, dctx, lse, dqkv, dvec, B, L, heads, d, st);
  const size_t lds_q = (size_t)4 * (L + 2 * d) * sizeof(float);
  const unsigned grid = (unsigned)((rows + 3) / 4);
  if (act_dtype == MOE_F32) {
    hipLaunchKernelGGL(attention_bwd_dq_rows_kernel<float>, dim3(grid), dim3(256), lds_q, st,
                       static_cast<const float*>(qkv), static_cast<const float*>(ctx),
                       static_cast<const float*>(dctx), lse, static_cast<float*>(dqkv), dvec, L,
                       heads, d, rows);
    hipLaunchKernelGGL(attention_bwd_dkv_rows_kernel<float>, dim3(grid), dim3(256), lds, st,
                       static_cast<const float*>(qkv), static_cast<const float*>(dctx), lse, dvec,
                       static_cast<float*>(dqkv), L, heads, d, rows);
  } else {
    hipLaunchKernelGGL(attention_bwd_dq_rows_kernel<bf16_t>, dim3(grid), dim3(256), lds_q, st,
                       static_cast<const bf16_t*>(qkv), static_cast<const bf16_t*>(ctx),
                       static_cast<const bf16_t*>(dctx), lse, static_cast<bf16_t*>(dqkv), dvec, L,
                       heads, d, rows);
    hipLaunchKernelGGL(attention_bwd_dkv_rows_kernel<bf16_t>, dim3(grid), dim3(256), lds, st,
                       static_cast<const bf16_t*>(qkv), static_cast<const bf16_t*>(dctx), lse, dvec,
                       static_cast<bf16_t*>(dqkv), L, heads, d, rows);
  }
  return check_launch();
}

}  // namespace moe
