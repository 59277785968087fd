// Losses on the token losses of a vocabulary (nll = -log p of each token's target) and their gradients at them.
//
//   preference   ratio_i = sum_t ref_t - nll_t over a sequence's tokens with a target, h = ratio_2p - ratio_2p+1,
//                loss = -(1 - e) log sigmoid(b h) - e log sigmoid(-b h)   or   (h - 1/(2b))^2;  d loss / d nll_t = -+ d loss / d h
//   policy       r = exp(old - nll), x = nll - ref:  loss = -min(r a, clip(r) a) + b (e^x - 1 - x),
//                d loss / d nll = r a (unless the bound holds r) + b (e^x - 1)
//
// All are bound by memory where tokens are many and by one launch where they are few.  A pair's sums are formed in 64 bits (a
// sequence's log-ratio is what remains of thousands of token losses that nearly cancel), by one block in a fixed order; the backward pass has the
// ratios as they are stored, in fp32, and takes their margin from these.
// us of a kernel: 64 pairs, 262144 tokens 4.8 forward, 4.5 backward; a policy's 1048576 tokens 5.8 (25 MB: 4.3 TB/s), 32768 backward 3.7.
#include <math.h>
#include "common.h"

namespace moe {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ long long clamped(long long v, long long lo, long long hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// -log sigmoid(x)
__device__ __forceinline__ double softplus_neg(double x) { return fmax(-x, 0.0) + log1p(exp(-fabs(x))); }

// One block per pair: its wavefronts walk the tokens of both sequences, four tokens a lane ahead of their use.
__global__ __launch_bounds__(1024) void preference_kernel(moe_preference_dims d, long long N, const float* __restrict__ nll,
                                                          const float* __restrict__ ref, const int32_t* __restrict__ target,
                                                          const int32_t* __restrict__ start, float* __restrict__ loss,
                                                          float* __restrict__ ratio) {
  __shared__ double sums[2][16];
  const int p = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  double total[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const long long from = clamped(start[2 * p + s], 0, N), to = clamped(start[2 * p + s + 1], from, N);
    double sum = 0.0;
    for (long long t0 = from + threadIdx.x; t0 < to; t0 += 4 * blockDim.x) {
      float a[4], b[4];
      int y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long t = t0 + i * blockDim.x, at = t < to ? t : to - 1;
        a[i] = nll[at];
        b[i] = ref[at];
        y[i] = t < to ? target[at] : -1;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += (unsigned)y[i] < (unsigned)d.V ? (double)b[i] - (double)a[i] : 0.0;
    }
    sum = wave_sum_f64(sum);
    if (lane == 0) sums[s][wave] = sum;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    total[s] = 0.0;
    for (int w = 0; w < waves; ++w) total[s] += sums[s][w];
    ratio[2 * p + s] = (float)total[s];
  }
  const double h = total[0] - total[1];
  double l;
  if (d.kind == MOE_PREFERENCE_LOGISTIC) {
    l = (1.0 - d.smoothing) * softplus_neg(d.beta * h);
    if (d.smoothing > 0.0) l += d.smoothing * softplus_neg(-d.beta * h);
  } else {
    l = h - 0.5 / d.beta;
    l *= l;
  }
  loss[p] = (float)l;
}

// The last i in lo .. hi with start[i] <= t, or lo if none has.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ start, int lo, int hi, long long t) {
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (start[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Four tokens a thread.  A wavefront looks for the sequences of its first and last token, 64 candidates at a time; its
// threads look between these, where there is mostly one.
__global__ __launch_bounds__(256) void preference_bwd_kernel(moe_preference_dims d, long long N, const int32_t* __restrict__ target,
                                                             const int32_t* __restrict__ start, const float* __restrict__ ratio,
                                                             const float* __restrict__ dloss, float* __restrict__ dnll) {
  const int lane = threadIdx.x & 63, edges = 2 * d.P + 1;
  const long long wave0 = ((long long)blockIdx.x * 256 + (threadIdx.x & ~63)) * 4, t0 = wave0 + 4 * lane;
  if (wave0 >= N) return;                                      // wavefront-uniform
  i32x4_t y = {-1, -1, -1, -1};
  const bool whole = t0 + 4 <= N;
  if (whole) y = *reinterpret_cast<const i32x4_t*>(target + t0);
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t0 + i < N) y[i] = target[t0 + i];
  }
  // the number of edges at or before a token, found by steps of 64, 64^2, ..: all edges before `lo` are
  auto edges_to = [&](long long t) {
    int lo = 0, step = 1;
    while ((long long)step * 64 < edges) step *= 64;
    for (; step > 0; step /= 64) {
      const long long e = lo + (long long)(lane + 1) * step - 1;
      const bool before = e < edges && start[e] <= t;
      lo += step * __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
      if (lo > edges) lo = edges;
    }
    return lo;
  };
  const int first = edges_to(wave0), last = edges_to(wave0 + 255 < N ? wave0 + 255 : N - 1);
  f32x4_t g = {0.f, 0.f, 0.f, 0.f};
  int seen = -1;
  float slope = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((unsigned)y[i] >= (unsigned)d.V) continue;
    const long long t = t0 + i;
    const int from = first > 0 ? first - 1 : 0, to = last > from ? last - 1 : from;
    const int s = sequence_of(start, from, to < from ? from : to, t);
    if (start[s] > t || s >= 2 * d.P) continue;                // before the first sequence, or past the last
    if (s != seen) {
      seen = s;
      const int p = s / 2;
      const double h = (double)ratio[2 * p] - (double)ratio[2 * p + 1];
      double dh;
      if (d.kind == MOE_PREFERENCE_LOGISTIC) {
        // -(1 - e) sigmoid(-x) + e sigmoid(x): each sigmoid from the side on which nothing cancels
        const double x = d.beta * h, z = exp(-fabs(x)), small = z / (1.0 + z), large = 1.0 / (1.0 + z);
        dh = d.beta * (d.smoothing * (x >= 0 ? large : small) - (1.0 - d.smoothing) * (x >= 0 ? small : large));
      } else {
        dh = 2.0 * (h - 0.5 / d.beta);
      }
      dh *= (double)dloss[p];
      slope = (float)((s & 1) != 0 ? dh : -dh);
    }
    g[i] = slope;
  }
  if (whole) *reinterpret_cast<f32x4_t*>(dnll + t0) = g;
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t0 + i < N) dnll[t0 + i] = g[i];
  }
}

// e^x - 1 - x.  Below 1 the terms of its series from x^2/2 on: the difference would lose 2 / x of its digits.
__device__ __forceinline__ float exp_rest(float x) {
  if (fabsf(x) >= 1.f) {
    const float e = expf(x);
    return e == INFINITY ? e : e - 1.f - x;                    // (of x = inf too)
  }
  float s = 1.f / 39916800.f;                                  // those left out, from x^12 / 12! on, are below 6e-9 of the sum (at -1)
  s = fmaf(s, x, 1.f / 3628800.f);
  s = fmaf(s, x, 1.f / 362880.f);
  s = fmaf(s, x, 1.f / 40320.f);
  s = fmaf(s, x, 1.f / 5040.f);
  s = fmaf(s, x, 1.f / 720.f);
  s = fmaf(s, x, 1.f / 120.f);
  s = fmaf(s, x, 1.f / 24.f);
  s = fmaf(s, x, 1.f / 6.f);
  s = fmaf(s, x, 0.5f);
  return x * x * s;
}

struct PolicyBounds { double log_low, log_high; float low, high, beta; };

// Four tokens a thread, every array read and written once in 16-byte pieces.
template <bool BACKWARD>
__global__ __launch_bounds__(256) void policy_kernel(PolicyCall a, PolicyBounds d, int V, bool adv_per_token, long long N, int S) {
  const long long t0 = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (t0 >= N) return;
  const int n = N - t0 < 4 ? (int)(N - t0) : 4;
  f32x4_t nll = {}, old = {}, ref = {}, adv = {}, up = {}, out, kl;
  i32x4_t y = {-1, -1, -1, -1};
  auto load = [&](auto& v, const auto* from) __attribute__((always_inline)) {
    using V4 = std::remove_reference_t<decltype(v)>;
    if (n == 4) v = *reinterpret_cast<const V4*>(from + t0);
    else
      for (int i = 0; i < n; ++i) v[i] = from[t0 + i];
  };
  load(y, a.target);
  load(nll, a.nll);
  load(old, a.old_nll);
  if (a.ref != nullptr) load(ref, a.ref);
  if (BACKWARD) load(up, a.dloss);
  if (adv_per_token) load(adv, a.adv);
  else {
    long long g = t0 / S;
    int s = (int)(t0 - g * S);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < n) adv[i] = a.adv[g];
      if (++s == S) { s = 0; ++g; }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool has = (unsigned)y[i] < (unsigned)V;
    // the difference of two fp32 numbers is exact in 64 bits, and so is its side of a bound's logarithm, but for its last digits
    const double lr = (double)old[i] - (double)nll[i];
    const float A = adv[i], r = expf((float)lr);
    const bool high = A > 0.f && lr > d.log_high, low = A < 0.f && lr < d.log_low;
    const float x = nll[i] - ref[i];
    if constexpr (BACKWARD) {
      float g = high || low || A == 0.f ? 0.f : r * A;
      if (d.beta != 0.f) g = fmaf(d.beta, expm1f(x), g);
      out[i] = has ? g * up[i] : 0.f;
    } else {
      float l = A == 0.f ? 0.f : -A * (high ? d.high : low ? d.low : r);
      kl[i] = 0.f;
      if (a.ref != nullptr) {
        const float k = exp_rest(x);
        if (d.beta != 0.f) l = fmaf(d.beta, k, l);
        kl[i] = has ? k : 0.f;
      }
      out[i] = has ? l : 0.f;
    }
  }
  auto store = [&](float* to, const f32x4_t& v) __attribute__((always_inline)) {
    if (n == 4) *reinterpret_cast<f32x4_t*>(to + t0) = v;
    else
      for (int i = 0; i < n; ++i) to[t0 + i] = v[i];
  };
  store(BACKWARD ? a.dnll : a.loss, out);
  if (!BACKWARD && a.kl != nullptr) store(a.kl, kl);
}

}  // namespace

int launch_preference(const moe_preference_dims& d, long long N, const float* nll, const float* ref, const int32_t* target,
                      const int32_t* start, float* loss, float* ratio, hipStream_t st) {
  const int threads = N / d.P >= 4096 ? 1024 : 256;
  hipLaunchKernelGGL(preference_kernel, dim3(d.P), dim3(threads), 0, st, d, N, nll, ref, target, start, loss, ratio);
  return check_launch();
}

int launch_preference_bwd(const moe_preference_dims& d, long long N, const int32_t* target, const int32_t* start, const float* ratio,
                          const float* dloss, float* dnll, hipStream_t st) {
  hipLaunchKernelGGL(preference_bwd_kernel, dim3((unsigned)((N + 1023) / 1024)), dim3(256), 0, st, d, N, target, start, ratio, dloss, dnll);
  return check_launch();
}

int launch_policy(const moe_policy_dims& d, long long N, int S, const PolicyCall& a, hipStream_t st) {
  PolicyBounds b;
  b.log_low = d.clip_low < 1.0 ? log1p(-d.clip_low) : -INFINITY;
  b.log_high = log1p(d.clip_high);
  b.low = (float)(1.0 - d.clip_low);
  b.high = (float)(1.0 + d.clip_high);
  b.beta = (float)d.beta;
  const dim3 grid((unsigned)((N + 1023) / 1024)), threads(256);
  if (a.dnll != nullptr) hipLaunchKernelGGL((policy_kernel<true>), grid, threads, 0, st, a, b, d.V, d.adv_per_token != 0, N, S);
  else hipLaunchKernelGGL((policy_kernel<false>), grid, threads, 0, st, a, b, d.V, d.adv_per_token != 0, N, S);
  return check_launch();
}

}  // namespace moe
