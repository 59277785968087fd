// Attention of a decoder's tokens to an encoder's states, forward and backward.
#include <float.h>
#include <math.h>
#include "cross_attention.h"

namespace moe {
namespace {

// One wavefront per column (a query, or backward a state), lanes over d: for every case, and nothing else.
template <typename T, int D>
struct Lanes {
  static constexpr int PER = D / 64;
  float v[PER];
  __device__ void load(const T* p, int lane) {
    for (int i = 0; i < PER; ++i) v[i] = Elt<T>::load(p + lane * PER + i);
  }
  __device__ void store(T* p, int lane, float f) const {
    for (int i = 0; i < PER; ++i) Elt<T>::store(p + lane * PER + i, v[i] * f);
  }
  __device__ float dot(const Lanes& o) const {
    float s = 0.f;
    for (int i = 0; i < PER; ++i) s = fmaf(v[i], o.v[i], s);
    return wave_sum(s);
  }
  __device__ void add(const Lanes& o, float f) {
    for (int i = 0; i < PER; ++i) v[i] = fmaf(o.v[i], f, v[i]);
  }
  __device__ void clear() {
    for (int i = 0; i < PER; ++i) v[i] = 0.f;
  }
};
__device__ __forceinline__ int held(const int32_t* src_len, long long b, int Lk) {
  if (src_len == nullptr) return Lk;
  const int n = src_len[b];
  return n < 0 ? 0 : n > Lk ? Lk : n;
}
struct Geo { int Lq, Lk, heads, kv_heads, share; };

template <typename T, int D>
__global__ void cross_plain_kernel(Geo g, const T* q, const T* kv, const int32_t* src_len, T* ctx, float* lse) {
  const int lane = threadIdx.x, cols = g.Lq * g.share;
  const long long item = blockIdx.x, bk = item / cols, b = bk / g.kv_heads;
  const int c = (int)(item % cols), k = (int)(bk % g.kv_heads), h = k * g.share + c % g.share, A = g.heads * D, Akv = g.kv_heads * D;
  const size_t row = ((size_t)b * g.Lq + c / g.share) * A + (size_t)h * D;
  const int n = held(src_len, b, g.Lk);
  Lanes<T, D> qv, o, x;
  qv.load(q + row, lane);
  o.clear();
  float m = -FLT_MAX, l = 0.f;
  const float scale = 1.f / sqrtf((float)D);
  for (int j = 0; j < n; ++j) {
    const T* kr = kv + ((size_t)b * g.Lk + j) * 2 * Akv + (size_t)k * D;
    x.load(kr, lane);
    const float s = qv.dot(x) * scale, mn = fmaxf(m, s), f = expf(m - mn), p = expf(s - mn);
    x.load(kr + Akv, lane);
    for (int i = 0; i < Lanes<T, D>::PER; ++i) o.v[i] = o.v[i] * f + p * x.v[i];
    l = l * f + p;
    m = mn;
  }
  o.store(ctx + row, lane, n > 0 ? 1.f / l : 0.f);
  if (lse != nullptr && lane == 0) lse[item] = n > 0 ? m + logf(l) : 0.f;
}
template <typename T, int D>
__global__ void cross_plain_dq_kernel(Geo g, const T* q, const T* kv, const int32_t* src_len, const T* ctx, const T* dctx, const float* lse, T* dq,
                                      float* dvec) {
  const int lane = threadIdx.x, cols = g.Lq * g.share;
  const long long item = blockIdx.x, bk = item / cols, b = bk / g.kv_heads;
  const int c = (int)(item % cols), k = (int)(bk % g.kv_heads), h = k * g.share + c % g.share, A = g.heads * D, Akv = g.kv_heads * D;
  const size_t row = ((size_t)b * g.Lq + c / g.share) * A + (size_t)h * D;
  const int n = held(src_len, b, g.Lk);
  Lanes<T, D> qv, gv, o, x, y;
  qv.load(q + row, lane);
  gv.load(dctx + row, lane);
  x.load(ctx + row, lane);
  const float dd = gv.dot(x), scale = 1.f / sqrtf((float)D);
  if (lane == 0) dvec[item] = dd;
  o.clear();
  for (int j = 0; j < n; ++j) {
    const T* kr = kv + ((size_t)b * g.Lk + j) * 2 * Akv + (size_t)k * D;
    x.load(kr, lane);
    y.load(kr + Akv, lane);
    o.add(x, expf(qv.dot(x) * scale - lse[item]) * (gv.dot(y) - dd) * scale);
  }
  o.store(dq + row, lane, 1.f);
}
template <typename T, int D>
__global__ void cross_plain_dkv_kernel(Geo g, const T* q, const T* kv, const int32_t* src_len, const T* dctx, const float* lse, const float* dvec, T* dkv) {
  const int lane = threadIdx.x, cols = g.Lq * g.share;
  const long long item = blockIdx.x, bk = item / g.Lk, b = bk / g.kv_heads;
  const int j = (int)(item % g.Lk), k = (int)(bk % g.kv_heads), A = g.heads * D, Akv = g.kv_heads * D;
  const size_t row = ((size_t)b * g.Lk + j) * 2 * Akv + (size_t)k * D;
  Lanes<T, D> kk, vv, dk, dv, x, y;
  dk.clear();
  dv.clear();
  if (j < held(src_len, b, g.Lk)) {
    kk.load(kv + row, lane);
    vv.load(kv + row + Akv, lane);
    const float scale = 1.f / sqrtf((float)D);
    for (int c = 0; c < cols; ++c) {
      const size_t at = ((size_t)b * g.Lq + c / g.share) * A + (size_t)(k * g.share + c % g.share) * D;
      x.load(q + at, lane);
      y.load(dctx + at, lane);
      const float p = expf(kk.dot(x) * scale - lse[bk * cols + c]);
      dv.add(y, p);
      dk.add(x, p * (vv.dot(y) - dvec[bk * cols + c]) * scale);
    }
  }
  dk.store(dkv + row, lane, 1.f);
  dv.store(dkv + row + Akv, lane, 1.f);
}

}  // namespace


template <typename T, int D>
int plain(const CrossShape& s, const void* q, const void* kv, const int32_t* len, void* ctx, float* lse, hipStream_t st) {
  const Geo g{s.Lq, s.Lk, s.heads, s.kv_heads, s.share()};
  hipLaunchKernelGGL((cross_plain_kernel<T, D>), dim3((unsigned)(s.B * s.kv_heads * s.columns())), dim3(64), 0, st, g, (const T*)q, (const T*)kv, len, (T*)ctx, lse);
  return check_launch();
}
template <typename T, int D>
int plain_bwd(const CrossShape& s, const void* q, const void* kv, const int32_t* len, const void* ctx, const void* dctx, const float* lse,
              void* dq, void* dkv, float* dvec, hipStream_t st) {
  const Geo g{s.Lq, s.Lk, s.heads, s.kv_heads, s.share()};
  hipLaunchKernelGGL((cross_plain_dq_kernel<T, D>), dim3((unsigned)(s.B * s.kv_heads * s.columns())), dim3(64), 0, st, g, (const T*)q, (const T*)kv, len, (const T*)ctx,
                     (const T*)dctx, lse, (T*)dq, dvec);
  hipLaunchKernelGGL((cross_plain_dkv_kernel<T, D>), dim3((unsigned)(s.B * s.kv_heads * s.Lk)), dim3(64), 0, st, g, (const T*)q, (const T*)kv, len, (const T*)dctx, lse,
                     dvec, (T*)dkv);
  return check_launch();
}

int launch_cross_attention_f32(const CrossShape& s, const void* q, const void* kv, const int32_t* src_len, void* ctx, float* lse, void*, hipStream_t st) {
  return s.d == 64 ? plain<float, 64>(s, q, kv, src_len, ctx, lse, st) : plain<float, 128>(s, q, kv, src_len, ctx, lse, st);
}
int launch_cross_attention_f32_bwd(const CrossShape& s, const void* q, const void* kv, const int32_t* src_len,
                               const void* ctx, const void* dctx, const float* lse, void* dq, void* dkv, float* dvec, hipStream_t st) {
    return s.d == 64 ? plain_bwd<float, 64>(s, q, kv, src_len, ctx, dctx, lse, dq, dkv, dvec, st)
                     : plain_bwd<float, 128>(s, q, kv, src_len, ctx, dctx, lse, dq, dkv, dvec, st);
}

}  // namespace moe
