// What the kernels of a decoder's attention to an encoder's states share.
#pragma once
#include "common.h"

namespace moe {

struct CrossGeo {
  int Lq, Lk, heads, kv_heads, share_log2;
  explicit CrossGeo(const CrossShape& s) : Lq(s.Lq), Lk(s.Lk), heads(s.heads), kv_heads(s.kv_heads), share_log2(0) {
    while (1 << share_log2 < s.share()) ++share_log2;
  }
};
// The columns of one key head of a source: column c is head (c % share) of token c / share.
struct CrossCols {
  int count, log2, Lq;
  size_t A;
  __device__ __forceinline__ CrossCols(const CrossGeo& g, int d) : count(g.Lq << g.share_log2), log2(g.share_log2), Lq(g.Lq), A((size_t)g.heads * d) {}
  // elements from q (ctx, ..) to column 0 of key head k of source b, and from there to column c
  __device__ __forceinline__ size_t base(long long b, int k, int d) const { return (size_t)b * Lq * A + ((size_t)k << log2) * d; }
  template <int D> __device__ __forceinline__ size_t offset(int c) const { return (size_t)(c >> log2) * A + (size_t)(c & ((1 << log2) - 1)) * D; }
  __device__ __forceinline__ int within(int c) const { return c < count ? c : count - 1; }
};
// states of source b that hold
__device__ __forceinline__ int held_states(const int32_t* src_len, long long b, int Lk) {
  int n = Lk;
  if (src_len != nullptr) n = __builtin_amdgcn_readfirstlane(src_len[b]);
  return n < 0 ? 0 : n > Lk ? Lk : n;
}

// fp32 (cross_attention_f32.hip)
int launch_cross_attention_f32(const CrossShape& s, const void* q, const void* kv, const int32_t* src_len, void* ctx, float* lse,
                               void* scratch, hipStream_t st);
int launch_cross_attention_f32_bwd(const CrossShape& s, const void* q, const void* kv, const int32_t* src_len, const void* ctx,
                                   const void* dctx, const float* lse, void* dq, void* dkv, float* dvec, hipStream_t st);

}  // namespace moe
