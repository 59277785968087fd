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

// The forward pass of few columns cuts the states into ranges, side by side; what each leaves of a column: its maximum (log2 units in bf16, natural in
// fp32) and sum, and its sum of rows of V.
struct CrossParts {
  int splits;
  float2* stats;             // [B kv_heads columns, splits]
  float* sums;               // [B kv_heads columns, splits, d]
};
// few: blocks of 32 columns whose wavefronts take the states' blocks in turn, in `splits` ranges; else blocks of 128 columns
struct CrossPlan { bool few; int splits; };
CrossPlan cross_plan(int act_dtype, const CrossShape& s);
CrossPlan cross_pair_plan(const CrossShape& s);            // q and ctx in pairs: of 16 and 64 columns
// Blocks of 64 columns in a range of dK's and dV's (bf16), by what the calls are expected to take (us): a block of 128 states walks its range's blocks in
// steps, the ranges' sums cost a launch and their way to memory and back, and ranges are only made while all blocks run at once (a unit has two at d 64).
// us of one range / the best number of them: 4 x 2000 tokens, 1000 states, 8 heads of 128 on one 455 / 87 (8), of 64 295 / 51 (16); 7 x 1561, up to 66, 2 on one
// of 128 93 / 19 (16), of 64 61 / 16 (16); 1 x 2000, 60, 2 heads of 128 63 / 17 (12); 8 x 1000, 100, 8 heads of 64 24 / 18 (4), of 128 37 / 26 (4); 1 x 500, 500,
// 8 heads of 64 14.5 / 15.9 (4).  Left to one range although more are a little faster: 3 x 700, up to 700, 4 heads of 128 28.2 / 24.8 (3); 2 x 1000, 1000, 8
// heads of 128 39.3 / 37.2 (2).
int cross_dkv_blocks(const CrossShape& s);
int cross_pair_dkv_blocks(const CrossShape& s);

// fp32 (cross_attention_f32.hip)
int launch_cross_attention_f32(const CrossShape& s, const CrossPlan& plan, const float* q, const float* kv, const int32_t* src_len,
                               float* ctx, float* lse, const CrossParts& parts, hipStream_t st);
int launch_cross_attention_f32_bwd(const CrossShape& s, const float* q, const float* kv, const int32_t* src_len, const float* ctx,
                                   const float* dctx, const float* lse, float* dq, float* dkv, float* dvec, hipStream_t st);

}  // namespace moe
