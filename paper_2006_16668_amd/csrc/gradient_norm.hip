// The norm over all of a model's gradients, and the gradients scaled by min(1, max_norm / norm).
//
// Squares are formed and added in 64 bits: the square of any fp32 or bf16 number is exact there and neither overflows nor
// vanishes, and the fp64 units add far faster than memory delivers (2.5e12 bf16 elements a second at 5 TB/s are 5e12 of some 4e13 operations).
// Both passes are bound by memory.  Tensors are cut into chunks of one size in bytes, a block each, whatever tensor they belong
// to, so a list of many small tensors is as few launches as one large one.  Where the tensors are travels as a kernel argument, kPieces of them a launch:
// nothing is copied to the device, and a captured graph holds it.  The second pass walks backwards: what the first has read last is
// still in the memory-side cache.  us: 1141 MB 193 (5.9 TB/s) and 400 (5.7 TB/s); 102 tensors of 19 MB in all 6.3, 2.3 and 8.5 in three launches.
#include <math.h>
#include "common.h"

namespace moe {
namespace {

struct Piece {                               // of a tensor, whole up to 2 GB
  uintptr_t src;                             // lowest bit: fp32
  void* dst;
  unsigned bytes, first;                     // its first chunk of the launch
};
constexpr int kPieces = 165;                 // of a launch, which has 4 KB of arguments
struct Table {
  Piece t[kPieces];
  int n;
  unsigned chunks;
  unsigned chunk_bytes;                      // a multiple of 4 KB
};
static_assert(sizeof(Table) + 64 <= 4096, "the arguments of a launch");

struct Chunk { const char* src; char* dst; unsigned bytes; bool f32; };
template <bool BACKWARDS>
__device__ __forceinline__ Chunk chunk_of(const Table& tab, unsigned c) {
  int lo = 0, hi = tab.n - 1;                // the last piece that begins at or before c
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (tab.t[mid].first <= c) lo = mid;
    else hi = mid - 1;
  }
  const Piece& p = tab.t[lo];
  unsigned k = c - p.first;
  if (BACKWARDS) k = (p.bytes - 1) / tab.chunk_bytes - k;
  const unsigned from = k * tab.chunk_bytes, rest = p.bytes - from;
  return {reinterpret_cast<const char*>(p.src & ~(uintptr_t)1) + from, static_cast<char*>(p.dst) + from,
          rest < tab.chunk_bytes ? rest : tab.chunk_bytes, (p.src & 1) != 0};
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sums[16];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (unsigned w = 0; w < blockDim.x >> 6; ++w) s += sums[w];
  return s;
}

template <typename T>
__device__ __forceinline__ double squares(const Chunk& c) {
  constexpr int E = Vec16<T>::kElts, AHEAD = 4;
  double s[2] = {0.0, 0.0};
  const unsigned vecs = c.bytes / 16;
  auto add = [&](const uint4& v) __attribute__((always_inline)) {
    float f[E];
    Vec16<T>::unpack(v, f);
#pragma unroll
    for (int i = 0; i < E; ++i) s[i & 1] = fma((double)f[i], (double)f[i], s[i & 1]);
  };
  unsigned v = threadIdx.x;
  for (; v + (AHEAD - 1) * 256 < vecs; v += AHEAD * 256) {
    uint4 x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) x[k] = reinterpret_cast<const uint4*>(c.src)[v + k * 256];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) add(x[k]);
  }
  for (; v < vecs; v += 256) add(reinterpret_cast<const uint4*>(c.src)[v]);
  const unsigned tail = (c.bytes - vecs * 16) / sizeof(T);
  if (threadIdx.x < tail) {
    const double f = Elt<T>::load(reinterpret_cast<const T*>(c.src + vecs * 16) + threadIdx.x);
    s[0] = fma(f, f, s[0]);
  }
  return s[0] + s[1];
}

__global__ __launch_bounds__(256) void gradient_squares_kernel(Table tab, double* __restrict__ partial) {
  const Chunk c = chunk_of<false>(tab, blockIdx.x);
  const double s = block_sum(c.f32 ? squares<float>(c) : squares<bf16_t>(c));
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void gradient_norm_kernel(const double* __restrict__ partial, unsigned n, float* __restrict__ norm) {
  double s = 0.0;
  for (unsigned i = threadIdx.x; i < n; i += 1024) s += partial[i];
  s = block_sum(s);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// A scale as m 2^e, m in [1/2, 1]: max_norm / norm may be below the normal numbers of fp32 where the clipped gradients are not.
struct Scale {
  float m;
  int e;
  __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_ldexpf(x * m, e); }
};
template <typename T, bool STREAM>
__device__ __forceinline__ void scale_chunk(const Chunk& c, const Scale& scale) {
  constexpr int E = Vec16<T>::kElts, AHEAD = 4;
  const unsigned vecs = c.bytes / 16;
  auto scaled = [&](const uint4& v) __attribute__((always_inline)) {
    float f[E];
    Vec16<T>::unpack(v, f);
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = scale(f[i]);
    return Vec16<T>::pack(f);
  };
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  const u32x4_t* const src = reinterpret_cast<const u32x4_t*>(c.src);
  u32x4_t* const dst = reinterpret_cast<u32x4_t*>(c.dst);
  auto put = [&](unsigned at, const uint4& x) __attribute__((always_inline)) { __builtin_nontemporal_store(u32x4_t{x.x, x.y, x.z, x.w}, dst + at); };
  auto get = [&](unsigned at) __attribute__((always_inline)) {
    const u32x4_t x = STREAM ? __builtin_nontemporal_load(src + at) : src[at];
    return uint4{x[0], x[1], x[2], x[3]};
  };
  unsigned v = threadIdx.x;
  for (; v + (AHEAD - 1) * 256 < vecs; v += AHEAD * 256) {
    uint4 x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) x[k] = get(v + k * 256);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) put(v + k * 256, scaled(x[k]));
  }
  for (; v < vecs; v += 256) put(v, scaled(get(v)));
  const unsigned tail = (c.bytes - vecs * 16) / sizeof(T);
  if (threadIdx.x < tail) {
    const T* from = reinterpret_cast<const T*>(c.src + vecs * 16) + threadIdx.x;
    Elt<T>::store(reinterpret_cast<T*>(c.dst + vecs * 16) + threadIdx.x, scale(Elt<T>::load(from)));
  }
}
__device__ __forceinline__ void copy_chunk(const Chunk& c) {
  const unsigned vecs = c.bytes / 16;
  for (unsigned v = threadIdx.x; v < vecs; v += 256) reinterpret_cast<uint4*>(c.dst)[v] = reinterpret_cast<const uint4*>(c.src)[v];
  const unsigned tail = (c.bytes - vecs * 16) / 2;
  if (threadIdx.x < tail)
    reinterpret_cast<bf16_t*>(c.dst + vecs * 16)[threadIdx.x] = reinterpret_cast<const bf16_t*>(c.src + vecs * 16)[threadIdx.x];
}

// The clipped gradients are not kept in the caches, where they would take the place of gradients that are still to be read.  STREAM: neither are those
// once they are read, for lists larger than the memory-side cache.  us, norm and clip, into other tensors / in place: 1141 MB 652 / 644 with
// ordinary stores and loads, 609 / 642 with such stores, 598 / 603 with both; 336 MB 164 / 163 and 161 / 162; 176 MB 90 / 83, 84 / 83 and 88 / 89.
constexpr size_t kMemorySideCache = (size_t)256 << 20;
template <bool STREAM>
__global__ __launch_bounds__(256) void clip_gradients_kernel(Table tab, const float* __restrict__ norm, double max_norm) {
  const Chunk c = chunk_of<true>(tab, blockIdx.x);
  const float n = *norm;
  // (a comparison with NaN is false, and an infinite norm scales nothing either: bits are kept, NaN and all)
  if (!((double)n > max_norm && n < INFINITY)) {
    if (c.dst != c.src) copy_chunk(c);
    return;
  }
  int e = 0;
  const float m = (float)frexp(max_norm / (double)n, &e);
  const Scale scale{m, e};
  if (c.f32) scale_chunk<float, STREAM>(c, scale);
  else scale_chunk<bf16_t, STREAM>(c, scale);
}

size_t bytes_of(const moe_gradient& g) { return (size_t)g.count * (g.dtype == MOE_F32 ? 4 : 2); }
size_t total_bytes(const moe_gradient* list, int n) {
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += bytes_of(list[i]);
  return total;
}
// Chunks of 16 KB, or as many times that as keep their number near 4096 (16 of a compute unit).
size_t chunk_size(size_t total) {
  const size_t unit = (size_t)16 << 10, most = (size_t)1 << 30;
  const size_t c = (total / 4096 + unit - 1) / unit * unit;
  return c < unit ? unit : c < most ? c : most;
}
size_t chunks_of(size_t bytes, size_t chunk) { return (bytes + chunk - 1) / chunk; }

// f(table) for as many pieces at a time as a launch takes, forwards or backwards
template <typename F>
int for_tables(const moe_gradient* list, int n, size_t chunk, bool backwards, F&& f) {
  Table tab;
  tab.n = 0;
  tab.chunk_bytes = (unsigned)chunk;
  unsigned long long chunks = 0;
  auto flush = [&]() {
    if (tab.n == 0) return (int)MOE_OK;
    if (chunks > 0x7fffffffULL) return (int)MOE_EUNSUPPORTED;
    tab.chunks = (unsigned)chunks;
    const int rc = f(tab);
    tab.n = 0;
    chunks = 0;
    return rc;
  };
  const size_t piece = ((size_t)1 << 31) / chunk * chunk;      // whole chunks
  for (int j = 0; j < n; ++j) {
    const moe_gradient& g = list[backwards ? n - 1 - j : j];
    const size_t bytes = bytes_of(g), parts = (bytes + piece - 1) / piece;
    for (size_t x = 0; x < parts; ++x) {
      if (tab.n == kPieces) {
        const int rc = flush();
        if (rc != MOE_OK) return rc;
      }
      const size_t from = (backwards ? parts - 1 - x : x) * piece, part = bytes - from < piece ? bytes - from : piece;
      tab.t[tab.n++] = Piece{(reinterpret_cast<uintptr_t>(g.src) + from) | (g.dtype == MOE_F32 ? 1u : 0u),
                             reinterpret_cast<void*>(reinterpret_cast<uintptr_t>(g.dst) + from), (unsigned)part, (unsigned)chunks};
      chunks += chunks_of(part, chunk);
    }
  }
  return flush();
}

}  // namespace

size_t gradient_norm_bytes(const moe_gradient* list, int n) {
  const size_t chunk = chunk_size(total_bytes(list, n));
  size_t chunks = 0;
  for (int i = 0; i < n; ++i) chunks += chunks_of(bytes_of(list[i]), chunk);
  return align_up((chunks + 1) * sizeof(double), 256);
}

int launch_gradient_norm(const moe_gradient* list, int n, float* norm, void* ws, hipStream_t st) {
  double* const partial = static_cast<double*>(ws);
  size_t used = 0;
  const int rc = for_tables(list, n, chunk_size(total_bytes(list, n)), false, [&](const Table& tab) {
    hipLaunchKernelGGL(gradient_squares_kernel, dim3(tab.chunks), dim3(256), 0, st, tab, partial + used);
    used += tab.chunks;
    return check_launch();
  });
  if (rc != MOE_OK) return rc;
  hipLaunchKernelGGL(gradient_norm_kernel, dim3(1), dim3(1024), 0, st, partial, (unsigned)used, norm);
  return check_launch();
}

int launch_clip_gradients(const moe_gradient* list, int n, const float* norm, double max_norm, hipStream_t st) {
  const size_t total = total_bytes(list, n);
  return for_tables(list, n, chunk_size(total), true, [&](const Table& tab) {
    const dim3 grid(tab.chunks), threads(256);
    if (total > kMemorySideCache) hipLaunchKernelGGL((clip_gradients_kernel<true>), grid, threads, 0, st, tab, norm, max_norm);
    else hipLaunchKernelGGL((clip_gradients_kernel<false>), grid, threads, 0, st, tab, norm, max_norm);
    return check_launch();
  });
}

}  // namespace moe
