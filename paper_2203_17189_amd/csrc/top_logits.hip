// The K largest logits of each row, in descending order, equal ones by ascending id: what a teacher hands to the
// distillation loss.  Bound by bytes: every logit is read, 8 K bytes a row are written.
//
// A logit and its id form one 64-bit key, (value ordered as an unsigned number) * 2^32 + (2^32 - 1 - id): keys of a row
// differ, so "the K largest" has one answer.  Each of a workgroup's threads takes the largest key of the elements it
// owns; the K-th largest of these is a lower bound of the K-th largest key, and few keys lie above it (a thread holds
// one of the K largest for every one that another lacks): those are collected in LDS, ranked against each other, and
// written.  Rows laid out against that (thousands of keys above the bound) are searched bit by bit instead.
#include "kernels.h"
#include <algorithm>

namespace t5mi {

namespace {

constexpr int kCand = 2048;  // keys collected in LDS at most

// -0 counts as +0, NaN as larger than everything else.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  if (x != x) return 0xFFFFFFFFu;
  if (b == 0x80000000u) return 0x80000000u;
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __builtin_bit_cast(float, o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t make_key(float x, int id) { return (uint64_t)ordered(x) << 32 | (uint32_t)~id; }

template <typename T, int EPV> struct Pieces { typedef __attribute__((ext_vector_type(EPV))) T type; };
template <typename T> struct Pieces<T, 1> { typedef T type; };

// f(key) for every element of the row that this thread owns.
template <typename T, int EPV, typename F>
__device__ __forceinline__ void each_key(const T* __restrict__ x, int V, F f) {
  typedef typename Pieces<T, EPV>::type P;
  for (int c = (int)threadIdx.x * EPV; c < V; c += 256 * EPV) {
    const P v = *reinterpret_cast<const P*>(x + c);
    if constexpr (EPV == 1) {
      f(make_key(to_f32(v), c));
    } else {
#pragma unroll
      for (int k = 0; k < EPV; ++k) f(make_key(to_f32(v[k]), c + k));
    }
  }
}

template <typename T, int EPV>
__global__ __launch_bounds__(256) void top_logits_kernel(const T* __restrict__ logits, int V, int64_t ld, int K,
                                                         float* __restrict__ values, int32_t* __restrict__ ids) {
  __shared__ uint64_t best[256];
  __shared__ uint64_t cand[kCand];
  __shared__ uint64_t bound;
  __shared__ uint32_t count;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  uint64_t mine = 0;
  each_key<T, EPV>(x, V, [&](uint64_t k) { mine = k > mine ? k : mine; });
  best[tid] = mine;
  if (tid == 0) { bound = 0; count = 0; }
  __syncthreads();
  int above = 0;
  for (int i = 0; i < 256; ++i) above += best[i] > mine ? 1 : 0;
  if (mine != 0 && above == K - 1) bound = mine;  // (threads without elements leave no bound)
  __syncthreads();
  uint64_t b = bound;
  each_key<T, EPV>(x, V, [&](uint64_t k) {
    if (k >= b) {
      const uint32_t i = atomicAdd(&count, 1u);
      if (i < kCand) cand[i] = k;
    }
  });
  __syncthreads();
  int C = (int)count;
  if (C > kCand) {
    // the K-th largest key, from its highest bit down
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t probe = t | 1ull << bit;
      __syncthreads();
      if (tid == 0) count = 0;
      __syncthreads();
      uint32_t n = 0;
      each_key<T, EPV>(x, V, [&](uint64_t k) { n += k >= probe ? 1 : 0; });
      if (n) atomicAdd(&count, n);
      __syncthreads();
      if ((int)count >= K) t = probe;
    }
    __syncthreads();
    if (tid == 0) count = 0;
    __syncthreads();
    each_key<T, EPV>(x, V, [&](uint64_t k) {
      if (k >= t) cand[atomicAdd(&count, 1u) & (kCand - 1)] = k;
    });
    __syncthreads();
    C = K;
  }
  for (int i = tid; i < C; i += 256) {
    const uint64_t k = cand[i];
    int r = 0;
    for (int j = 0; j < C; ++j) r += cand[j] > k ? 1 : 0;
    if (r < K) {
      values[row * K + r] = unordered((uint32_t)(k >> 32));
      ids[row * K + r] = (int32_t) ~(uint32_t)k;
    }
  }
}

}  // namespace

size_t top_logits_ws_bytes(int64_t rows, int V, int K, int type) {
  (void)rows; (void)V; (void)K; (void)type;
  return 0;
}

hipError_t launch_top_logits(const void* logits, int type, int64_t rows, int V, int64_t ld, int K, float* values,
                             int32_t* ids, void* ws, hipStream_t st) {
  (void)ws;
  if (rows <= 0) return hipSuccess;
  const int epv = type == IN_BF16 ? 8 : 4;
  const bool vec = V >= 256 * epv && V % epv == 0 && ld % epv == 0 && ((uintptr_t)logits & 15) == 0;
  const unsigned grid = (unsigned)rows;
  if (type == IN_BF16) {
    if (vec) top_logits_kernel<bf16, 8><<<grid, 256, 0, st>>>((const bf16*)logits, V, ld, K, values, ids);
    else top_logits_kernel<bf16, 1><<<grid, 256, 0, st>>>((const bf16*)logits, V, ld, K, values, ids);
  } else {
    if (vec) top_logits_kernel<float, 4><<<grid, 256, 0, st>>>((const float*)logits, V, ld, K, values, ids);
    else top_logits_kernel<float, 1><<<grid, 256, 0, st>>>((const float*)logits, V, ld, K, values, ids);
  }
  return hipGetLastError();
}

}  // namespace t5mi
