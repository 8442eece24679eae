// The K largest logits of each row, in descending order, equal ones by ascending id: what a teacher hands to the
// distillation loss.  Bound by bytes: every logit is read once, 8 K bytes a row are written.
//
// A logit and its id form one 64-bit key, (value ordered as an unsigned number) * 2^32 + (2^32 - 1 - id): keys of a row
// differ, so "the K largest" has one answer.  A workgroup reads its row a chunk at a time into registers.  In the first
// chunk the K-th largest of 64 to 256 groups' largest values is a lower bound of the row's K-th largest value, and few
// elements reach it: these are collected in LDS.  Later chunks add what exceeds the K-th largest key so far.  Rows laid
// out against that (thousands of elements above the bound) are searched bit by bit instead.
#include "kernels.h"
#include "vocab_rows.h"
#include <algorithm>

namespace t5mi {

namespace {

constexpr int kCand = 2048;   // keys collected in LDS at most
constexpr int kPieces = 16;   // 16-byte pieces of a thread in a chunk

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

template <int NT>
struct TopShared {
  alignas(16) uint32_t best[256];
  alignas(16) uint64_t cand[kCand];
  uint64_t floor;  // no smaller key is of interest
  uint32_t count, sum, level;
};

// Number of threads' `n` in all, the same in every thread.
template <int NT>
__device__ __forceinline__ uint32_t block_total(TopShared<NT>& s, uint32_t n) {
  __syncthreads();
  if (threadIdx.x == 0) s.sum = 0;
  __syncthreads();
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
  if ((threadIdx.x & 63) == 0) atomicAdd(&s.sum, n);
  __syncthreads();
  return s.sum;
}

// Keeps the K largest of the C >= K keys in s.cand, in descending order, and raises s.floor to the K-th.
template <int NT>
__device__ __forceinline__ void keep_top(TopShared<NT>& s, int C, int K) {
  constexpr int R = (kCand + NT - 1) / NT;
  uint64_t key[R];
  if (C > 512) {
    // the K-th largest, from its highest bit down; the keys below it are dropped
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = r * NT + (int)threadIdx.x < C ? s.cand[r * NT + threadIdx.x] : 0;
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t probe = t | 1ull << bit;
      uint32_t n = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) n += key[r] >= probe ? 1 : 0;
      if ((int)block_total(s, n) >= K) t = probe;
    }
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (key[r] >= t && key[r] != 0) s.cand[atomicAdd(&s.count, 1u)] = key[r];
    __syncthreads();
    C = K;
  }
  // each key's place is the number of larger ones
  constexpr int Q = (512 + NT - 1) / NT;
  int place[Q];
  const bool some = (int)(threadIdx.x & ~63u) < C, more = Q > 1 && C > NT;  // this wavefront holds keys; a second each
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int i = q * NT + threadIdx.x;
    key[q] = i < C ? s.cand[i] : 0;
    place[q] = 0;
  }
  if (threadIdx.x == 0 && C & 1) s.cand[C] = 0;  // (C < kCand here)
  __syncthreads();
  const u32x4* pair = reinterpret_cast<const u32x4*>(s.cand);
  if (some) {
#pragma unroll 4
    for (int j = 0; j < (C + 1) / 2; ++j) {
      const u32x4 two = pair[j];
      const uint64_t a = (uint64_t)two[1] << 32 | two[0], b = (uint64_t)two[3] << 32 | two[2];
      place[0] += (a > key[0]) + (b > key[0]);
      if (more) place[Q - 1] += (a > key[Q - 1]) + (b > key[Q - 1]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < Q; ++q)
    if (q * NT + (int)threadIdx.x < C && place[q] < K) {
      s.cand[place[q]] = key[q];
      if (place[q] == K - 1) s.floor = key[q];
    }
  if (threadIdx.x == 0) s.count = K;
  __syncthreads();
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void top_logits_kernel(const T* __restrict__ logits, int V, int64_t ld, int K,
                                                        float* __restrict__ values, int32_t* __restrict__ ids) {
  constexpr int EPV = RowSplit<T>::EPV;
  typedef typename RowVec<T>::type VT;
  __shared__ TopShared<NT> s;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  const RowSplit<T> sp(x, V);
  const u32x4* body = reinterpret_cast<const u32x4*>(x + sp.head);
  if (tid == 0) {
    s.level = 0;
    s.count = 0;
  }
  const int own = sp.single(tid, NT, V);
  const float xs = own >= 0 ? to_f32(x[own]) : -INFINITY;
  const int last = sp.pieces - 1;
  const int groups = K <= 32 ? 64 : K <= 64 ? 128 : 256;  // twice K bounds nearly as well as more, for fewer comparisons
  bool crowded = false;
  for (int p0 = 0; p0 == 0 || p0 < sp.pieces; p0 += NT * kPieces) {
    float top[kPieces];  // largest of each piece; the pieces themselves are read again (from L2) where they matter
    {
      u32x4 raw[kPieces];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) raw[i] = last >= 0 ? body[min(p0 + i * NT + tid, last)] : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const VT v = __builtin_bit_cast(VT, raw[i]);
        float m = to_f32(v[0]);
#pragma unroll
        for (int k = 1; k < EPV; ++k) m = __builtin_elementwise_maximum(m, to_f32(v[k]));  // (a NaN stays)
        top[i] = m;
      }
    }
    const bool with_single = p0 == 0 && own >= 0;
    if (p0 == 0) {
      // the K-th largest of `groups` groups' largest values: the largest that at least K of them reach
      uint32_t g = with_single ? ordered(xs) : 0;
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        if (p0 + i * NT + tid < sp.pieces) g = max(g, ordered(top[i]));
      for (int off = 1; off < NT / groups; off <<= 1) g = max(g, (uint32_t)__shfl_xor(g, off, 64));
      if (tid % (NT / groups) == 0) s.best[tid / (NT / groups)] = g;
      __syncthreads();
      if (tid < groups) {
        const uint32_t mine = s.best[tid];
        int level = 0;
        const u32x4* four = reinterpret_cast<const u32x4*>(s.best);
#pragma unroll 4
        for (int i = 0; i < groups / 4; ++i) {
          const u32x4 o = four[i];
          level += (o[0] >= mine) + (o[1] >= mine) + (o[2] >= mine) + (o[3] >= mine);
        }
        if (level >= K) atomicMax(&s.level, mine);  // (0 where fewer groups than K hold elements)
      }
      __syncthreads();
    }
    const uint64_t floor = p0 == 0 ? (uint64_t)s.level << 32 : s.floor;
    const uint32_t level = (uint32_t)(floor >> 32);
    auto offer = [&](float v, int id) {
      const uint64_t k = make_key(v, id);
      if (k >= floor) {
        const uint32_t at = atomicAdd(&s.count, 1u);
        if (at < kCand) s.cand[at] = k;
      }
    };
    if (with_single) offer(xs, own);
    uint32_t reach = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) reach |= p0 + i * NT + tid < sp.pieces && ordered(top[i]) >= level ? 1u << i : 0;
    while (reach) {
      const int p = p0 + (__ffs(reach) - 1) * NT + tid;
      reach &= reach - 1;
      const VT v = __builtin_bit_cast(VT, body[p]);
#pragma unroll
      for (int k = 0; k < EPV; ++k) offer(to_f32(v[k]), sp.head + p * EPV + k);
    }
    __syncthreads();
    const int C = (int)s.count;
    if (C > kCand) {
      crowded = true;
      break;
    }
    if (C > K || p0 == 0) keep_top(s, C, K);
    else __syncthreads();
  }
  if (crowded) {
    // the row's K-th largest key, from its highest bit down; the row is read for each
    auto each = [&](auto f) {
      for (int c = tid; c < V; c += NT) f(make_key(to_f32(x[c]), c));
    };
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t probe = t | 1ull << bit;
      uint32_t n = 0;
      each([&](uint64_t k) { n += k >= probe ? 1 : 0; });
      if ((int)block_total(s, n) >= K) t = probe;
    }
    if (tid == 0) s.count = 0;
    __syncthreads();
    each([&](uint64_t k) {
      if (k >= t) s.cand[atomicAdd(&s.count, 1u) & (kCand - 1)] = k;  // K of them
    });
    __syncthreads();
    keep_top(s, K, K);
  }
  for (int i = tid; i < K; i += NT) {
    const uint64_t k = s.cand[i];
    values[row * K + i] = unordered((uint32_t)(k >> 32));
    ids[row * K + i] = (int32_t) ~(uint32_t)k;
  }
}

}  // namespace

hipError_t launch_top_logits(const void* logits, int type, int64_t rows, int V, int64_t ld, int K, float* values,
                             int32_t* ids, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  // few rows: all of a compute unit's wavefronts on one; many: four workgroups of a compute unit overlap
  const bool wide = rows < 512 && V >= 16384;
  auto go = [&](auto kern, auto* p) { kern<<<(unsigned)rows, wide ? 1024 : 256, 0, st>>>(p, V, ld, K, values, ids); };
  if (type == IN_BF16) {
    if (wide) go(top_logits_kernel<bf16, 1024>, (const bf16*)logits);
    else go(top_logits_kernel<bf16, 256>, (const bf16*)logits);
  } else {
    if (wide) go(top_logits_kernel<float, 1024>, (const float*)logits);
    else go(top_logits_kernel<float, 256>, (const float*)logits);
  }
  return hipGetLastError();
}

}  // namespace t5mi
