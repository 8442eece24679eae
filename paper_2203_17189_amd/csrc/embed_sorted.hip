// Token embedding with a scale, and the gradient of its table by sorted tokens:
//   x[t, :] = scale * E[id_t, :],      dE[v, :] (+)= scale * sum over { t : id_t = v } of dx[t, :].
// Both are bound by bytes: the lookup moves 2 n d elements, the gradient reads n d elements and writes the table's
// float32 gradient once.  The gradient needs neither atomics nor a cleared table: positions are sorted by id (stable,
// so the positions of a row ascend), and every row of the table is written by the wavefront that sums it.
#include "kernels.h"
#include <algorithm>

namespace t5mi {

namespace {

__device__ __forceinline__ uint32_t clamp_id(int32_t id, int vocab) {
  return (uint32_t)(id < 0 ? 0 : (id >= vocab ? vocab - 1 : id));
}

template <typename T, int N> struct Piece { typedef __attribute__((ext_vector_type(N))) T type; };
template <typename T> struct Piece<T, 1> { typedef T type; };

// ------------------------------------------------------------------------------------------------
// Lookup.  A workgroup takes rows_per_block consecutive tokens, their rows cut into pieces of EPV elements (16 bytes
// where rows allow it), four pieces per thread in flight.
// ------------------------------------------------------------------------------------------------
template <typename T, int EPV>
__global__ __launch_bounds__(256) void embed_scaled_fwd_kernel(const int32_t* __restrict__ tok, const T* __restrict__ E,
                                                               T* __restrict__ x, int64_t n, int d, int vocab,
                                                               float scale, int rows_per_block) {
  typedef typename Piece<T, EPV>::type P;
  const uint32_t cpr = (uint32_t)d / EPV;
  const int64_t r0 = (int64_t)blockIdx.x * rows_per_block;
  const uint32_t m = (uint32_t)(n - r0 < rows_per_block ? n - r0 : rows_per_block) * cpr;
  for (uint32_t t0 = threadIdx.x; t0 < m; t0 += 1024) {
    P v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t t = t0 + 256 * u;
      if (t >= m) break;
      const uint32_t r = t / cpr, c = t - r * cpr;
      v[u] = reinterpret_cast<const P*>(E + (size_t)clamp_id(tok[r0 + r], vocab) * d)[c];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t t = t0 + 256 * u;
      if (t >= m) break;
      if constexpr (EPV == 1) {
        v[u] = from_f32<T>(to_f32(v[u]) * scale);
      } else {
#pragma unroll
        for (int k = 0; k < EPV; ++k) v[u][k] = from_f32<T>(to_f32(v[u][k]) * scale);
      }
      reinterpret_cast<P*>(x + (size_t)r0 * d)[t] = v[u];
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Stable sort of (id, position) by id: least significant digit first, `bits` bits a pass, two launches a pass.
// Workgroup b owns positions [b * chunk, (b + 1) * chunk) of the pass's input.
// ------------------------------------------------------------------------------------------------
constexpr int kSortItems = 8;                 // keys of a thread at a time
constexpr int kSortTile = 256 * kSortItems;   // keys of a workgroup at a time
constexpr int kSortBlocks = 256;              // at most; a workgroup then loops over its chunk

struct SortPass {
  const int32_t* tok;  // first pass: ids as given; else null
  const u32x2* in;     // (id, position), sorted by the lower digits
  u32x2* out;
  uint32_t* hist;      // [blocks][1 << bits]
  int32_t n, vocab, chunk, blocks, shift, bits;
};

__device__ __forceinline__ u32x2 sort_load(const SortPass& p, int i) {
  if (p.tok) return u32x2{clamp_id(p.tok[i], p.vocab), (uint32_t)i};
  return p.in[i];
}

__global__ __launch_bounds__(256) void embed_sort_count_kernel(SortPass p) {
  extern __shared__ uint32_t lds[];
  const int bins = 1 << p.bits;
  for (int i = threadIdx.x; i < bins; i += 256) lds[i] = 0;
  __syncthreads();
  const int i0 = blockIdx.x * p.chunk, i1 = min(i0 + p.chunk, p.n);
  for (int i = i0 + (int)threadIdx.x; i < i1; i += 256)
    atomicAdd(&lds[(sort_load(p, i).x >> p.shift) & (bins - 1)], 1u);  // whole numbers: the order does not matter
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 256) p.hist[(size_t)blockIdx.x * bins + i] = lds[i];
}

// base[d]: first place of digit d's keys of this workgroup = keys of smaller digits + keys of digit d of earlier
// workgroups.  Then tile by tile: each wavefront ranks 512 consecutive keys among equal digits (64 at a time, with
// ballots), the four wavefronts' counts are joined, and every key goes to its place.
__global__ __launch_bounds__(256) void embed_sort_place_kernel(SortPass p) {
  extern __shared__ uint32_t lds[];
  const int bins = 1 << p.bits, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  uint32_t* base = lds;                 // [bins]
  uint32_t* cnt = lds + bins + w * bins;  // this wavefront's, of [4][bins]
  __shared__ uint32_t wsum[4];
  // totals per digit, and the part of earlier workgroups
  uint32_t carry = 0;
  for (int d0 = 0; d0 < bins; d0 += 256) {
    const int d = d0 + tid;
    uint32_t total = 0, before = 0;
    if (d < bins)
      for (int b = 0; b < p.blocks; ++b) {
        const uint32_t c = p.hist[(size_t)b * bins + d];
        total += c;
        before += b < (int)blockIdx.x ? c : 0;
      }
    uint32_t incl = total;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(incl, off, 64);
      incl += lane >= off ? o : 0;
    }
    if (lane == 63) wsum[w] = incl;
    __syncthreads();
    uint32_t pre = carry, all = 0;
    for (int q = 0; q < 4; ++q) {
      pre += q < w ? wsum[q] : 0;
      all += wsum[q];
    }
    if (d < bins) base[d] = pre + incl - total + before;
    carry += all;
    __syncthreads();
  }
  const int i0 = blockIdx.x * p.chunk, i1 = min(i0 + p.chunk, p.n);
  for (int t0 = i0; t0 < i1; t0 += kSortTile) {
    for (int i = lane; i < bins; i += 64) cnt[i] = 0;
    u32x2 key[kSortItems];
    uint32_t rank[kSortItems];
    const int k0 = t0 + w * 64 * kSortItems + lane;
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) key[r] = k0 + r * 64 < i1 ? sort_load(p, k0 + r * 64) : u32x2{0, 0};
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      const bool on = k0 + r * 64 < i1;
      const uint32_t d = (key[r].x >> p.shift) & (bins - 1);
      uint64_t same = __ballot(on);
      for (int b = 0; b < p.bits; ++b) {
        const uint64_t m = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? m : ~m;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the counts of the round before
      if (on) {
        const uint32_t old = cnt[d], below = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        rank[r] = old + below;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (below == 0) cnt[d] = old + (uint32_t)__popcll(same);
      }
    }
    __syncthreads();
    for (int d = tid; d < bins; d += 256) {
      uint32_t s = base[d];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t c = lds[bins + q * bins + d];
        lds[bins + q * bins + d] = s;
        s += c;
      }
      base[d] = s;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r)
      if (k0 + r * 64 < i1) p.out[cnt[(key[r].x >> p.shift) & (bins - 1)] + rank[r]] = key[r];
    __syncthreads();
  }
}

// First index i in sorted[0, n) with id >= v, by one wavefront: 64 probes a step.
__device__ __forceinline__ int wave_lower_bound(const u32x2* __restrict__ sorted, int n, uint32_t v) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;  // the answer is in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + (lane + 1) * step - 1;  // last index of this lane's part
    const uint64_t below = __ballot(i < hi && sorted[i < hi ? i : hi - 1].x < v);
    const int parts = __popcll(below);  // whole parts that lie below v
    const int nlo = lo + parts * step;
    hi = min(hi, nlo + step - 1);
    lo = min(nlo, hi);
  }
  return lo;
}

// One wavefront per row of the table.
template <typename T>
__global__ __launch_bounds__(256) void embed_row_sum_kernel(const u32x2* __restrict__ sorted, int n,
                                                            const T* __restrict__ dx, float* __restrict__ dE, int d,
                                                            int vocab, float scale, int accumulate) {
  const int lane = threadIdx.x & 63;
  const int v = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (v >= vocab) return;
  const int a = wave_lower_bound(sorted, n, (uint32_t)v);
  int b = a;
  for (int i = a;; i += 64) {
    const uint64_t hit = __ballot(i + lane < n && sorted[min(i + lane, n - 1)].x == (uint32_t)v);
    b = i + __popcll(hit);
    if (~hit) break;
  }
  if (a == b && accumulate) return;
  for (int c = lane; c < d; c += 64) {
    float s = 0.f;
    for (int i = a; i < b; ++i) s += to_f32(dx[(size_t)sorted[i].y * d + c]);
    float* o = dE + (size_t)v * d + c;
    *o = accumulate ? *o + scale * s : scale * s;
  }
}

struct SortPlan {
  int bits_each, passes, blocks, chunk;
};
// Ids of up to 16 bits take one or two passes of at most 8 bits, longer ones (22 bits at most) two of at most 11.
SortPlan sort_plan(int64_t n, int vocab) {
  SortPlan s;
  int bits = 1;
  while (bits < 31 && (vocab - 1) >> bits) ++bits;
  s.passes = bits <= 8 ? 1 : 2;
  s.bits_each = ceil_div(bits, s.passes);
  s.blocks = (int)std::min<int64_t>(kSortBlocks, std::max<int64_t>(1, (n + kSortTile - 1) / kSortTile));
  s.chunk = ceil_div(n, (int64_t)s.blocks * kSortTile) * kSortTile;
  s.blocks = std::max(1, ceil_div(n, s.chunk > 0 ? s.chunk : 1));
  return s;
}

}  // namespace

hipError_t launch_embed_scaled_fwd(const int32_t* tokens, const void* E, void* x, int type, int64_t n, int d, int vocab,
                                   float scale, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int epv = type == IN_BF16 ? 8 : 4;
  const bool vec = d % epv == 0 && (((uintptr_t)E | (uintptr_t)x) & 15) == 0;
  const int cpr = vec ? d / epv : d;
  const int rpb = std::max(1, 1024 / cpr);
  const unsigned grid = (unsigned)ceil_div(n, rpb);
  if (type == IN_BF16) {
    if (vec) embed_scaled_fwd_kernel<bf16, 8><<<grid, 256, 0, st>>>(tokens, (const bf16*)E, (bf16*)x, n, d, vocab, scale, rpb);
    else embed_scaled_fwd_kernel<bf16, 1><<<grid, 256, 0, st>>>(tokens, (const bf16*)E, (bf16*)x, n, d, vocab, scale, rpb);
  } else {
    if (vec) embed_scaled_fwd_kernel<float, 4><<<grid, 256, 0, st>>>(tokens, (const float*)E, (float*)x, n, d, vocab, scale, rpb);
    else embed_scaled_fwd_kernel<float, 1><<<grid, 256, 0, st>>>(tokens, (const float*)E, (float*)x, n, d, vocab, scale, rpb);
  }
  return hipGetLastError();
}

size_t embed_sorted_ws_bytes(int64_t n, int vocab, int d) {
  (void)d;
  const SortPlan s = sort_plan(n, vocab);
  return 2 * align_up((size_t)n * sizeof(u32x2)) + align_up(((size_t)s.blocks << s.bits_each) * 4);
}

hipError_t launch_embed_sorted_bwd(const int32_t* tokens, const void* dx, int type, float* dE, int64_t n, int d, int vocab,
                                   float scale, int accumulate, void* ws, hipStream_t st) {
  if (n <= 0 && accumulate) return hipSuccess;
  const SortPlan s = sort_plan(n, vocab);
  u32x2* buf[2] = {(u32x2*)ws, (u32x2*)((char*)ws + align_up((size_t)n * sizeof(u32x2)))};
  uint32_t* hist = (uint32_t*)((char*)ws + 2 * align_up((size_t)n * sizeof(u32x2)));
  const u32x2* sorted = buf[0];
  for (int q = 0; q < s.passes && n > 0; ++q) {
    SortPass p;
    p.tok = q == 0 ? tokens : nullptr;
    p.in = buf[(q + 1) & 1];
    p.out = buf[q & 1];
    p.hist = hist;
    p.n = (int)n; p.vocab = vocab; p.chunk = s.chunk; p.blocks = s.blocks; p.shift = q * s.bits_each; p.bits = s.bits_each;
    embed_sort_count_kernel<<<s.blocks, 256, 4u << s.bits_each, st>>>(p);
    embed_sort_place_kernel<<<s.blocks, 256, 20u << s.bits_each, st>>>(p);
    sorted = p.out;
  }
  const unsigned grid = (unsigned)ceil_div(vocab, 4);
  if (type == IN_BF16)
    embed_row_sum_kernel<bf16><<<grid, 256, 0, st>>>(sorted, (int)n, (const bf16*)dx, dE, d, vocab, scale, accumulate);
  else
    embed_row_sum_kernel<float><<<grid, 256, 0, st>>>(sorted, (int)n, (const float*)dx, dE, d, vocab, scale, accumulate);
  return hipGetLastError();
}

}  // namespace t5mi
