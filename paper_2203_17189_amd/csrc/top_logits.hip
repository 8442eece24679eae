// The K largest logits of each row, in descending order, equal ones by ascending id: what a teacher hands to the
// distillation loss.  Bound by bytes: every logit is read once, 8 K bytes a row are written.
//
// A logit and its id form one 64-bit key, (value ordered as an unsigned number) * 2^32 + (2^32 - 1 - id): keys of a row
// differ, so "the K largest" has one answer.  A workgroup reads its row a chunk at a time into registers.  In the first
// chunk a value that the largest of K of 64 to 256 groups reach is a lower bound of the row's K-th largest value, and few
// elements reach it: these are collected in LDS.  Later chunks add what exceeds the K-th largest key so far.  A wavefront's 64
// groups are asked for their share of K and the least share counts, so rows whose large values lie side by side are bounded
// badly; with more keys at the bound than LDS holds (128 in the form of one wavefront, 512 in that of two, else 2048) a row is
// read again: for its ties if these are what is too many, else once for each of a key's 64 bits.
// Measured on one MI355X, independent logits, captured into a graph: 8192 rows of 32128 in bf16, K = 64, 100 to 105 us (5.0 to
// 5.3 TB/s; a copy's 5.2 come to 103); 1023 rows of 100003 in float32, 13 elements between them, K = 100, 90 us (4.5 TB/s); 8 rows
// of 32128 in float32, K = 16, 8.4 us: one pass of a workgroup each, from the loads to the ranking.  Bit by bit: 19.8 ms for the
// first of these with all but 600 neighbouring logits at -inf, 5.9 ms for 8192 x 8000, K = 32, with 200 neighbours above the rest
// (36.7 us without).
#include "kernels.h"
#include "vocab_rows.h"
#include <algorithm>
#include <type_traits>

namespace t5mi {

namespace {

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

// Largest element of a 16-byte piece; a NaN stays.  (bf16 by its bits: from values the compiler forms bf16 maxima, four
// instructions an element.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
template <typename T>
__device__ __forceinline__ float piece_max(u32x4 r);
template <>
__device__ __forceinline__ float piece_max<float>(u32x4 r) {
  const f32x4 v = __builtin_bit_cast(f32x4, r);
  return __builtin_elementwise_maximum(max3(v[0], v[1], v[2]), v[3]);
}
template <>
__device__ __forceinline__ float piece_max<bf16>(u32x4 r) {
  float m = __builtin_bit_cast(float, r[0] << 16);
  m = __builtin_elementwise_maximum(m, __builtin_bit_cast(float, r[0] & 0xFFFF0000u));
#pragma unroll
  for (int k = 1; k < 4; ++k)
    m = max3(m, __builtin_bit_cast(float, r[k] << 16), __builtin_bit_cast(float, r[k] & 0xFFFF0000u));
  return m;
}

template <int NT>
struct TopShared {
  // keys collected at most: with 1024 and 2048 for one and two wavefronts, LDS holds fewer rows on a compute unit (16384 x 500,
  // K = 16: 21.5 us against 17.3; 8192 x 8000, K = 64: 57.0 and 47.8)
  static constexpr int kKeys = NT == 64 ? 256 : NT == 128 ? 512 : 2048;
  alignas(16) uint32_t best[256];
  alignas(16) uint64_t cand[kKeys];
  uint32_t places[NT];
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
  const int tid = threadIdx.x;
  constexpr int R = (TopShared<NT>::kKeys + NT - 1) / NT;
  if (C > (NT < 1024 ? 2 * NT : NT)) {
    // the K-th largest, from its highest bit down; the keys below it are dropped
    uint64_t key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = r * NT + tid < C ? s.cand[r * NT + tid] : 0;
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t probe = t | 1ull << bit;
      uint32_t n = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) n += key[r] >= probe ? 1 : 0;
      if ((int)block_total(s, n) >= K) t = probe;
    }
    if (tid == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (key[r] >= t && key[r] != 0) s.cand[atomicAdd(&s.count, 1u)] = key[r];
    __syncthreads();
    C = K;
  }
  // Each key's place is the number of larger ones; where keys are few, several threads count a part of the list each.
  // (C <= 2 NT, and C <= 1024.)
  const int keys = C <= 64 ? 64 : C <= 128 ? 128 : C <= 256 ? 256 : C <= 512 ? 512 : 1024;  // threads a part, C and more (or 2 NT)
  const int parts = keys < NT ? NT / keys : 1, part = keys < NT ? tid / keys : 0, own = keys < NT ? tid % keys : tid;
  if (tid == 0 && C & 1) s.cand[C] = 0;  // (C < kKeys here)
  const bool two = C > NT;
  const uint64_t k0 = own < C ? s.cand[own] : 0, k1 = two && NT + tid < C ? s.cand[NT + tid] : 0;
  int place0 = 0, place1 = 0;
  __syncthreads();
  const u32x4* pair = reinterpret_cast<const u32x4*>(s.cand);
  const int pairs = (C + 1) / 2, each = (pairs + parts - 1) / parts, j1 = min(pairs, (part + 1) * each);
  if ((own & ~63) < C) {  // (this wavefront holds keys)
    if (!two) {
#pragma unroll 4
      for (int j = part * each; j < j1; ++j) {
        const u32x4 o = pair[j];
        place0 += (((uint64_t)o[1] << 32 | o[0]) > k0) + (((uint64_t)o[3] << 32 | o[2]) > k0);
      }
    } else {
#pragma unroll 4
      for (int j = 0; j < pairs; ++j) {
        const u32x4 o = pair[j];
        const uint64_t a = (uint64_t)o[1] << 32 | o[0], b = (uint64_t)o[3] << 32 | o[2];
        place0 += (a > k0) + (b > k0);
        place1 += (a > k1) + (b > k1);
      }
    }
  }
  s.places[tid] = place0;
  __syncthreads();
  if (part == 0) {
    for (int q = 1; q < parts; ++q) place0 += s.places[q * keys + own];
    if (own < C && place0 < K) {
      s.cand[place0] = k0;
      if (place0 == K - 1) s.floor = k0;
    }
    if (two && NT + tid < C && place1 < K) {
      s.cand[place1] = k1;
      if (place1 == K - 1) s.floor = k1;
    }
  }
  if (tid == 0) s.count = K;
  __syncthreads();
}

// NT threads a row, NP pieces of 16 bytes a thread in a chunk, or (ONE) of one element: rows too short to give every
// thread a whole piece.
template <typename T, int NT, int NP, bool ONE>
__global__ __launch_bounds__(NT, NT == 256 ? (NP > 4 && !ONE ? 5 : 6) : NP == 8 ? 8 : 4) void top_logits_kernel(
    const T* __restrict__ logits, int V, int64_t ld, int K, float* __restrict__ values, int32_t* __restrict__ ids) {
  constexpr int EPV = ONE ? 1 : RowSplit<T>::EPV;
  constexpr bool kAgain = NP > 4 && !ONE;  // pieces that matter are read again (from L2) instead of held
  typedef typename RowVec<T>::type VT;
  __shared__ TopShared<NT> s;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  const RowSplit<T> sp(x, V);
  const int head = ONE ? 0 : sp.head, pieces = ONE ? V : sp.pieces, last = pieces - 1;
  const u32x4* body = reinterpret_cast<const u32x4*>(x + head);
  if (tid == 0) {
    s.level = ~0u;
    s.count = 0;
  }
  const int own = ONE ? -1 : sp.single(tid, NT, V);
  const float xs = own >= 0 ? to_f32(x[own]) : -INFINITY;
  // twice K groups: fewer wavefronts to share K among than with 256 of them, which bound independent values no better (8192 x
  // 32128, K = 16: 90 us with either; K = 64: 101 and 99)
  const int groups = K <= 32 ? 64 : K <= 96 ? 128 : 256;
  bool crowded = false;
  uint32_t level = 0;  // value of the bound
  for (int p0 = 0; p0 == 0 || p0 < pieces; p0 += NT * NP) {
    float top[NP];  // largest of each piece
    u32x4 raw[ONE ? 1 : NP];
    if constexpr (ONE) {
#pragma unroll
      for (int i = 0; i < NP; ++i) top[i] = to_f32(x[min(p0 + i * NT + tid, last)]);
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) raw[i] = last >= 0 ? body[min(p0 + i * NT + tid, last)] : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NP; ++i) top[i] = piece_max<T>(raw[i]);
    }
    const bool with_single = p0 == 0 && own >= 0;
    if (p0 == 0) {
      // a value that at least K of `groups` groups' largest values reach
      uint32_t g = with_single ? ordered(xs) : 0;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (i * NT + tid < pieces) g = max(g, ordered(top[i]));
      for (int off = 1; off < NT / groups; off <<= 1) g = max(g, (uint32_t)__shfl_xor(g, off, 64));
      if (NT <= groups || tid % (NT / groups) == 0) s.best[NT <= groups ? tid : tid / (NT / groups)] = g;
      __syncthreads();
      // each wavefront's share of K among its 64 groups, bit by bit (K = 16: 16384 x 64 9.9 us, 16.4 by counting, for each group,
      // the larger ones in LDS; 8 x 32128 in float32 8.0 and 9.5)
      if (tid < groups) {
        constexpr bool kHalf = sizeof(T) == 2;
        const uint32_t mine = s.best[tid];
        const int need = (K * 64 + groups - 1) / groups;
        uint32_t t = 0;
#pragma unroll 4
        for (int bit = 31; bit >= (kHalf ? 16 : 0); --bit) {
          const uint32_t probe = t | 1u << bit;
          if (__popcll(__ballot(mine >= probe)) >= need) t = probe;
        }
        if (kHalf) t |= t > 0xFF800000u ? 0xFFFFu : t >> 31 ? 0u : 0xFFFFu;  // the lower half of a bf16's order: NaN, +, -
        if ((tid & 63) == 0) atomicMin(&s.level, t);  // (no element is less where some groups hold none)
      }
      __syncthreads();
    }
    const uint64_t floor = p0 == 0 ? (uint64_t)s.level << 32 : s.floor;
    level = (uint32_t)(floor >> 32);
    auto offer = [&](const float* v, int n, int id) {
      uint32_t take = 0;
#pragma unroll
      for (int k = 0; k < n; ++k) take |= make_key(v[k], id + k) >= floor ? 1u << k : 0;
      if (!take) return;
      uint32_t at = atomicAdd(&s.count, (uint32_t)__popc(take));
#pragma unroll
      for (int k = 0; k < n; ++k)
        if (take >> k & 1) {
          if (at < (uint32_t)TopShared<NT>::kKeys) s.cand[at] = make_key(v[k], id + k);
          ++at;
        }
    };
    auto offer_piece = [&](u32x4 r, int p) {
      const VT v = __builtin_bit_cast(VT, r);
      float f[EPV];
#pragma unroll
      for (int k = 0; k < EPV; ++k) f[k] = to_f32(v[k]);
      offer(f, EPV, head + p * EPV);
    };
    if (with_single) offer(&xs, 1, own);
    if constexpr (kAgain) {
      uint32_t reach = 0;
#pragma unroll
      for (int i = 0; i < NP; ++i) reach |= p0 + i * NT + tid < pieces && ordered(top[i]) >= level ? 1u << i : 0;
      while (reach) {
        const int p = p0 + (__ffs(reach) - 1) * NT + tid;
        reach &= reach - 1;
        offer_piece(body[p], p);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int p = p0 + i * NT + tid;
        if (p < pieces && ordered(top[i]) >= level) {
          if constexpr (ONE) offer(&top[i], 1, p);
          else offer_piece(raw[i], p);
        }
      }
    }
    __syncthreads();
    const int C = (int)s.count;
    if (C > TopShared<NT>::kKeys || (NT == 64 && C > 128)) {
      crowded = true;
      break;
    }
    if (C > K || p0 == 0) keep_top(s, C, K);
    else __syncthreads();
  }
  if (crowded) {
    // Mostly ties: if fewer than K elements exceed the bound's value, they and the first of those equal to it are the answer.
    uint32_t more = 0, same = 0;
    for (int c = tid; c < V; c += NT) {
      const uint32_t o = ordered(to_f32(x[c]));
      more += o > level;
      same += o == level;
    }
    more = block_total(s, more);
    same = block_total(s, same);
    if (tid == 0) s.count = 0;
    __syncthreads();
    if ((int)more < K && (int)(more + same) >= K) {
      int need = K - (int)more;  // of those equal to the bound, in order of ids
      for (int c0 = 0; c0 < V; c0 += NT) {
        const int c = c0 + tid;
        const uint64_t k = c < V ? make_key(to_f32(x[c]), c) : 0;
        if ((uint32_t)(k >> 32) > level) s.cand[atomicAdd(&s.count, 1u)] = k;
        if (need > 0) {
          const uint64_t eq = __ballot(c < V && (uint32_t)(k >> 32) == level);
          if ((tid & 63) == 0) s.places[tid >> 6] = (uint32_t)__popcll(eq);
          __syncthreads();
          int before = 0, all = 0;
          for (int q = 0; q < NT / 64; ++q) {
            before += q < tid >> 6 ? (int)s.places[q] : 0;
            all += (int)s.places[q];
          }
          if ((eq >> (tid & 63) & 1) && before + __popcll(eq & ((1ull << (tid & 63)) - 1)) < need)
            s.cand[atomicAdd(&s.count, 1u)] = k;
          need -= all;
          __syncthreads();
        }
      }
    } else {
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
        if (k >= t) s.cand[atomicAdd(&s.count, 1u) & (TopShared<NT>::kKeys - 1)] = k;  // K of them
      });
    }
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
  const int pieces = ceil_div(V, type == IN_BF16 ? 8 : 4);
  auto go = [&](auto kern, int nt, auto* p) { kern<<<(unsigned)rows, nt, 0, st>>>(p, V, ld, K, values, ids); };
  auto of_type = [&](auto* p) {
    typedef typename std::remove_const<typename std::remove_pointer<decltype(p)>::type>::type T;
    // (bf16 unless it says otherwise, us.)  One element at a time where pieces are too few to bound K well (16384 x 500,
    // K = 100: 64, by pieces 275 and 306; 4096 x 4000: 31.0 and 34.0).  Many rows: one or two wavefronts each as long as 16
    // pieces a lane hold the row and their 64 or 128 groups bound K, so that more rows are on their way at a time (with four
    // wavefronts second: 16384 x 500, K = 16: 16.9 and 42.3; 8192 x 2048, K = 16: 15.9 and 28.7; 8192 x 8000, K = 64: 47.5 and 60.7;
    // 8192 x 16000, K = 64: 71.7 and 82.7; 8192 x 32128, K = 64, which two wavefronts take in chunks: 123 and 101).  Of 513 to 1024
    // pieces one wavefront gains nothing on two (8192 x 5000, K = 8: 21.9 and 22.4; 8192 x 8000, K = 32: 36.5 and 35.1; 600 x
    // 8000, K = 16: 9.0 and 7.7).  Fewer than 512 rows: four wavefronts (400 x 8000, K = 64: 10.0, with two 12.6), or 16 on rows of
    // more than 64 KB as long as each row has a compute unit (8 x 32128 in float32: 8.4, with four 10.5; 256 x 131072: 20.2 and
    // 29.2; 300 rows of 36000: 21.3 and 18.0, of 131072 in float32 56.8 and 54.2, in bf16 29.9 and 32.7).  Rows of up to 16 KB are
    // one chunk of four pieces a lane (8192 x 8000, K = 120: 84, with sixteen 103); the shortest take as few loads as they have
    // elements for (16384 x 64, K = 8: 9.9 and 12.3; 8192 x 500, K = 64: 18.0 and 20.0).
    const bool many = rows >= 512;
    if (V <= 256 && K <= 32) go(top_logits_kernel<T, 64, 4, true>, 64, p);
    else if (V <= 1024 && K <= 32) go(top_logits_kernel<T, 64, 16, true>, 64, p);
    else if (V <= 1024 && K <= 96 && many) go(top_logits_kernel<T, 128, 8, true>, 128, p);
    else if (V <= 2048 && K > pieces / 8 && K <= 96 && many) go(top_logits_kernel<T, 128, 16, true>, 128, p);
    else if (V <= 4096 && K > pieces / 8) go(top_logits_kernel<T, 256, 16, true>, 256, p);
    else if (rows <= 256 && pieces > 4096) go(top_logits_kernel<T, 1024, 16, false>, 1024, p);
    else if (pieces <= 512 && K <= 32 && many) go(top_logits_kernel<T, 64, 8, false>, 64, p);
    else if (pieces <= 1024 && K <= 32 && many) go(top_logits_kernel<T, 64, 16, false>, 64, p);
    else if (pieces <= 1024 && K <= 96 && many) go(top_logits_kernel<T, 128, 8, false>, 128, p);
    else if (pieces <= 2048 && K <= 96 && many) go(top_logits_kernel<T, 128, 16, false>, 128, p);
    else if (pieces <= 1024) go(top_logits_kernel<T, 256, 4, false>, 256, p);
    else go(top_logits_kernel<T, 256, 16, false>, 256, p);
  };
  if (type == IN_BF16) of_type((const bf16*)logits);
  else of_type((const float*)logits);
  return hipGetLastError();
}

}  // namespace t5mi
