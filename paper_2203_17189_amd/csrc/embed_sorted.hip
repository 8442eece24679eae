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

// Clears out[0, count) with this launch's workgroups from `first` on; the others sort meanwhile.
struct Fill {
  float* out;     // null: nothing to clear
  int64_t count;
  int32_t first;  // workgroup of the launch at which the clearing ones start
};
__device__ __forceinline__ void fill_zero(const Fill& f) {
  const int64_t nb = gridDim.x - f.first, b = blockIdx.x - f.first;
  const int64_t at = ((intptr_t)f.out >> 2) & 3, lead = at ? 4 - at : 0;  // elements in front of a 16-byte boundary
  const int64_t pre = lead < f.count ? lead : f.count, quads = (f.count - pre) / 4;
  f32x4* q = reinterpret_cast<f32x4*>(f.out + pre);
  const int64_t each = (quads + nb - 1) / nb, q1 = (b + 1) * each < quads ? (b + 1) * each : quads;
  for (int64_t i = b * each + threadIdx.x; i < q1; i += blockDim.x) st_stream(q + i, f32x4{0.f, 0.f, 0.f, 0.f});
  if (b == 0 && threadIdx.x < pre) f.out[threadIdx.x] = 0.f;
  const int64_t tail = pre + 4 * quads;
  if (b == nb - 1 && threadIdx.x < f.count - tail) f.out[tail + threadIdx.x] = 0.f;
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
  Fill fill;
};

__device__ __forceinline__ u32x2 sort_load(const SortPass& p, int i) {
  if (p.tok) return u32x2{clamp_id(p.tok[i], p.vocab), (uint32_t)i};
  return p.in[i];
}

__global__ __launch_bounds__(256) void embed_sort_count_kernel(SortPass p) {
  extern __shared__ uint32_t lds[];
  if ((int)blockIdx.x >= p.blocks) {
    fill_zero(p.fill);
    return;
  }
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
  if ((int)blockIdx.x >= p.blocks) {
    fill_zero(p.fill);
    return;
  }
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

// ------------------------------------------------------------------------------------------------
// The same sort by one workgroup, for n <= kOneSort and id and position in 32 bits together: keys in registers, one
// exchange through LDS a pass.  The LDS of the counts is that of the exchange (64 KB in all).
// ------------------------------------------------------------------------------------------------
constexpr int kOneRounds = 16, kOneSort = 1024 * kOneRounds;

__global__ __launch_bounds__(1024) void embed_sort_one_kernel(const int32_t* __restrict__ tok, u32x2* __restrict__ out, int n,
                                                              int vocab, int pos_bits, int passes, int bits, Fill fill) {
  __shared__ uint32_t lds[kOneSort];
  if ((int)blockIdx.x >= fill.first) {
    fill_zero(fill);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int rounds = (n + 1023) / 1024, k0 = w * 64 * rounds + lane;  // wavefront w: 64 * rounds consecutive keys
  const uint32_t bins = 1u << bits;                                   // at most 256
  uint32_t* cnt = lds + w * 256;
  uint32_t* wsum = lds + 16 * 256;
  uint32_t key[kOneRounds], place[kOneRounds];
#pragma unroll
  for (int r = 0; r < kOneRounds; ++r) {
    const int i = k0 + r * 64;
    key[r] = r < rounds && i < n ? clamp_id(tok[i], vocab) << pos_bits | (uint32_t)i : 0;
  }
  for (int q = 0; q < passes; ++q) {
    const int shift = pos_bits + q * bits;
    for (int i = lane; i < 256; i += 64) cnt[i] = 0;
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r) {
      if (r < rounds) {
        const bool on = k0 + r * 64 < n;
        const uint32_t d = (key[r] >> shift) & (bins - 1);
        uint64_t same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
          const uint64_t m = __ballot((d >> b) & 1);
          same &= (d >> b) & 1 ? m : ~m;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the counts of the round before
        if (on) {
          const uint32_t old = cnt[d], below = (uint32_t)__popcll(same & ((1ull << lane) - 1));
          place[r] = old + below;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          if (below == 0) cnt[d] = old + (uint32_t)__popcll(same);
        }
      }
    }
    __syncthreads();
    // places of digit d: after all smaller digits, then wavefront by wavefront
    uint32_t total = 0, incl = 0;
    if (tid < 256) {
#pragma unroll
      for (int i = 0; i < 16; ++i) total += lds[i * 256 + tid];
      incl = total;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_up(incl, off, 64);
        incl += lane >= off ? o : 0;
      }
      if (lane == 63) wsum[w] = incl;
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t p = incl - total;
      for (int i = 0; i < w; ++i) p += wsum[i];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t c = lds[i * 256 + tid];
        lds[i * 256 + tid] = p;
        p += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && k0 + r * 64 < n) place[r] += cnt[(key[r] >> shift) & (bins - 1)];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && k0 + r * 64 < n) lds[place[r]] = key[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && k0 + r * 64 < n) key[r] = lds[k0 + r * 64];
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kOneRounds; ++r)
    if (r < rounds && k0 + r * 64 < n) out[k0 + r * 64] = u32x2{key[r] >> pos_bits, key[r] & ((1u << pos_bits) - 1)};
}

// ------------------------------------------------------------------------------------------------
// Sums over the sorted positions, cut into tiles of `tile` positions however long the runs of equal ids are, so that
// a padding id with half of all positions costs no more than any other.  G lanes take a tile and VEC columns each, eight
// rows in flight.  A run inside its tile is written to its row at once; the part of a run that reaches over an end
// of the tile goes to partial[tile][slot], slot 0 if it is the tile's first run, else 1, and is joined afterwards.
// ------------------------------------------------------------------------------------------------
struct SumArgs {
  const u32x2* sorted;
  const void* dx;
  float* dE;
  float* partial;  // [tiles][2][d]
  int32_t n, d, tile, tiles, slabs, accumulate;
  float scale;
};

template <typename T, int VEC, int G>
__global__ __launch_bounds__(256) void embed_tile_sum_kernel(SumArgs a) {
  typedef typename Piece<T, VEC>::type P;
  typedef typename Piece<float, VEC>::type F;
  uint32_t unit = blockIdx.x * (256 / G) + threadIdx.x / G;
  if (G == 64) unit = __builtin_amdgcn_readfirstlane(unit);
  const int t = unit / a.slabs;
  if (t >= a.tiles) return;
  const int c = ((unit - t * a.slabs) * G + threadIdx.x % G) * VEC;
  const bool on = c < a.d;
  const T* dx = (const T*)a.dx + (on ? c : 0);
  const int t0 = t * a.tile, t1 = min(t0 + a.tile, a.n);
  uint32_t cur = a.sorted[t0].x;
  const bool from_before = t0 > 0 && a.sorted[t0 - 1].x == cur;
  bool first = true;
  F acc{};
  auto flush = [&](bool part) {
    if (!on) return;
    const F v = acc * a.scale;
    if (part) {
      *reinterpret_cast<F*>(a.partial + ((size_t)t * 2 + (first ? 0 : 1)) * a.d + c) = v;
    } else {
      F* o = reinterpret_cast<F*>(a.dE + (size_t)cur * a.d + c);
      *o = a.accumulate ? *o + v : v;
    }
  };
  for (int i = t0; i < t1; i += 8) {
    u32x2 s[8];
    P v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = a.sorted[min(i + j, t1 - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const P*>(dx + (size_t)s[j].y * a.d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i + j >= t1) break;
      if (s[j].x != cur) {
        flush(first && from_before);
        first = false;
        cur = s[j].x;
        acc = F{};
      }
      if constexpr (VEC == 1) {
        acc += to_f32(v[j]);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += to_f32(v[j][k]);
      }
    }
  }
  flush((first && from_before) || (t1 < a.n && a.sorted[t1].x == cur));
}

// First index i in [lo, n) with sorted id > v, by one wavefront: 64 probes a step.
__device__ __forceinline__ int wave_upper_bound(const u32x2* __restrict__ sorted, int lo, int n, uint32_t v) {
  const int lane = threadIdx.x & 63;
  int hi = n;  // the answer is in [lo, hi]
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + (lane + 1) * step - 1;  // last index of this lane's part
    const int parts = __popcll(__ballot(i < hi && sorted[i < hi ? i : hi - 1].x <= v));  // whole parts below the answer
    const int nlo = lo + parts * step;
    hi = min(hi, nlo + step - 1);
    lo = min(nlo, hi);
  }
  return lo;
}

// A workgroup per tile and 256 columns: if a run begins in the tile and reaches over its end, adds the run's parts, in
// order within each wavefront's share of them, and writes the row.
__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs a) {
  const int t = blockIdx.x, t0 = t * a.tile, t1 = min(t0 + a.tile, a.n);
  const uint32_t last = a.sorted[t1 - 1].x;
  if (t1 >= a.n || a.sorted[t1].x != last) return;
  const bool whole = a.sorted[t0].x == last;
  if (whole && t0 > 0 && a.sorted[t0 - 1].x == last) return;  // begins earlier
  __shared__ float red[4][256];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int parts = (wave_upper_bound(a.sorted, t1, a.n, last) - 1) / a.tile - t + 1;  // part 0 here, part i in tile t + i
  const int each = (parts + 3) / 4, p0 = w * each, p1 = min(p0 + each, parts);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  const int c0 = blockIdx.y * 256 + lane;
  for (int p = p0; p < p1; p += 4) {
    float v[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = min(p + j, p1 - 1);
      const float* src = a.partial + ((size_t)(t + q) * 2 + (q == 0 && !whole ? 1 : 0)) * a.d;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[j][k] = c0 + k * 64 < a.d ? src[c0 + k * 64] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += p + j < p1 ? v[j][k] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) red[w][k * 64 + lane] = s[k];
  __syncthreads();
  const int c = blockIdx.y * 256 + threadIdx.x;
  if (c >= a.d) return;
  const float v = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
  float* o = a.dE + (size_t)last * a.d + c;
  *o = a.accumulate ? *o + v : v;
}

// ------------------------------------------------------------------------------------------------
// Few tokens and a small table: one launch.  A workgroup owns kScanRows rows of the table and 64 columns, lists the
// positions of its rows in order, shares the list among its 16 wavefronts (each with sums of its own in LDS), and adds
// these up.
// ------------------------------------------------------------------------------------------------
constexpr int kScanRows = 8, kScanTokens = 4096;

template <typename T>
__global__ __launch_bounds__(1024) void embed_scan_sum_kernel(const int32_t* __restrict__ tok, const T* __restrict__ dx,
                                                              float* __restrict__ dE, int n, int d, int vocab, float scale,
                                                              int accumulate) {
  __shared__ uint32_t list[kScanTokens];  // row << 16 | position
  __shared__ float acc[16][kScanRows][64];
  __shared__ uint32_t wcnt[16], seen[kScanRows];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const uint32_t v0 = blockIdx.x * kScanRows;
  const int c = blockIdx.y * 64 + lane;
  if (tid < kScanRows) seen[tid] = 0;
#pragma unroll
  for (int r = 0; r < kScanRows; ++r) acc[w][r][lane] = 0.f;
  int found = 0;
  for (int b = 0; b < n; b += 1024) {
    const int i = b + tid;
    const uint32_t r = i < n ? clamp_id(tok[i], vocab) - v0 : kScanRows;
    const uint64_t hit = __ballot(r < (uint32_t)kScanRows);
    if (lane == 0) wcnt[w] = (uint32_t)__popcll(hit);
    __syncthreads();
    int at = found;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      at += q < w ? wcnt[q] : 0;
      found += wcnt[q];
    }
    if (r < (uint32_t)kScanRows) {
      list[at + __popcll(hit & ((1ull << lane) - 1))] = r << 16 | (uint32_t)i;
      seen[r] = 1;
    }
    __syncthreads();
  }
  const int each = (found + 15) / 16, l0 = w * each, l1 = min(l0 + each, found);
  for (int l = l0; l < l1; l += 8) {
    uint32_t e[8];
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = list[min(l + j, l1 - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = dx[(size_t)(e[j] & 0xFFFFu) * d + (c < d ? c : 0)];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (l + j < l1) acc[w][e[j] >> 16][lane] += to_f32(v[j]);
  }
  __syncthreads();
  if (tid >= kScanRows * 64 || c >= d || v0 + w >= (uint32_t)vocab || (accumulate && !seen[w])) return;
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) s += acc[q][w][lane];
  float* o = dE + (size_t)(v0 + w) * d + c;
  *o = accumulate ? *o + s * scale : s * scale;
}

struct SortPlan {
  int bits_each, passes, blocks, chunk, pos_bits;  // pos_bits > 0: one workgroup sorts
};
int bits_of(int64_t v) {  // of the numbers 0 .. v, at least 1
  int b = 1;
  while (v >> b) ++b;
  return b;
}
SortPlan sort_plan(int64_t n, int vocab) {
  SortPlan s;
  const int bits = bits_of(vocab - 1);
  s.pos_bits = 0;
  s.blocks = 1;
  s.chunk = 0;
  const int pos_bits = bits_of(n > 0 ? n - 1 : 0);
  if (n <= kOneSort && bits + pos_bits <= 32) {
    s.pos_bits = pos_bits;
    s.passes = ceil_div(bits, 8);
    s.bits_each = ceil_div(bits, s.passes);
    return s;
  }
  // ids of up to 16 bits take one or two passes of at most 8 bits, longer ones (22 bits at most) two of at most 11
  s.passes = bits <= 8 ? 1 : 2;
  s.bits_each = ceil_div(bits, s.passes);
  s.blocks = (int)std::min<int64_t>(kSortBlocks, ceil_div(n, kSortTile));
  s.chunk = ceil_div(n, (int64_t)s.blocks * kSortTile) * kSortTile;
  s.blocks = ceil_div(n, s.chunk);
  return s;
}
int sum_tile(int64_t n) { return n <= 32768 ? 16 : n <= 65536 ? 32 : 64; }

struct BwdWs {
  u32x2* buf[2];
  uint32_t* hist;
  float* partial;
};
size_t carve_bwd_ws(int64_t n, int vocab, int d, void* base, BwdWs* w) {
  const SortPlan s = sort_plan(n, vocab);
  char* p = (char*)base;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* q = p ? p + off : nullptr;
    off += align_up(bytes);
    return (void*)q;
  };
  w->buf[0] = (u32x2*)take((size_t)n * sizeof(u32x2));
  w->buf[1] = (u32x2*)take(s.pos_bits ? 0 : (size_t)n * sizeof(u32x2));
  w->hist = (uint32_t*)take(s.pos_bits ? 0 : ((size_t)s.blocks << s.bits_each) * 4);
  w->partial = (float*)take((size_t)ceil_div(n, sum_tile(n)) * 2 * d * 4);
  return off;
}

template <typename T>
void launch_tile_sum(const SumArgs& a, bool vec, hipStream_t st) {
  SumArgs b = a;
  auto go = [&](auto kern, int vec_n, int G) {
    b.slabs = ceil_div(a.d, G * vec_n);
    kern<<<(unsigned)ceil_div((int64_t)b.tiles * b.slabs, 256 / G), 256, 0, st>>>(b);
  };
  // 64 lanes a tile where they have columns to hold, else 16 (a wavefront then takes four tiles)
  if (vec) {
    if (a.d > 128) go(embed_tile_sum_kernel<T, 4, 64>, 4, 64);
    else go(embed_tile_sum_kernel<T, 4, 16>, 4, 16);
  } else {
    if (a.d > 32) go(embed_tile_sum_kernel<T, 1, 64>, 1, 64);
    else go(embed_tile_sum_kernel<T, 1, 16>, 1, 16);
  }
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
  BwdWs w;
  return carve_bwd_ws(n, vocab, d, nullptr, &w);
}

hipError_t launch_embed_sorted_bwd(const int32_t* tokens, const void* dx, int type, float* dE, int64_t n, int d, int vocab,
                                   float scale, int accumulate, void* ws, hipStream_t st) {
  if (n <= 0 && accumulate) return hipSuccess;
  // one launch where the workgroups of the scan are few (each reads all ids)
  if (n <= kScanTokens && (int64_t)ceil_div(vocab, kScanRows) * ceil_div(d, 64) <= 1024) {
    const dim3 grid((unsigned)ceil_div(vocab, kScanRows), (unsigned)ceil_div(d, 64));
    if (type == IN_BF16)
      embed_scan_sum_kernel<bf16><<<grid, 1024, 0, st>>>(tokens, (const bf16*)dx, dE, (int)n, d, vocab, scale, accumulate);
    else
      embed_scan_sum_kernel<float><<<grid, 1024, 0, st>>>(tokens, (const float*)dx, dE, (int)n, d, vocab, scale, accumulate);
    return hipGetLastError();
  }
  const SortPlan s = sort_plan(n, vocab);
  BwdWs w;
  carve_bwd_ws(n, vocab, d, ws, &w);
  // rows of ids that do not occur: the whole table's gradient is cleared beside the sort, which leaves most of the
  // chip idle, in equal shares of its launches
  const int launches = s.pos_bits ? 1 : 2 * s.passes;
  const int64_t all = accumulate ? 0 : (int64_t)vocab * d, share = ((all + launches - 1) / launches + 3) / 4 * 4;
  int turn = 0;
  auto fill_next = [&](int first) {
    Fill f;
    const int64_t i0 = std::min(all, share * turn), i1 = std::min(all, share * (turn + 1));
    f.out = dE + i0; f.count = i1 - i0; f.first = first;
    ++turn;
    return f;
  };
  auto fill_blocks = [&](const Fill& f, int threads) { return (int)std::min<int64_t>(2048 * 256 / threads, ceil_div(f.count, 64 * threads)); };
  const u32x2* sorted = w.buf[0];
  if (s.pos_bits) {
    const Fill f = fill_next(1);
    embed_sort_one_kernel<<<1 + fill_blocks(f, 1024), 1024, 0, st>>>(tokens, w.buf[0], (int)n, vocab, s.pos_bits, s.passes,
                                                                     s.bits_each, f);
  } else {
    for (int q = 0; q < s.passes; ++q) {
      SortPass p;
      p.tok = q == 0 ? tokens : nullptr;
      p.in = w.buf[(q + 1) & 1];
      p.out = w.buf[q & 1];
      p.hist = w.hist;
      p.n = (int)n; p.vocab = vocab; p.chunk = s.chunk; p.blocks = s.blocks; p.shift = q * s.bits_each; p.bits = s.bits_each;
      p.fill = fill_next(s.blocks);
      embed_sort_count_kernel<<<s.blocks + fill_blocks(p.fill, 256), 256, 4u << s.bits_each, st>>>(p);
      p.fill = fill_next(s.blocks);
      embed_sort_place_kernel<<<s.blocks + fill_blocks(p.fill, 256), 256, 20u << s.bits_each, st>>>(p);
      sorted = p.out;
    }
  }
  if (n == 0) return hipGetLastError();
  SumArgs a;
  a.sorted = sorted; a.dx = dx; a.dE = dE; a.partial = w.partial;
  a.n = (int)n; a.d = d; a.tile = sum_tile(n); a.tiles = ceil_div(n, a.tile); a.slabs = 0; a.accumulate = accumulate;
  a.scale = scale;
  const bool vec = d % 4 == 0 && (((uintptr_t)dx & (type == IN_BF16 ? 7 : 15)) | ((uintptr_t)dE & 15)) == 0;
  if (type == IN_BF16) launch_tile_sum<bf16>(a, vec, st);
  else launch_tile_sum<float>(a, vec, st);
  if (a.tiles > 1) embed_join_kernel<<<dim3((unsigned)a.tiles, (unsigned)ceil_div(d, 256)), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace t5mi
