// Token embedding with a scale, and the gradient of its table by sorted tokens:
//   x[t, :] = scale * E[id_t, :],      dE[v, :] (+)= scale * sum over { t : id_t = v } of dx[t, :].
// Both are bound by bytes: the lookup moves 2 n d elements, the gradient reads n d elements and writes the table's
// float32 gradient once.  The gradient needs no atomics: positions are brought in the order of their ids (stable, so the
// positions of a row ascend), and every row of an id that occurs is written by the wavefronts that sum it.
// Measured on one MI355X (a copy moves 5.2 TB/s there, a fill 6.9), three sets of inputs in turn, bf16: lookup of 16384 rows
// of 768, 8.0 us (50 MB; a part of the table comes from the Infinity Cache); gradient of the same for 32128 rows, a
// seventh of the tokens padding, 40 to 43 us (124 MB, 24 us at a copy's rate); 32768 x 2048, 113 us (397 MB, 77 us).  Added to a
// gradient that is there, as the models do, for some 5900 and 10400 rows that occur: 37 us (61 MB, 12 us;
// 13 in the sort, which has no clearing beside it, 19 in the sums, 6 in the join) and 97 us (304 MB, 59 us; 19, 76 and 7).
#include "kernels.h"
#include <algorithm>

namespace t5mi {

namespace {

__device__ __forceinline__ uint32_t clamp_id(int32_t id, int vocab) {
  return (uint32_t)(id < 0 ? 0 : (id >= vocab ? vocab - 1 : id));
}

// N elements at an address that is a multiple of the element's size and need be of nothing more (the part loads and stores
// them whole, wherever they lie).
template <typename T, int N> struct Piece {
  typedef __attribute__((ext_vector_type(N))) T vec;
  typedef vec __attribute__((aligned(sizeof(T)))) type;
};
template <typename T> struct Piece<T, 1> { typedef T vec, type; };

// VEC columns of a row of d >= VEC, as many as end with the row where the lane's own would reach beyond it: then the first
// `shift` belong to the lane before and are read but not written.
struct Cols {
  int c, shift;
  bool on;
  __device__ __forceinline__ Cols(int at, int d, int vec) {
    on = at < d;
    c = on ? min(at, d - vec) : 0;
    shift = on ? at - c : 0;
  }
};
template <int VEC, typename F>
__device__ __forceinline__ void put_cols(float* o, const Cols& q, F v, bool add) {
  if constexpr (VEC == 1) {
    *o = add ? *o + v : v;
  } else if (q.shift == 0) {
    typedef typename Piece<float, VEC>::type P;
    *reinterpret_cast<P*>(o) = add ? *reinterpret_cast<P*>(o) + v : v;
  } else {
#pragma unroll
    for (int k = 1; k < VEC; ++k)
      if (k >= q.shift) o[k] = add ? o[k] + v[k] : v[k];
  }
}

// ------------------------------------------------------------------------------------------------
// Lookup, bound by bytes.  A workgroup takes rows_per_block consecutive tokens, their rows cut into 16-byte pieces of EPV
// elements, four pieces per thread in flight.  A row's last piece ends with the row: it may share elements with the one
// before, which then get the same values twice.
// ------------------------------------------------------------------------------------------------
template <typename T, int EPV>
__global__ __launch_bounds__(256) void embed_scaled_fwd_kernel(const int32_t* __restrict__ tok, const T* __restrict__ E,
                                                               T* __restrict__ x, int64_t n, int d, int vocab,
                                                               float scale, int rows_per_block) {
  typedef typename Piece<T, EPV>::type P;
  const uint32_t cpr = ((uint32_t)d + EPV - 1) / EPV;
  const int64_t r0 = (int64_t)blockIdx.x * rows_per_block;
  const uint32_t m = (uint32_t)(n - r0 < rows_per_block ? n - r0 : rows_per_block) * cpr;
  for (uint32_t t0 = threadIdx.x; t0 < m; t0 += 1024) {
    typename Piece<T, EPV>::vec v[4];
    uint32_t at[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t t = t0 + 256 * u;
      if (t >= m) break;
      const uint32_t r = t / cpr, c = min((t - r * cpr) * EPV, (uint32_t)d - EPV);
      at[u] = r * (uint32_t)d + c;
      v[u] = *reinterpret_cast<const P*>(E + (size_t)clamp_id(tok[r0 + r], vocab) * d + c);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (t0 + 256 * u >= m) break;
      if constexpr (EPV == 1) {
        v[u] = from_f32<T>(to_f32(v[u]) * scale);
      } else {
#pragma unroll
        for (int k = 0; k < EPV; ++k) v[u][k] = from_f32<T>(to_f32(v[u][k]) * scale);
      }
      *reinterpret_cast<P*>(x + (size_t)r0 * d + at[u]) = v[u];
    }
  }
}

// Clears out[0, count) with this launch's workgroups from `first` on, kFillEach floats each; the others sort meanwhile.
// (Sorting leaves most of the chip idle and the fill is nearly all that a sorting launch takes: 10.2 to 10.9 us for 66 MB.
// Clearing none but the rows that no token writes, in the launch of the sums, gained 2% of 32768 x 2048: not worth its code.)
constexpr int kFillEach = 1024 * 16;
struct Fill {
  float* out;
  int64_t count;
  int32_t first;
};
__device__ __forceinline__ void fill_zero(const Fill& f) {
  const int b = blockIdx.x - f.first;
  const int at = ((intptr_t)f.out >> 2) & 3;
  const int64_t pre = at && f.count > 4 - at ? 4 - at : at ? f.count : 0;  // elements in front of a 16-byte boundary
  const int64_t quads = (f.count - pre) / 4;
  f32x4* q = reinterpret_cast<f32x4*>(f.out + pre);
  const int64_t i0 = (int64_t)b * (kFillEach / 4);
  for (int j = threadIdx.x; j < kFillEach / 4; j += blockDim.x)
    if (i0 + j < quads) q[i0 + j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t tail = pre + 4 * quads;
  if (b == 0 && threadIdx.x < pre) f.out[threadIdx.x] = 0.f;
  if (b == 0 && threadIdx.x < f.count - tail) f.out[tail + threadIdx.x] = 0.f;
}

// ------------------------------------------------------------------------------------------------
// Stable sort of (id, position) by id: least significant digit first, `bits` bits a pass (at most 8, or at most 10 where
// that saves a pass), two launches a pass.  Workgroup b owns keys [b * chunk, (b + 1) * chunk) of the pass's input, 1024
// at a time.  (One launch less a pass, each counting the next one's digits as it places its keys, costs more than it
// saves where an id is frequent: atomics on few addresses, 36 -> 47 us with 30% padding among 40000.)
// ------------------------------------------------------------------------------------------------
constexpr int kSortTile = 1024;
constexpr int kSortBlocks = 256;  // at most; a workgroup then loops over its chunk

struct SortPass {
  const int32_t* tok;  // first pass: ids as given; else null
  const u32x2* in;     // (id, position), sorted by the lower digits
  u32x2* out;
  uint32_t* hist;      // [blocks][DIGITS]
  int32_t n, vocab, chunk, blocks, shift, bits;
  Fill fill;
};

__device__ __forceinline__ u32x2 sort_load(const SortPass& p, int i) {
  if (p.tok) return u32x2{clamp_id(p.tok[i], p.vocab), (uint32_t)i};
  return p.in[i];
}

template <int DIGITS>
__global__ __launch_bounds__(1024) void embed_sort_count_kernel(SortPass p) {
  __shared__ uint32_t cnt[DIGITS];
  if ((int)blockIdx.x >= p.blocks) {
    fill_zero(p.fill);
    return;
  }
  const int tid = threadIdx.x;
  if (tid < DIGITS) cnt[tid] = 0;
  __syncthreads();
  const int i0 = blockIdx.x * p.chunk, i1 = min(i0 + p.chunk, p.n);
  for (int i = i0 + tid; i < i1; i += 1024)
    atomicAdd(&cnt[(sort_load(p, i).x >> p.shift) & ((1u << p.bits) - 1)], 1u);  // whole numbers: the order does not matter
  __syncthreads();
  if (tid < DIGITS) p.hist[blockIdx.x * DIGITS + tid] = cnt[tid];
}

// base[d]: first place of digit d's keys of this workgroup = keys of smaller digits + keys of digit d of earlier
// workgroups.  Then 1024 keys at a time: each wavefront ranks its 64 among equal digits with ballots, the sixteen
// wavefronts' counts are joined, and every key goes to its place.
template <int DIGITS>
__global__ __launch_bounds__(1024) void embed_sort_place_kernel(SortPass p) {
  constexpr int kParts = 1024 / DIGITS;  // threads a digit
  __shared__ uint16_t cnt[16][DIGITS];
  __shared__ uint32_t base[DIGITS], all[kParts][DIGITS], before[kParts][DIGITS], wsum[DIGITS / 64];
  if ((int)blockIdx.x >= p.blocks) {
    fill_zero(p.fill);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, own = tid % DIGITS, part = tid / DIGITS;
  const uint32_t mask = (1u << p.bits) - 1;
  const int i0 = blockIdx.x * p.chunk, i1 = min(i0 + p.chunk, p.n);
  u32x2 key = i0 + tid < i1 ? sort_load(p, i0 + tid) : u32x2{0, 0};
  uint32_t total = 0, mine = 0;
  for (int b = part; b < p.blocks; b += 8 * kParts) {  // a share of the workgroups' counts each, eight in flight
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = b + kParts * j < p.blocks ? p.hist[(b + kParts * j) * DIGITS + own] : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      total += c[j];
      mine += b + kParts * j < (int)blockIdx.x ? c[j] : 0;
    }
  }
  all[part][own] = total;
  before[part][own] = mine;
  __syncthreads();
  uint32_t incl = 0;
  if (tid < DIGITS) {
    total = mine = 0;
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      total += all[q][tid];
      mine += before[q][tid];
    }
    incl = total;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t o = __shfl_up(incl, off, 64);
      incl += lane >= off ? o : 0;
    }
    if (lane == 63) wsum[w] = incl;
  }
  __syncthreads();
  if (tid < DIGITS) {
    uint32_t at = incl - total + mine;
    for (int q = 0; q < w; ++q) at += wsum[q];
    base[tid] = at;
  }
  for (int t0 = i0; t0 < i1; t0 += kSortTile) {
    const bool on = t0 + tid < i1;
    if (t0 > i0) key = on ? sort_load(p, t0 + tid) : u32x2{0, 0};
    const uint32_t d = (key.x >> p.shift) & mask;
    uint64_t same = __ballot(on);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const uint32_t below = (uint32_t)__popcll(same & ((1ull << lane) - 1));
#pragma unroll
    for (int i = 0; i < DIGITS / 64; ++i) cnt[w][i * 64 + lane] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (on && below == 0) cnt[w][d] = (uint16_t)__popcll(same);
    __syncthreads();
    uint32_t here = 0;  // of digit tid among these 1024 keys
    if (tid < DIGITS) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const uint32_t c = cnt[q][tid];
        cnt[q][tid] = (uint16_t)here;
        here += c;
      }
    }
    __syncthreads();
    if (on) p.out[base[d] + cnt[w][d] + below] = key;
    __syncthreads();
    if (tid < DIGITS) base[tid] += here;
  }
}

// ------------------------------------------------------------------------------------------------
// The same order in two launches, for n <= kMergeSort and id and position in 32 bits together: blocks of 1024 keys are
// sorted by a workgroup each, then the place of a key is its place in its block plus the number of smaller keys in every
// other block, found by bisection in LDS, which holds all keys.  768 columns, whole gradient: 5000 tokens 26.3 us against
// 33.2 by digits, 16384 39.8 against 44.1; beyond that the keys do not fit beside a second workgroup in LDS.
// ------------------------------------------------------------------------------------------------
constexpr int kMergeSort = 16384;
// (the clearing workgroups hold those 64 KB too: with 256 threads they leave the chip half empty, 8192 x 768 31.1 us against 29.7)
constexpr int kMergeThreads = 512;

__global__ __launch_bounds__(1024) void embed_sort_block_kernel(const int32_t* __restrict__ tok, uint32_t* __restrict__ out,
                                                                int n, int vocab, int pos_bits, int passes, int bits,
                                                                Fill fill) {
  __shared__ uint32_t cnt[16][256], base[256], wsum[4], keys[1024];
  if ((int)blockIdx.x >= fill.first) {
    fill_zero(fill);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, i = blockIdx.x * 1024 + tid;
  uint32_t key = i < n ? clamp_id(tok[i], vocab) << pos_bits | (uint32_t)i : 0xFFFFFFFFu;  // (the last block's end stays last)
  for (int q = 0; q < passes; ++q) {
    const uint32_t d = (key >> (pos_bits + q * bits)) & ((1u << bits) - 1);
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const uint64_t m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const uint32_t below = (uint32_t)__popcll(same & ((1ull << lane) - 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) cnt[w][j * 64 + lane] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (below == 0) cnt[w][d] = (uint32_t)__popcll(same);
    __syncthreads();
    uint32_t total = 0, incl = 0;
    if (tid < 256) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const uint32_t c = cnt[j][tid];
        cnt[j][tid] = total;
        total += c;
      }
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
      uint32_t at = incl - total;
      for (int j = 0; j < w; ++j) at += wsum[j];
      base[tid] = at;
    }
    __syncthreads();
    keys[base[d] + cnt[w][d] + below] = key;
    __syncthreads();
    key = keys[tid];
  }
  out[i] = key;
}

__global__ __launch_bounds__(kMergeThreads) void embed_sort_merge_kernel(const u32x4* __restrict__ in, u32x2* __restrict__ out, int n,
                                                               int pos_bits, Fill fill) {
  __shared__ uint32_t keys[kMergeSort];
  if ((int)blockIdx.x >= fill.first) {
    fill_zero(fill);
    return;
  }
  const int tid = threadIdx.x, blocks = (n + 1023) / 1024;
  for (int j = tid; j < blocks * 256; j += kMergeThreads) reinterpret_cast<u32x4*>(keys)[j] = in[j];
  __syncthreads();
  const int i = blockIdx.x * kMergeThreads + tid;
  if (i >= n) return;
  const uint32_t mine = keys[i];
  uint32_t place = i & 1023;
#pragma unroll 4
  for (int b = 0; b < blocks; ++b) {
    const uint32_t* k = keys + b * 1024;
    uint32_t lo = 0;
#pragma unroll
    for (int step = 512; step > 0; step >>= 1) lo += k[lo + step - 1] < mine ? step : 0;
    lo += k[lo] < mine ? 1 : 0;  // (lo <= 1023)
    place += b == i >> 10 ? 0 : lo;
  }
  out[place] = u32x2{mine >> pos_bits, mine & ((1u << pos_bits) - 1)};
}

// ------------------------------------------------------------------------------------------------
// Sums over the sorted positions, cut into tiles of `tile` positions however long the runs of equal ids are, so that a
// padding id with half of all positions costs no more than any other.  A wavefront takes a tile, VEC columns a lane and
// sixteen rows in flight.  Bound by bytes and by the dirty lines that the fill before it leaves to be written back: 14.4 us
// for 16384 x 768, bf16, 64 us for 32768 x 2048 (135 MB read, 87 MB written, 3.5 TB/s).  (16384 x 768: 40.7 us in all, 42.2
// with eight rows in flight.)  Rows of fewer than 64 pieces leave lanes idle; two or four tiles a wavefront, which no longer walks
// its runs together, cost more (32768 x 64: 27.0 us against 25.2).  A run inside its tile is written to its row at once;
// the part of a run that reaches over an end of the tile goes to partial[tile][slot], slot 0 if it is the tile's first run,
// else 1, and is joined afterwards.
// ------------------------------------------------------------------------------------------------
struct SumArgs {
  const u32x2* sorted;
  const void* dx;
  float* dE;
  float* partial;  // [tiles][2][d]
  int32_t n, d, tile, tiles, slabs, join, accumulate;
  float scale;
};

template <typename T, int VEC>
__global__ __launch_bounds__(256) void embed_tile_sum_kernel(SumArgs a) {
  constexpr int NB = 16;  // rows in flight
  typedef typename Piece<T, VEC>::type P;
  typedef typename Piece<float, VEC>::vec F;
  const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int t = unit / a.slabs;
  if (t >= a.tiles) return;
  const Cols q(((unit - t * a.slabs) * 64 + threadIdx.x % 64) * VEC, a.d, VEC);
  const T* dx = (const T*)a.dx + q.c;
  const int t0 = t * a.tile, t1 = min(t0 + a.tile, a.n);
  uint32_t cur = a.sorted[t0].x;
  const bool from_before = t0 > 0 && a.sorted[t0 - 1].x == cur;
  bool first = true;
  F acc{};
  auto flush = [&](bool part) {
    if (!q.on) return;
    float* o = part ? a.partial + ((size_t)t * 2 + (first ? 0 : 1)) * a.d : a.dE + (size_t)cur * a.d;
    put_cols<VEC, F>(o + q.c, q, acc * a.scale, a.accumulate && !part);
  };
  for (int i = t0; i < t1; i += NB) {
    u32x2 s[NB];
    typename Piece<T, VEC>::vec v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) s[j] = a.sorted[min(i + j, t1 - 1)];
#pragma unroll
    for (int j = 0; j < NB; ++j) v[j] = *reinterpret_cast<const P*>(dx + (size_t)s[j].y * a.d);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (i + j < t1) {
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
  }
  flush((first && from_before) || (t1 < a.n && a.sorted[t1].x == cur));
}

// A workgroup per tile and `join` pieces of 64 * VEC columns: if a run begins in the tile and reaches over its end, adds
// the run's parts and writes the row.  5.6 us at 16384 x 768, mostly dependent loads.  The eight wavefronts take a piece
// each, or a share of a piece's parts, in order.
template <int VEC>
__global__ __launch_bounds__(512) void embed_join_kernel(SumArgs a) {
  typedef typename Piece<float, VEC>::type P;
  typedef typename Piece<float, VEC>::vec F;
  __shared__ F red[8][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int t = blockIdx.x, t0 = t * a.tile, t1 = min(t0 + a.tile, a.n);
  auto id_at = [&](int64_t i) { return a.sorted[i < a.n ? i : a.n - 1].x; };
  // (all of these loads are in flight together)
  const uint32_t last = id_at(t1 - 1), next = id_at(t1), head = id_at(t0), prev = id_at(t0 > 0 ? t0 - 1 : 0);
  uint32_t begin = id_at((int64_t)t1 + (int64_t)lane * a.tile);  // of tile t + 1 + lane
  if (t1 >= a.n || next != last) return;
  const bool whole = head == last;
  if (whole && t0 > 0 && prev == last) return;  // the run begins earlier
  // parts of the run: part 0 here, part i in tile t + i for as long as tiles begin with its id
  int parts = 1;
  for (int64_t first = t1;;) {
    const uint64_t same = __ballot(first + (int64_t)lane * a.tile < a.n && begin == last);
    parts += __popcll(same);
    if (~same) break;
    first += 64 * (int64_t)a.tile;
    begin = id_at(first + (int64_t)lane * a.tile);
  }
  const int slabs = min(a.join, a.slabs - (int)blockIdx.y * a.join);
  const int shares = slabs == 1 ? 8 : slabs == 2 ? 4 : 2;
  const int slab = w / shares, each = (parts + shares - 1) / shares, p0 = (w % shares) * each, p1 = min(p0 + each, parts);
  const Cols cols(((blockIdx.y * a.join + slab) * 64 + lane) * VEC, a.d, VEC);
  const bool on = slab < slabs && cols.on;
  const float* src = a.partial + (size_t)t * 2 * a.d + cols.c;
  F s{};
  for (int p = p0; p < p1; p += 8) {
    F v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int q = min(p + j, p1 - 1);
      v[j] = *reinterpret_cast<const P*>(src + (size_t)(2 * q + (q == 0 && !whole ? 1 : 0)) * a.d);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (p + j < p1) s += v[j];
  }
  red[w][lane] = s;
  __syncthreads();
  if (w % shares != 0 || !on) return;
  for (int q = 1; q < shares && q * each < parts; ++q) s += red[w + q][lane];
  put_cols<VEC, F>(a.dE + (size_t)last * a.d + cols.c, cols, s, a.accumulate);
}

// ------------------------------------------------------------------------------------------------
// Few tokens: one launch and no sort, bound by latency (777 tokens, half of them one id, 509 x 67 in float32: 6.9 us; 2000
// x 768 in bf16 with a table of 8000 rows: 10.8 us against 18.7 by sorting).  A wavefront per position looks for its id
// among all ids, held in LDS; if the position is the first of its id it sums the rows of all of them in order.  Ids that
// occur more than kOwnerAlone times are left to the whole workgroup, which shares their list out (1624 x 960, float32: 8.8
// us, 9.4 with a bound of 24).  `splits` workgroups of every eight positions take a part of the columns each.  Behind
// these, workgroups that clear `zero_rows` rows of the table each, all but those whose ids they find.
// ------------------------------------------------------------------------------------------------
constexpr int kOwnerTokens = 4096, kOwnerAlone = 48, kZeroRows = 512;

struct OwnerArgs {
  const int32_t* tok;
  const void* dx;
  float* dE;
  int32_t n, d, vocab, zero_rows, accumulate, sum_blocks, splits, split_cols;
  float scale;
};

// Sum over list[l0, l1) of the rows' VEC columns at dx, eight in flight.
template <typename T, int VEC, typename F>
__device__ __forceinline__ F sum_listed(const T* dx, int d, const uint16_t* list, int l0, int l1) {
  typedef typename Piece<T, VEC>::type P;
  F acc{};
  for (int l = l0; l < l1; l += 8) {
    typename Piece<T, VEC>::vec x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const P*>(dx + (size_t)list[min(l + j, l1 - 1)] * d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool in = l + j < l1;
      if constexpr (VEC == 1) {
        acc += in ? to_f32(x[j]) : 0.f;
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += in ? to_f32(x[j][k]) : 0.f;
      }
    }
  }
  return acc;
}

template <typename F>
__device__ __forceinline__ F add_lanes(F s, int off) {  // the lane's and that of lane ^ off
  if constexpr (sizeof(F) == 4) {
    s += __shfl_xor(s, off, 64);
  } else {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(F) / 4); ++k) s[k] += __shfl_xor(s[k], off, 64);
  }
  return s;
}

template <typename T, int VEC>
__global__ __launch_bounds__(512) void embed_owner_sum_kernel(OwnerArgs a) {
  typedef typename Piece<float, VEC>::vec F;
  __shared__ uint32_t ids[kOwnerTokens];
  __shared__ uint16_t list[kOwnerTokens], few[8][kOwnerAlone];
  __shared__ F red[8][64];
  __shared__ uint32_t many[8], n_many;
  __shared__ int found[8];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t lower = (1ull << lane) - 1;
  const int pieces = (min(a.split_cols, a.d) + VEC - 1) / VEC, width = pieces > 32 ? 64 : pieces > 16 ? 32 : pieces > 8 ? 16 : 8;
  uint32_t id[kOwnerTokens / 512];
#pragma unroll
  for (int k = 0; k < kOwnerTokens / 512; ++k) id[k] = k * 512 + tid < a.n ? clamp_id(a.tok[k * 512 + tid], a.vocab) : ~0u;
  if ((int)blockIdx.x >= a.sum_blocks) {
    __shared__ uint8_t seen[kZeroRows];
    const uint32_t v0 = (uint32_t)(blockIdx.x - a.sum_blocks) * a.zero_rows;
    seen[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kOwnerTokens / 512; ++k)
      if (id[k] - v0 < (uint32_t)a.zero_rows) seen[id[k] - v0] = 1;
    __syncthreads();
    for (int r = w; r < a.zero_rows && v0 + r < (uint32_t)a.vocab; r += 8) {
      if (seen[r]) continue;
      float* o = a.dE + (size_t)(v0 + r) * a.d;
      for (int c = lane * VEC; c < a.d; c += 64 * VEC) {
        const Cols q(c, a.d, VEC);
        put_cols<VEC, F>(o + q.c, q, F{}, false);
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kOwnerTokens / 512; ++k) ids[k * 512 + tid] = id[k];
  if (tid == 0) n_many = 0;
  __syncthreads();
  auto put = [&](uint32_t v, const Cols& q, F s) { put_cols<VEC, F>(a.dE + (size_t)v * a.d + q.c, q, s * a.scale, a.accumulate); };
  const int split = blockIdx.x % a.splits, own = blockIdx.x / a.splits * 8 + w;
  const int c_begin = split * a.split_cols, c_end = min(c_begin + a.split_cols, a.d);
  if (own < a.n) {
    const uint32_t v = ids[own];
    // 256 ids at a time (places behind the last id hold none): first those in front of the position, then all behind
    const int start = own & ~255;
    bool first = true;
    int m = 0;
    uint64_t hit[4];
    auto look = [&](int k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) hit[j] = __ballot(ids[k + j * 64 + lane] == v);
    };
    for (int k = 0; k < start && first; k += 256) {
      look(k);
      first = !(hit[0] | hit[1] | hit[2] | hit[3]);
    }
    for (int k = start; k < a.n && first; k += 256) {
      look(k);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (hit[j]) {
          const int i = k + j * 64, at = m + __popcll(hit[j] & lower);
          if ((hit[j] >> lane & 1) && at < kOwnerAlone) few[w][at] = (uint16_t)(i + lane);
          if (m == 0 && i + __ffsll((long long)hit[j]) - 1 < own) first = false;
          m += __popcll(hit[j]);
        }
      }
    }
    if (first && m > kOwnerAlone) {
      if (lane == 0) many[atomicAdd(&n_many, 1u)] = v;
    } else if (first) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      // `width` lanes a row; where that leaves lanes, each group of them takes a share of the list
      const int groups = 64 / width, each = (m + groups - 1) / groups, l0 = lane / width * each, l1 = min(l0 + each, m);
      for (int c = c_begin + lane % width * VEC; c < c_end; c += 64 * VEC) {
        const Cols q(c, a.d, VEC);
        F s = sum_listed<T, VEC, F>((const T*)a.dx + q.c, a.d, few[w], l0, l1);
        for (int off = width; off < 64; off <<= 1) s = add_lanes(s, off);
        if (lane < width) put(v, q, s);
      }
    }
  }
  __syncthreads();
  for (uint32_t h = 0; h < n_many; ++h) {
    const uint32_t v = many[h];
    // the list, each wavefront an eighth of the ids
    uint64_t hit[kOwnerTokens / 512];
    int here = 0, mine = 0, m = 0;
#pragma unroll
    for (int k = 0; k < kOwnerTokens / 512; ++k) {
      hit[k] = __ballot(ids[w * (kOwnerTokens / 8) + k * 64 + lane] == v);
      here += __popcll(hit[k]);
    }
    if (lane == 0) found[w] = here;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      mine += q < w ? found[q] : 0;
      m += found[q];
    }
#pragma unroll
    for (int k = 0; k < kOwnerTokens / 512; ++k) {
      if (hit[k] >> lane & 1) list[mine + __popcll(hit[k] & lower)] = (uint16_t)(w * (kOwnerTokens / 8) + k * 64 + lane);
      mine += __popcll(hit[k]);
    }
    __syncthreads();
    const int shares = 8 * (64 / width), share = (w * 64 + lane) / width, each = (m + shares - 1) / shares;
    const int l0 = share * each, l1 = min(l0 + each, m);
    for (int c0 = c_begin; c0 < c_end; c0 += 64 * VEC) {
      const Cols q(c0 + lane % width * VEC, c_end, VEC);  // (a part ends with the row, or with whole pieces)
      red[w][lane] = sum_listed<T, VEC, F>((const T*)a.dx + q.c, a.d, list, l0, l1);
      __syncthreads();
      if (tid < width && q.on) {
        const F* part = &red[0][0] + tid;  // of share j: part[j * width]
        F s = part[0];
        for (int j = 1; j < shares && j * each < m; ++j) s += part[j * width];
        put(v, q, s);
      }
      __syncthreads();
    }
  }
}

// Columns that a workgroup of the kernel above takes: as many parts as leave about two thousand workgroups.
int owner_cols(int64_t n, int d) {
  const int piece = d >= 4 ? 256 : 64, pieces = ceil_div(d, piece), groups = std::max(1, ceil_div(n, 8));
  return ceil_div(pieces, std::max(1, std::min(pieces, 2048 / groups))) * piece;
}
// All rows of an id that occurs often go through one compute unit a part: up to 2^19 elements of them (2000 x 768, 40%
// padding: 17.1 us against 18.7 by sorting; 4000 x 768: 27.3 against 21.3, and 18.1 against 20.5 without padding).
bool owner_takes(int64_t n, int d) { return n <= kOwnerTokens && n * std::min(owner_cols(n, d), d) <= 1 << 19; }

struct SortPlan {
  int bits_each, passes, digits, blocks, chunk;
  int pos_bits;  // > 0: blocks and a merge
};
int bits_of(int64_t v) {  // of the numbers 0 .. v, at least 1
  int b = 1;
  while (v >> b) ++b;
  return b;
}
SortPlan sort_plan(int64_t n, int vocab) {
  SortPlan s;
  const int bits = bits_of(vocab - 1), pos_bits = bits_of(std::max<int64_t>(n - 1, 0));
  s.pos_bits = n <= kMergeSort && bits + pos_bits <= 32 ? pos_bits : 0;
  // ten bits a pass where that saves one, as long as the workgroups' counts of 1024 digits are few (29103 x 149, 327 ids: 29.7 us
  // against 34.0; 32768 x 128, 100000 ids: 38.2 and 39.3; but 200000 x 64: 78.5 and 67.8)
  s.digits = n <= 65536 && ceil_div(bits, 10) < ceil_div(bits, 8) ? 1024 : 256;
  s.passes = ceil_div(bits, s.pos_bits || s.digits == 256 ? 8 : 10);
  s.bits_each = ceil_div(bits, s.passes);
  s.chunk = std::max(1, ceil_div(n, (int64_t)kSortBlocks * kSortTile)) * kSortTile;
  s.blocks = ceil_div(n, s.chunk);
  return s;
}
// Positions of a tile: as many as leave 1024 wavefronts and more, up to 64 (60000 x 512: 54 us with 32, 51 with 64)
int sum_tile(int64_t n, int d) {
  const int64_t slabs = ceil_div(d, 256);
  int t = 64;
  while (t > 16 && ceil_div(n, t) * slabs < 1024) t /= 2;
  return t;
}

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
  w->buf[1] = (u32x2*)take((size_t)std::max<int64_t>(n, 1024) * sizeof(u32x2));
  w->hist = (uint32_t*)take(s.pos_bits ? 0 : (size_t)s.blocks * s.digits * 4);
  w->partial = (float*)take((size_t)ceil_div(n, sum_tile(n, d)) * 2 * d * 4);
  return off;
}

template <typename T>
void launch_tile_sum(const SumArgs& a, bool vec, hipStream_t st) {
  const unsigned grid = (unsigned)ceil_div((int64_t)a.tiles * a.slabs, 4);
  if (vec) embed_tile_sum_kernel<T, 4><<<grid, 256, 0, st>>>(a);
  else embed_tile_sum_kernel<T, 1><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t launch_embed_scaled_fwd(const int32_t* tokens, const void* E, void* x, int type, int64_t n, int d, int vocab,
                                   float scale, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int epv = type == IN_BF16 ? 8 : 4;
  const bool whole = d >= epv;
  const int rpb = std::max(1, 1024 / (whole ? ceil_div(d, epv) : d));
  const unsigned grid = (unsigned)ceil_div(n, rpb);
  if (type == IN_BF16) {
    if (whole) embed_scaled_fwd_kernel<bf16, 8><<<grid, 256, 0, st>>>(tokens, (const bf16*)E, (bf16*)x, n, d, vocab, scale, rpb);
    else embed_scaled_fwd_kernel<bf16, 1><<<grid, 256, 0, st>>>(tokens, (const bf16*)E, (bf16*)x, n, d, vocab, scale, rpb);
  } else {
    if (whole) embed_scaled_fwd_kernel<float, 4><<<grid, 256, 0, st>>>(tokens, (const float*)E, (float*)x, n, d, vocab, scale, rpb);
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
  const bool vec = d >= 4;
  if (owner_takes(n, d)) {
    OwnerArgs a;
    a.tok = tokens; a.dx = dx; a.dE = dE; a.n = (int)n; a.d = d; a.vocab = vocab; a.accumulate = accumulate; a.scale = scale;
    // rows that one workgroup clears: 128 KB at most, fewer where the table leaves compute units idle (777 tokens, 509 x 67:
    // 12.3 us with 128 KB each, 6.8 with 32 rows)
    a.zero_rows = std::max(1, std::min({kZeroRows, 32768 / d, std::max(32, ceil_div(vocab, 512))}));
    a.split_cols = owner_cols(n, d);
    a.splits = ceil_div(d, a.split_cols);
    a.sum_blocks = ceil_div(n, 8) * a.splits;
    const unsigned grid = (unsigned)(a.sum_blocks + (accumulate ? 0 : ceil_div(vocab, a.zero_rows)));
    if (type == IN_BF16) {
      if (vec) embed_owner_sum_kernel<bf16, 4><<<grid, 512, 0, st>>>(a);
      else embed_owner_sum_kernel<bf16, 1><<<grid, 512, 0, st>>>(a);
    } else {
      if (vec) embed_owner_sum_kernel<float, 4><<<grid, 512, 0, st>>>(a);
      else embed_owner_sum_kernel<float, 1><<<grid, 512, 0, st>>>(a);
    }
    return hipGetLastError();
  }
  const SortPlan s = sort_plan(n, vocab);
  BwdWs w;
  carve_bwd_ws(n, vocab, d, ws, &w);
  // rows of ids that do not occur: the whole table's gradient is cleared beside the sort, which leaves most of the
  // chip idle, in equal shares of its launches
  const int launches = s.pos_bits ? 2 : 2 * s.passes;
  const int64_t all = accumulate ? 0 : (int64_t)vocab * d, share = ((all + launches - 1) / launches + 3) / 4 * 4;
  const u32x2* sorted = w.buf[0];
  SortPass p;
  p.hist = w.hist;
  p.n = (int)n; p.vocab = vocab; p.chunk = s.chunk; p.blocks = s.blocks; p.bits = s.bits_each;
  int turn = 0;
  auto blocks = [&](int sorters) {  // of the next launch, its share of the clearing among them
    const int64_t i0 = std::min(all, share * turn), i1 = std::min(all, share * (turn + 1));
    ++turn;
    p.fill.out = dE + i0; p.fill.count = i1 - i0; p.fill.first = sorters;
    return (unsigned)(sorters + ceil_div(p.fill.count, kFillEach));
  };
  if (s.pos_bits) {
    unsigned grid = blocks(s.blocks);
    embed_sort_block_kernel<<<grid, 1024, 0, st>>>(tokens, (uint32_t*)w.buf[1], (int)n, vocab, s.pos_bits, s.passes, s.bits_each, p.fill);
    grid = blocks(ceil_div(n, kMergeThreads));
    embed_sort_merge_kernel<<<grid, kMergeThreads, 0, st>>>((const u32x4*)w.buf[1], w.buf[0], (int)n, s.pos_bits, p.fill);
  }
  for (int q = 0; q < s.passes && !s.pos_bits; ++q) {
    p.tok = q == 0 ? tokens : nullptr;
    p.in = w.buf[(q + 1) & 1];
    p.out = w.buf[q & 1];
    p.shift = q * s.bits_each;
    if (s.digits == 1024) {
      embed_sort_count_kernel<1024><<<blocks(s.blocks), 1024, 0, st>>>(p);
      embed_sort_place_kernel<1024><<<blocks(s.blocks), 1024, 0, st>>>(p);
    } else {
      embed_sort_count_kernel<256><<<blocks(s.blocks), 1024, 0, st>>>(p);
      embed_sort_place_kernel<256><<<blocks(s.blocks), 1024, 0, st>>>(p);
    }
    sorted = p.out;
  }
  SumArgs a;
  a.sorted = sorted; a.dx = dx; a.dE = dE; a.partial = w.partial;
  a.n = (int)n; a.d = d; a.tile = sum_tile(n, d); a.tiles = ceil_div(n, a.tile); a.slabs = ceil_div(d, vec ? 256 : 64);
  a.accumulate = accumulate;
  a.scale = scale;
  if (type == IN_BF16) launch_tile_sum<bf16>(a, vec, st);
  else launch_tile_sum<float>(a, vec, st);
  if (a.tiles > 1) {
    // most workgroups have nothing to do and cost 0.3 ns a wavefront: four pieces each where there are more than four
    // (32768 x 2048: 111.5 us in all with one piece, 109.3 with four; 16384 x 768, a seventh of it padding: 39.0 and 41.1)
    a.join = a.slabs > 4 ? 4 : 1;
    const dim3 grid((unsigned)a.tiles, (unsigned)ceil_div(a.slabs, a.join));
    if (vec) embed_join_kernel<4><<<grid, 512, 0, st>>>(a);
    else embed_join_kernel<1><<<grid, 512, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace t5mi
