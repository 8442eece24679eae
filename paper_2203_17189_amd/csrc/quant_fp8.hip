// Quantisation of a matrix to 8-bit floating point in blocks of 128, by rows and transposed (see include/t5mi.h).
//
// Per block: e from the largest |x|, code = x 2^-e rounded to nearest even.  Everything is bound by memory: x is read once,
// whatever is asked for, and each code is written once.
//   rows alone, blocks of one row: 16 lanes hold a block, 8 values each; no lane waits for another workgroup or for LDS.
//   transposed, or blocks of 128 x 128: a workgroup holds a 128 x 128 tile in registers, 8 x 4 values a thread; row maxima
//   within 16 lanes, column maxima through LDS; the transposed codes go through LDS, 4 rows of a column at a time, so that
//   both matrices are written in rows of 128 bytes.
#include "fp8.h"
#include "kernels.h"

namespace t5mi {
namespace {

struct QuantArgs {
  const void* x;
  uint8_t *q, *scale, *qt, *scale_t;
  int64_t rows, ld;
  int cols;
  int64_t ldq, ldqt, lds_t;  // bytes between rows of q, of qt, of scale_t
  int kb, kbp;               // blocks of a row, and bytes between rows of scale
};

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {  // of both halves
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Eight neighbours of a row as words: two bfloat16 in each, or one float32.  Sizes |x| are whole numbers, ordered as the
// values are: both halves of a word, or all of it.
template <typename T> struct Eight;
template <> struct Eight<bf16> {
  static constexpr int W = 4;  // words
  static constexpr uint32_t MASK = 0x7FFF7FFFu;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max2(a, b); }
  static __device__ __forceinline__ uint32_t finite(uint32_t s) {
    return ((s & 0xFFFFu) < 0x7F80u ? s & 0xFFFFu : 0u) | (s < 0x7F800000u ? s & 0xFFFF0000u : 0u);
  }
  static __device__ __forceinline__ bool odd(uint32_t s) { return (s & 0xFFFFu) >= 0x7F80u || s >= 0x7F800000u; }
};
template <> struct Eight<float> {
  static constexpr int W = 8;
  static constexpr uint32_t MASK = 0x7FFFFFFFu;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ uint32_t finite(uint32_t s) { return s < 0x7F800000u ? s : 0u; }
  static __device__ __forceinline__ bool odd(uint32_t s) { return s >= 0x7F800000u; }
};

// Elements [c, c + 8) of a row, zeros from `cols` on.  more: rows follow, so that the end of a piece past `cols` is memory of
// the matrix too, and may be read (and is dropped).
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int cols, bool more, uint32_t (&v)[Eight<T>::W]) {
  if (VEC && quant_whole_piece(c, cols, more)) {
#pragma unroll
    for (int h = 0; h < Eight<T>::W / 4; ++h) {
      const u32x4 p = *reinterpret_cast<const u32x4*>(row + c + h * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[h * 4 + j] = p[j];
    }
    if (c + 8 > cols) {
#pragma unroll
      for (int j = 0; j < Eight<T>::W; ++j) {
        const int k = c + j * (8 / Eight<T>::W);
        v[j] = k >= cols ? 0u : sizeof(T) == 2 && k + 1 >= cols ? v[j] & 0xFFFFu : v[j];
      }
    }
  } else if constexpr (sizeof(T) == 2) {
    const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = (c + 2 * j < cols ? r[c + 2 * j] : 0u) | (c + 2 * j + 1 < cols ? (uint32_t)r[c + 2 * j + 1] << 16 : 0u);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? __float_as_uint(row[c + j]) : 0u;
  }
}

template <typename T, int Q>
__device__ __forceinline__ u32x2 codes8(const uint32_t (&v)[Eight<T>::W], float scale) {
  if constexpr (sizeof(T) == 2) return u32x2{pack_fp8x4<Q>(v[0], v[1], scale), pack_fp8x4<Q>(v[2], v[3], scale)};
  else
    return u32x2{pack_fp8x4<Q>(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]), scale),
                 pack_fp8x4<Q>(__uint_as_float(v[4]), __uint_as_float(v[5]), __uint_as_float(v[6]), __uint_as_float(v[7]), scale)};
}
// The larger half of a word of sizes as the bits of a float32.
template <typename T>
__device__ __forceinline__ uint32_t size_bits(uint32_t s) {
  if constexpr (sizeof(T) == 2) return max(s << 16, s & 0xFFFF0000u);
  else return s;
}

constexpr int kUnits = 2;  // blocks that 16 lanes hold at once

// Units are (row, block) pairs, kbp of them in a row: those past the row's blocks write the zeros behind its scales.
template <typename T, int Q, bool VEC>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a) {
  typedef Eight<T> E;
  const int64_t first = (int64_t)blockIdx.x * (16 * kUnits);
  const int64_t row0 = first / a.kbp;
  const uint32_t rem0 = (uint32_t)(first - row0 * a.kbp);
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  uint32_t v[kUnits][E::W];
  int64_t row[kUnits];
  int b[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint32_t at = rem0 + u * 16 + g;
    row[u] = row0 + at / (uint32_t)a.kbp;
    b[u] = (int)(at % (uint32_t)a.kbp);
    if (row[u] < a.rows) load8<T, VEC>((const T*)a.x + row[u] * a.ld, b[u] * kBlock + l * 8, a.cols, row[u] + 1 < a.rows, v[u]);
    else
#pragma unroll
      for (int j = 0; j < E::W; ++j) v[u][j] = 0;
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < E::W; ++j) m = E::larger(m, v[u][j] & E::MASK);
    if (E::odd(m)) {
      m = 0;
#pragma unroll
      for (int j = 0; j < E::W; ++j) m = E::larger(m, E::finite(v[u][j] & E::MASK));
    }
    const int e = block_exponent<Q>(max16(size_bits<T>(m)));
    if (row[u] >= a.rows) continue;
    const int c = b[u] * kBlock + l * 8;
    if (c < a.ldq) *reinterpret_cast<u32x2*>(a.q + row[u] * a.ldq + c) = codes8<T, Q>(v[u], scale_of(e));
    if (l == 0) a.scale[row[u] * a.kbp + b[u]] = b[u] < a.kb ? (uint8_t)(e + 127) : 0;
  }
}

// SQUARE: one scale for the tile; else one for each of its rows (q) and columns (qt).
template <typename T, int Q, bool VEC, bool SQUARE>
__global__ __launch_bounds__(512) void quant_tile_kernel(QuantArgs a) {
  typedef Eight<T> E;
  constexpr int W = E::W;
  __shared__ __align__(16) uint8_t turned[128 * 128];  // [column][row], words of 4 rows swizzled by the column's group
  __shared__ uint32_t part[8][16][W];                  // column sizes of each wavefront
  __shared__ __align__(16) float column_scale[128];
  const int kb = blockIdx.x % a.kb;
  const int64_t rb = blockIdx.x / a.kb;
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
  const int c0 = kb * kBlock + cg * 8;
  const int64_t r0 = rb * kBlock + rg * 4;
  uint32_t v[4][W];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (r0 + i < a.rows) load8<T, VEC>((const T*)a.x + (r0 + i) * a.ld, c0, a.cols, r0 + i + 1 < a.rows, v[i]);
    else
#pragma unroll
      for (int j = 0; j < W; ++j) v[i][j] = 0;
  }
  uint32_t rows[4], cols[W];  // largest sizes of the thread's rows and columns
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    rows[i] = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const uint32_t s = v[i][j] & E::MASK;
      rows[i] = E::larger(rows[i], s);
      cols[j] = i ? E::larger(cols[j], s) : s;
    }
  }
  uint32_t all = 0;
#pragma unroll
  for (int j = 0; j < W; ++j) all = E::larger(all, cols[j]);
  if (E::odd(all)) {  // something is not finite: it does not count
    all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      rows[i] = 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const uint32_t s = E::finite(v[i][j] & E::MASK);
        rows[i] = E::larger(rows[i], s);
        cols[j] = i ? E::larger(cols[j], s) : s;
      }
      all = E::larger(all, rows[i]);
    }
  }
  int e = 0;  // SQUARE: the tile's exponent
  if constexpr (SQUARE) {
    uint32_t m = max16(size_bits<T>(all));
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    if ((t & 63) == 0) part[wave][0][0] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, part[w][0][0]);
    e = block_exponent<Q>(m);
  } else if (a.qt) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      uint32_t m = cols[j];
      m = E::larger(m, (uint32_t)__shfl_xor((int)m, 16, 64));
      m = E::larger(m, (uint32_t)__shfl_xor((int)m, 32, 64));
      if ((t & 48) == 0) part[wave][cg][j] = m;
    }
  }
  if (a.q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (!SQUARE) e = block_exponent<Q>(max16(size_bits<T>(rows[i])));
      if (r0 + i < a.rows) {
        if (c0 < a.ldq) __builtin_nontemporal_store(codes8<T, Q>(v[i], scale_of(e)), reinterpret_cast<u32x2*>(a.q + (r0 + i) * a.ldq + c0));
        if (!SQUARE && cg == 0) a.scale[(r0 + i) * a.kbp + kb] = (uint8_t)(e + 127);
        if (!SQUARE && kb == a.kb - 1 && cg > 0 && kb + cg < a.kbp) a.scale[(r0 + i) * a.kbp + kb + cg] = 0;
      }
    }
    if (SQUARE && t < 4) {
      if (t == 0) a.scale[rb * a.kbp + kb] = (uint8_t)(e + 127);
      else if (kb == a.kb - 1 && kb + t < a.kbp) a.scale[rb * a.kbp + kb + t] = 0;
    }
  }
  if (!a.qt) return;
  const int64_t rbs = (a.rows + kBlock - 1) / kBlock;
  float by[8];  // scales of the thread's columns
  if constexpr (SQUARE) {
#pragma unroll
    for (int k = 0; k < 8; ++k) by[k] = scale_of(e);
  } else {
    // One thread for each column: every thread for its own eight took 64 reads of LDS (5120 x 1024 float32 11.1 us, like this 8.3).
    __syncthreads();
    if (t < 128) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = E::larger(m, part[w][t >> 3][(t & 7) / (8 / W)]);
      e = block_exponent<Q>(sizeof(T) == 4 ? m : t & 1 ? m & 0xFFFF0000u : m << 16);
      column_scale[t] = scale_of(e);
      if (kb * kBlock + t < a.cols) {
        uint8_t* to = a.scale_t + (int64_t)(kb * kBlock + t) * a.lds_t;
        to[rb] = (uint8_t)(e + 127);
        if (rb == rbs - 1)
          for (int64_t r = rb + 1; r < a.lds_t; ++r) to[r] = 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) by[k] = column_scale[cg * 8 + k];
  }
#pragma unroll
  for (int j = 0; j < W; ++j) {
#pragma unroll
    for (int h = 0; h < 8 / W; ++h) {  // a word's columns
      const int k = j * (8 / W) + h, c = cg * 8 + k;
      uint32_t four;  // the column's four rows
      if constexpr (sizeof(T) == 2) {
        const uint32_t pick = h ? 0x07060302u : 0x05040100u;
        four = pack_fp8x4<Q>(__builtin_amdgcn_perm(v[1][j], v[0][j], pick), __builtin_amdgcn_perm(v[3][j], v[2][j], pick), by[k]);
      } else {
        four = pack_fp8x4<Q>(__uint_as_float(v[0][j]), __uint_as_float(v[1][j]), __uint_as_float(v[2][j]), __uint_as_float(v[3][j]), by[k]);
      }
      *reinterpret_cast<uint32_t*>(turned + c * 128 + ((rg ^ (cg * 2)) << 2)) = four;
    }
  }
  if (SQUARE && t < 4) {
    if (t == 0) a.scale_t[(int64_t)kb * a.lds_t + rb] = (uint8_t)(e + 127);
    else if (rb == rbs - 1 && rb + t < a.lds_t) a.scale_t[(int64_t)kb * a.lds_t + rb + t] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = (t >> 3) + 64 * k, p = t & 7, s = (c >> 3) * 2;
    const int64_t at = rb * kBlock + p * 16;
    const u32x2 lo = *reinterpret_cast<const u32x2*>(turned + c * 128 + (((p * 4) ^ s) << 2));
    const u32x2 hi = *reinterpret_cast<const u32x2*>(turned + c * 128 + (((p * 4 + 2) ^ s) << 2));
    if (kb * kBlock + c < a.cols && at < a.ldqt)
      __builtin_nontemporal_store(u32x4{lo[0], lo[1], hi[0], hi[1]}, reinterpret_cast<u32x4*>(a.qt + (int64_t)(kb * kBlock + c) * a.ldqt + at));
  }
}

template <typename T, int Q, bool VEC>
hipError_t launch(const QuantArgs& a, int square, hipStream_t st) {
  if (!square && !a.qt) {
    const int64_t units = a.rows * a.kbp, grid = (units + 16 * kUnits - 1) / (16 * kUnits);
    quant_rows_kernel<T, Q, VEC><<<(unsigned)grid, 256, 0, st>>>(a);
  } else {
    const int64_t grid = (a.rows + kBlock - 1) / kBlock * a.kb;
    if (square) quant_tile_kernel<T, Q, VEC, true><<<(unsigned)grid, 512, 0, st>>>(a);
    else quant_tile_kernel<T, Q, VEC, false><<<(unsigned)grid, 512, 0, st>>>(a);
  }
  return hipGetLastError();
}
template <typename T, int Q>
hipError_t launch(const QuantArgs& a, int square, hipStream_t st) {
  return quant_in_pieces(a.x, a.ld, sizeof(T)) ? launch<T, Q, true>(a, square, st) : launch<T, Q, false>(a, square, st);
}

}  // namespace

int64_t fp8_ld(int64_t cols) { return (cols + 15) / 16 * 16; }
int64_t fp8_scale_ld(int64_t cols) { return ((cols + kBlock - 1) / kBlock + 3) / 4 * 4; }

hipError_t launch_quantize_fp8(const t5_quantize_cfg& c, const void* x, void* q, uint8_t* scale, void* qt, uint8_t* scale_t,
                               hipStream_t st) {
  QuantArgs a;
  a.x = x; a.q = (uint8_t*)q; a.scale = scale; a.qt = (uint8_t*)qt; a.scale_t = scale_t;
  a.rows = c.rows; a.ld = c.ld; a.cols = (int)c.cols;
  a.ldq = fp8_ld(c.cols); a.ldqt = fp8_ld(c.rows); a.lds_t = fp8_scale_ld(c.rows);
  a.kb = (int)((c.cols + kBlock - 1) / kBlock); a.kbp = (int)fp8_scale_ld(c.cols);
  const int square = c.block_rows == kBlock;
  if (c.dtype == T5_BF16)
    return c.q_dtype == T5_E4M3 ? launch<bf16, T5_E4M3>(a, square, st) : launch<bf16, T5_E5M2>(a, square, st);
  return c.q_dtype == T5_E4M3 ? launch<float, T5_E4M3>(a, square, st) : launch<float, T5_E5M2>(a, square, st);
}

}  // namespace t5mi
