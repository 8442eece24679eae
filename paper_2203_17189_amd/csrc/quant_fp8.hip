// Quantisation of a matrix to 8-bit floating point in blocks of 128, by rows and transposed (see include/t5mi.h).
//
// Per block: e from the largest |x|, code = x 2^-e rounded to nearest even.  Everything is bound by memory: x is read once,
// whatever is asked for, and each code is written once.
//   rows alone, blocks of one row: 16 lanes hold a block, 8 values each; no lane waits for another workgroup or for LDS.
//   transposed, or blocks of 128 x 128: a workgroup holds a 128 x 128 tile in registers, 8 x 8 values a thread; row maxima
//   within 16 lanes, column maxima through LDS; the transposed codes go through LDS, 8 rows of a column at a time, so that
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

// Elements [c, c + 8) of a row, zeros from `cols` on.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&v)[8]) {
  if (VEC && c + 8 <= cols) {
    if constexpr (sizeof(T) == 2) {
      const bf16x8 p = *reinterpret_cast<const bf16x8*>(row + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (float)p[j];
    } else {
      const f32x4 p = *reinterpret_cast<const f32x4*>(row + c), r = *reinterpret_cast<const f32x4*>(row + c + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[j] = p[j]; v[j + 4] = r[j]; }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_f32(row[c + j]) : 0.f;
  }
}

template <int Q>
__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float inv) {
  return u32x2{pack_fp8x4<Q>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
               pack_fp8x4<Q>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
}

constexpr int kUnits = 2;  // blocks that 16 lanes hold at once

// Units are (row, block) pairs, kbp of them in a row: those past the row's blocks write the zeros behind its scales.
template <typename T, int Q, bool VEC>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a) {
  const int64_t first = (int64_t)blockIdx.x * (16 * kUnits);
  const int64_t row0 = first / a.kbp;
  const uint32_t rem0 = (uint32_t)(first - row0 * a.kbp);
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
  float v[kUnits][8];
  int64_t row[kUnits];
  int b[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint32_t at = rem0 + u * 16 + g;
    row[u] = row0 + at / (uint32_t)a.kbp;
    b[u] = (int)(at % (uint32_t)a.kbp);
    if (row[u] < a.rows) load8<T, VEC>((const T*)a.x + row[u] * a.ld, b[u] * kBlock + l * 8, a.cols, v[u]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[u][j]));
    const int e = block_exponent<Q>(max16(m));
    if (row[u] >= a.rows) continue;
    const int c = b[u] * kBlock + l * 8;
    if (c < a.ldq) *reinterpret_cast<u32x2*>(a.q + row[u] * a.ldq + c) = codes8<Q>(v[u], block_inverse(e));
    if (l == 0) a.scale[row[u] * a.kbp + b[u]] = b[u] < a.kb ? (uint8_t)(e + 127) : 0;
  }
}

// SQUARE: one scale for the tile; else one for each of its rows (q) and columns (qt).
template <typename T, int Q, bool VEC, bool SQUARE>
__global__ __launch_bounds__(256) void quant_tile_kernel(QuantArgs a) {
  __shared__ __align__(16) uint8_t turned[128 * 128];  // [column][row], pieces of 8 rows swizzled by the column's group
  __shared__ uint32_t part[4][128];
  const int kb = blockIdx.x % a.kb;
  const int64_t rb = blockIdx.x / a.kb;
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
  const int c0 = kb * kBlock + cg * 8;
  const int64_t r0 = rb * kBlock + rg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (r0 + i < a.rows) load8<T, VEC>((const T*)a.x + (r0 + i) * a.ld, c0, a.cols, v[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
  }
  int e = 0;  // SQUARE: the tile's exponent
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[i][j]));
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    if ((t & 63) == 0) part[wave][0] = m;
    __syncthreads();
    e = block_exponent<Q>(max(max(part[0][0], part[1][0]), max(part[2][0], part[3][0])));
  } else if (a.qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, finite_bits(v[i][j]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
      if ((t & 48) == 0) part[wave][cg * 8 + j] = m;
    }
  }
  if (a.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (!SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[i][j]));
        e = block_exponent<Q>(max16(m));
      }
      if (r0 + i < a.rows) {
        if (c0 < a.ldq) *reinterpret_cast<u32x2*>(a.q + (r0 + i) * a.ldq + c0) = codes8<Q>(v[i], block_inverse(e));
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
  if constexpr (!SQUARE) __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = cg * 8 + j;
    if constexpr (!SQUARE) {
      e = block_exponent<Q>(max(max(part[0][c], part[1][c]), max(part[2][c], part[3][c])));
      if (c0 + j < a.cols) {
        if (rg == 0) a.scale_t[(int64_t)(c0 + j) * a.lds_t + rb] = (uint8_t)(e + 127);
        else if (rb == rbs - 1 && rg < 4 && rb + rg < a.lds_t) a.scale_t[(int64_t)(c0 + j) * a.lds_t + rb + rg] = 0;
      }
    }
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[i][j];
    *reinterpret_cast<u32x2*>(turned + c * 128 + ((rg ^ cg) << 3)) = codes8<Q>(w, block_inverse(e));
  }
  if (SQUARE && t < 4) {
    if (t == 0) a.scale_t[(int64_t)kb * a.lds_t + rb] = (uint8_t)(e + 127);
    else if (rb == rbs - 1 && rb + t < a.lds_t) a.scale_t[(int64_t)kb * a.lds_t + rb + t] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = (t >> 3) + 32 * k, p = (t & 7) * 2, s = c >> 3;
    const int64_t at = rb * kBlock + p * 8;
    const u32x2 lo = *reinterpret_cast<const u32x2*>(turned + c * 128 + ((p ^ s) << 3));
    const u32x2 hi = *reinterpret_cast<const u32x2*>(turned + c * 128 + (((p + 1) ^ s) << 3));
    if (kb * kBlock + c < a.cols && at < a.ldqt)
      *reinterpret_cast<u32x4*>(a.qt + (int64_t)(kb * kBlock + c) * a.ldqt + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
}

template <typename T, int Q, bool VEC>
hipError_t launch(const QuantArgs& a, int square, hipStream_t st) {
  if (!square && !a.qt) {
    const int64_t units = a.rows * a.kbp, grid = (units + 16 * kUnits - 1) / (16 * kUnits);
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    quant_rows_kernel<T, Q, VEC><<<(unsigned)grid, 256, 0, st>>>(a);
  } else {
    const int64_t grid = (a.rows + kBlock - 1) / kBlock * a.kb;
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (square) quant_tile_kernel<T, Q, VEC, true><<<(unsigned)grid, 256, 0, st>>>(a);
    else quant_tile_kernel<T, Q, VEC, false><<<(unsigned)grid, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}
template <typename T, int Q>
hipError_t launch(const QuantArgs& a, int square, hipStream_t st) {
  const bool vec = ((uintptr_t)a.x & 15) == 0 && (a.ld * (int64_t)sizeof(T)) % 16 == 0;
  return vec ? launch<T, Q, true>(a, square, st) : launch<T, Q, false>(a, square, st);
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
