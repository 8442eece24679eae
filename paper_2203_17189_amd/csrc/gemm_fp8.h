// Kernel template of the product of two quantised matrices; gemm_fp8_*.hip instantiate it, one pair of types each.
//
//   C[m, n] (+)= sum_k A[m, k] 2^(sa - 127) B[n, k] 2^(sb - 127)
//
// bfloat16 C: the matrix instructions for codes (v_mfma_scale_f32_32x32x64_f8f6f4) take a scale byte for every 32 values of
// k of each row: a block's power of two costs no vector instruction, and sums over all of K stay in one set of float32
// accumulators.  A lane's scale operand is a word that holds its row's bytes for four blocks of k; the instruction picks one.
// These instructions add products in groups of eight, and cut off each product's bits below 2^-13 of the group's largest
// (measured; toward zero; sums of groups and accumulators are float32): 1.6e-5 of the result on normal data, 6e-5 on data of
// a wide range, where rounding to bfloat16 is off by 1.7e-3.
// float32 C: that would be most of the error of a float32 result, so codes become bfloat16 on their way from LDS (with their
// scale: exact, a code has at most four significant bits) and take v_mfma_f32_32x32x16_bf16, whose sums are float32 (2e-7),
// at half the rate.
//
// Operands: both matrices have k along their rows, so a k-tile of 128 bytes is one block of scales, and a tile row is one
// cache line.  Tiles go from memory to LDS without passing registers (dma_1k), 16-byte pieces swizzled by row on the global
// side so that the fragments' reads meet no bank twice.  Rows past the matrix are its last row again: what they compute is
// not stored.
#pragma once
#include "fp8.h"
#include "kernels.h"
#include <algorithm>
#include <atomic>
#include <type_traits>

namespace t5mi {

struct Fp8Gemm {
  const uint8_t *A, *B, *sa, *sb;
  int64_t lda, ldb, lsa, lsb;
  int sha, shb;  // a row's scales are those of row >> sha
  int M, N, K;
  void* C;
  int64_t ldc;
  int out_bf16, accumulate;
  float* part;  // split > 1: slice s leaves its sums at part + s * M * N
  int split, slice_tiles, tiles_m, tiles_n;
};

// One pair of types each (A's, B's number of exponent bits).
hipError_t launch_gemm_fp8_44(const Fp8Gemm& g, hipStream_t st);
hipError_t launch_gemm_fp8_45(const Fp8Gemm& g, hipStream_t st);
hipError_t launch_gemm_fp8_54(const Fp8Gemm& g, hipStream_t st);
hipError_t launch_gemm_fp8_55(const Fp8Gemm& g, hipStream_t st);

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

// Row r (128 bytes) holds the logical 16-byte piece c at place c ^ swz(r).
__device__ __forceinline__ int fp8_swz(int row) { return (row ^ (row >> 3)) & 7; }

// Piece c (lanes 0 .. 31) or c + 1 (32 .. 63) of row base + lane % 32.  Which values of k a lane half holds is the same for
// both operands, and a row's scale is the same for all of them.
__device__ __forceinline__ i32x4 fp8_piece(const char* tile, int base, int c, int lane) {
  const int row = base + (lane & 31);
  return *reinterpret_cast<const i32x4*>(tile + row * 128 + (((c + (lane >> 5)) ^ fp8_swz(row)) << 4));
}
// 32 values of k for k-step kk (64 values) of a tile.
__device__ __forceinline__ i32x8 fp8_frag(const char* tile, int base, int kk, int lane) {
  const i32x4 lo = fp8_piece(tile, base, kk * 4, lane), hi = fp8_piece(tile, base, kk * 4 + 2, lane);
  return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// Eight codes as bfloat16, times 2^(byte - 127).
template <int T>
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, float scale) {
  bf16x2 v[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = h ? hi : lo;
    if constexpr (T == T5_E4M3) {
      v[h * 2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false);
      v[h * 2 + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true);
    } else {
      v[h * 2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, scale, false);
      v[h * 2 + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, scale, true);
    }
  }
  return bf16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}
// The scale of block OP of a word as the conversion takes it: only the exponent counts there (0: 2^-127).
template <int OP>
__device__ __forceinline__ float scale_operand(int word) { return __uint_as_float((uint32_t)((word >> (8 * OP)) & 255) << 23); }

template <int TA, int TB, int OP>
__device__ __forceinline__ f32x16 fp8_mfma(i32x8 b, i32x8 a, f32x16 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, TB == T5_E5M2, TA == T5_E5M2, OP, sb, OP, sa);
}

// Output tile and k-slice of a workgroup.  Consecutive ids go to the 8 XCDs in turn: each XCD takes a run of tiles, in
// columns of 8 tile rows, and shares their operands through its own L2.
__device__ __forceinline__ void fp8_place(const Fp8Gemm& g, int id, int& tm, int& tn, int& ks) {
  const int total = g.tiles_m * g.tiles_n * g.split, per = total / 8, more = total % 8;
  const int x = id % 8, at = id / 8;
  int t = x * per + min(x, more) + at;
  ks = t / (g.tiles_m * g.tiles_n);
  t -= ks * (g.tiles_m * g.tiles_n);
  const int grp = t / (8 * g.tiles_n), h = min(8, g.tiles_m - grp * 8);
  t -= grp * 8 * g.tiles_n;
  tm = grp * 8 + t % h;
  tn = t / h;
}

// F32: float32 C.
template <int BM, int BN, int WM, int WN, int TA, int TB, bool F32>
__global__ __launch_bounds__(WM * WN * 64) void gemm_fp8_kernel(Fp8Gemm g) {
  constexpr int NW = WM * WN, MJ = BM / WM / 32, NI = BN / WN / 32;
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
  constexpr int A_DMA = BM / 8 / NW, B_DMA = BN / 8 / NW;
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  int tm, tn, ks;
  fp8_place(g, blockIdx.x, tm, tn, ks);
  const int m0 = tm * BM, n0 = tn * BN;
  const int nk = (g.K + 127) >> 7, whole = g.K >> 7;
  const int t0 = ks * g.slice_tiles, t1 = min(t0 + g.slice_tiles, nk), tw = min(t1, whole);

  const uint8_t* pa = g.A + (int64_t)m0 * g.lda;
  const uint8_t* pb = g.B + (int64_t)n0 * g.ldb;
  uint32_t a_off[A_DMA], b_off[B_DMA];
#pragma unroll
  for (int i = 0; i < A_DMA; ++i) {
    const int row = (wave + i * NW) * 8 + (lane >> 3);
    a_off[i] = (uint32_t)min(row, g.M - 1 - m0) * (uint32_t)g.lda + (((lane & 7) ^ fp8_swz(row)) << 4);
  }
#pragma unroll
  for (int i = 0; i < B_DMA; ++i) {
    const int row = (wave + i * NW) * 8 + (lane >> 3);
    b_off[i] = (uint32_t)min(row, g.N - 1 - n0) * (uint32_t)g.ldb + (((lane & 7) ^ fp8_swz(row)) << 4);
  }
  const uint8_t *ra[MJ], *rb[NI];
#pragma unroll
  for (int j = 0; j < MJ; ++j)
    ra[j] = g.sa + (int64_t)(min(m0 + wm * (BM / WM) + j * 32 + (lane & 31), g.M - 1) >> g.sha) * g.lsa;
#pragma unroll
  for (int i = 0; i < NI; ++i)
    rb[i] = g.sb + (int64_t)(min(n0 + wn * (BN / WN) + i * 32 + (lane & 31), g.N - 1) >> g.shb) * g.lsb;

  f32x16 acc[NI][MJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < MJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  int xa[MJ], xb[NI];
  auto load_scales = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < MJ; ++j) xa[j] = *reinterpret_cast<const int*>(ra[j] + (t & ~3));
#pragma unroll
    for (int i = 0; i < NI; ++i) xb[i] = *reinterpret_cast<const int*>(rb[i] + (t & ~3));
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
  auto dma = [&](int t, int st) __attribute__((always_inline)) {
    const uint8_t *qa = pa + (int64_t)t * 128, *qb = pb + (int64_t)t * 128;
#pragma unroll
    for (int i = 0; i < A_DMA; ++i) dma_1k(lds0 + st * STAGE + (wave + i * NW) * 1024, qa, a_off[i]);
#pragma unroll
    for (int i = 0; i < B_DMA; ++i) dma_1k(lds0 + st * STAGE + A_BYTES + (wave + i * NW) * 1024, qb, b_off[i]);
  };
  auto compute = [&](int st, auto op_tag) __attribute__((always_inline)) {
    constexpr int OP = decltype(op_tag)::value;
    const char *sa = smem + st * STAGE, *sb = sa + A_BYTES;
    if constexpr (F32) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        i32x4 ca[MJ], cb[NI];
#pragma unroll
        for (int j = 0; j < MJ; ++j) ca[j] = fp8_piece(sa, wm * (BM / WM) + j * 32, kk * 2, lane);
#pragma unroll
        for (int i = 0; i < NI; ++i) cb[i] = fp8_piece(sb, wn * (BN / WN) + i * 32, kk * 2, lane);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 fa[MJ], fb[NI];
#pragma unroll
          for (int j = 0; j < MJ; ++j) fa[j] = widen8<TA>(ca[j][h * 2], ca[j][h * 2 + 1], scale_operand<OP>(xa[j]));
#pragma unroll
          for (int i = 0; i < NI; ++i) fb[i] = widen8<TB>(cb[i][h * 2], cb[i][h * 2 + 1], scale_operand<OP>(xb[i]));
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < MJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[i], fa[j], acc[i][j], 0, 0, 0);
        }
      }
      return;
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i32x8 fa[MJ], fb[NI];
#pragma unroll
      for (int j = 0; j < MJ; ++j) fa[j] = fp8_frag(sa, wm * (BM / WM) + j * 32, kk, lane);
#pragma unroll
      for (int i = 0; i < NI; ++i) fb[i] = fp8_frag(sb, wn * (BN / WN) + i * 32, kk, lane);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MJ; ++j) acc[i][j] = fp8_mfma<TA, TB, OP>(fb[i], fa[j], acc[i][j], xb[i], xa[j]);
    }
  };
  auto compute_at = [&](int t, int st) __attribute__((always_inline)) {
    switch (t & 3) {
      case 0: compute(st, std::integral_constant<int, 0>{}); break;
      case 1: compute(st, std::integral_constant<int, 1>{}); break;
      case 2: compute(st, std::integral_constant<int, 2>{}); break;
      default: compute(st, std::integral_constant<int, 3>{}); break;
    }
  };

  if (t0 < tw) dma(t0, 0);
  for (int t = t0; t < tw; ++t) {
    const int st = (t - t0) & 1;
    if (t + 1 < tw) dma(t + 1, st ^ 1);
    if ((t & 3) == 0) load_scales(t);
    if (t + 1 < tw) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(A_DMA + B_DMA) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    compute_at(t, st);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
  if (t1 > tw) {  // the last tile of K, through registers: zeros past its end
    const int left = g.K - whole * 128;
    const uint8_t *qa = pa + (int64_t)whole * 128, *qb = pb + (int64_t)whole * 128;
    auto piece = [&](const uint8_t* base, uint32_t off, int row) __attribute__((always_inline)) {
      const int c = ((lane & 7) ^ fp8_swz(row)) << 4;
      u32x4 v = {0, 0, 0, 0};
      if (c < left) v = *reinterpret_cast<const u32x4*>(base + off);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int keep = left - c - w * 4;
        v[w] = keep >= 4 ? v[w] : keep <= 0 ? 0u : v[w] & ((1u << (keep * 8)) - 1u);
      }
      return v;
    };
#pragma unroll
    for (int i = 0; i < A_DMA; ++i)
      *reinterpret_cast<u32x4*>(smem + (wave + i * NW) * 1024 + lane * 16) = piece(qa, a_off[i], (wave + i * NW) * 8 + (lane >> 3));
#pragma unroll
    for (int i = 0; i < B_DMA; ++i)
      *reinterpret_cast<u32x4*>(smem + A_BYTES + (wave + i * NW) * 1024 + lane * 16) = piece(qb, b_off[i], (wave + i * NW) * 8 + (lane >> 3));
    load_scales(whole);
    __syncthreads();
    compute_at(whole, 0);
  }

  // acc[i][j][r] is C[n0 + .. + (r / 4) * 8 + (lane / 32) * 4 + r % 4][m0 + .. + lane % 32] transposed: a lane holds runs of
  // four columns of one row.
  const bool part = g.split > 1;
  float* pf = part ? g.part + (int64_t)ks * g.M * g.N : (float*)g.C;
  const int64_t ld = part ? g.N : g.ldc;
  const bool bf = !F32 && !part, add = F32 && !part && g.accumulate;
  const bool vec = (ld & 3) == 0 && ((uintptr_t)pf & (bf ? 7 : 15)) == 0;
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int m = m0 + wm * (BM / WM) + j * 32 + (lane & 31);
    if (m >= g.M) continue;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn * (BN / WN) + i * 32 + q * 8 + (lane >> 5) * 4;
        float* p = pf + (int64_t)m * ld + n;
        bf16* pl = (bf16*)pf + (int64_t)m * ld + n;
        f32x4 v = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
        if (vec && n + 4 <= g.N) {
          if (bf) *reinterpret_cast<u32x2*>(pl) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
          else {
            if (add) v += *reinterpret_cast<const f32x4*>(p);
            *reinterpret_cast<f32x4*>(p) = v;
          }
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if (n + w < g.N) {
              if (bf) pl[w] = (bf16)v[w];
              else p[w] = add ? p[w] + v[w] : v[w];
            }
        }
      }
  }
}

template <int BM, int BN, int WM, int WN, int TA, int TB, bool F32>
hipError_t launch_fp8_tiles(Fp8Gemm g, hipStream_t st) {
  auto kern = gemm_fp8_kernel<BM, BN, WM, WN, TA, TB, F32>;
  constexpr int lds = 2 * (BM + BN) * 128;
  static std::atomic<bool> attr_set{false};  // once per instantiation; setting it twice is harmless
  if (!attr_set.load(std::memory_order_relaxed)) {
    const hipError_t err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (err != hipSuccess) return err;
    attr_set.store(true, std::memory_order_relaxed);
  }
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, BN);
  const int64_t grid = (int64_t)g.tiles_m * g.tiles_n * g.split;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  kern<<<(unsigned)grid, WM * WN * 64, lds, st>>>(g);
  return hipGetLastError();
}

template <int TA, int TB>
hipError_t launch_fp8_types(const Fp8Gemm& g, hipStream_t st) {
  return g.out_bf16 ? launch_fp8_tiles<128, 128, 2, 2, TA, TB, false>(g, st) : launch_fp8_tiles<128, 128, 2, 2, TA, TB, true>(g, st);
}

}  // namespace
}  // namespace t5mi
