// Product of a few quantised rows (single tokens, short batches) with a quantised matrix, and small products.
//
// Bound by reading B once.  A workgroup has 16 rows of B, or 32, and 16 to 64 of A (16 to 64 by 16, or 16 by 32); its
// wavefronts take the blocks of 128 k in turn, straight from memory into the operands of a matrix instruction: no LDS, no
// barrier before the end, and the loads of IN blocks of a wavefront are under way at once.  The wavefronts' sums meet in LDS, in order.  A is read again by each workgroup, from L2.
// The instructions are the ones of gemm_fp8.h, 16 x 16 wide: codes with scales for bfloat16 C, widened codes for float32.
#include "gemm_fp8.h"

namespace t5mi {
namespace {

// A lane's 32 bytes of a row's block of 128: 16 at p and 16 at p + 64, so that the four lanes of a row read 64 bytes in a
// row with each load.  `left`: bytes of the matrix from p on; pieces that begin there are in memory as wholes, zeros behind.
__device__ __forceinline__ i32x8 load32_part(const uint8_t* p, int left) {
  i32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    i32x4 q = {0, 0, 0, 0};
    if (left > h * 64) q = *reinterpret_cast<const i32x4*>(p + h * 64);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int keep = left - h * 64 - w * 4;
      v[h * 4 + w] = keep >= 4 ? q[w] : keep <= 0 ? 0 : (int)((uint32_t)q[w] & ((1u << (keep * 8)) - 1u));
    }
  }
  return v;
}
// The same of a whole block, lanes with `odd` the second piece first, so that even rows ask for one half of a line and odd
// ones for the other: sixteen rows a multiple of 128 bytes apart would ask for the same half together, which the L1 serves slowly (16 x 2048 x 16384: 23.3 us, like this 17.3).
__device__ __forceinline__ i32x8 load32(const uint8_t* p, bool odd) {
  const i32x4 a = *reinterpret_cast<const i32x4*>(p + (odd ? 64 : 0)), b = *reinterpret_cast<const i32x4*>(p + (odd ? 0 : 64));
  i32x8 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[w] = odd ? b[w] : a[w];
    v[4 + w] = odd ? a[w] : b[w];
  }
  return v;
}

template <int MT, int NT> struct Block {
  i32x8 b[NT], a[MT];
  int sb[NT], sa[MT];
};

// MT, NT: tiles of 16 rows of A and of B.  NW wavefronts, IN blocks each under way at a time.
template <int TA, int TB, bool F32, int MT, int NT, int NW, int IN>
__global__ __launch_bounds__(NW * 64) void gemm_fp8_rows_kernel(Fp8Gemm g) {
  __shared__ f32x4 sums[NW][NT * MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT), nk = (g.K + 127) >> 7, k0 = (lane >> 4) * 16;
  bool odd_a[MT], odd_b[NT];
  const uint8_t *pa[MT], *qa[MT], *pb[NT], *qb[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int rb = min(n0 + i * 16 + (lane & 15), g.N - 1);
    pb[i] = g.B + (int64_t)rb * g.ldb + k0;
    odd_b[i] = ((uintptr_t)pb[i] >> 6 ^ rb) & 1;
    qb[i] = g.sb + (int64_t)(rb >> g.shb) * g.lsb;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int ra = min(m0 + j * 16 + (lane & 15), g.M - 1);
    pa[j] = g.A + (int64_t)ra * g.lda + k0;
    odd_a[j] = ((uintptr_t)pa[j] >> 6 ^ ra) & 1;
    qa[j] = g.sa + (int64_t)(ra >> g.sha) * g.lsa;
  }
  f32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load = [&](Block<MT, NT>& x, int t) __attribute__((always_inline)) {
    const int left = g.K - t * 128 - k0;
    const bool whole = (t + 1) * 128 <= g.K;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      x.b[i] = whole ? load32(pb[i] + (int64_t)t * 128, odd_b[i]) : load32_part(pb[i] + (int64_t)t * 128, left);
      x.sb[i] = qb[i][t];
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      x.a[j] = whole ? load32(pa[j] + (int64_t)t * 128, odd_a[j]) : load32_part(pa[j] + (int64_t)t * 128, left);
      x.sa[j] = qa[j][t];
    }
  };
  auto add = [&](const Block<MT, NT>& x) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        bf16x8 wb[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) wb[i] = widen8<TB>(x.b[i][s * 2], x.b[i][s * 2 + 1], scale_operand<0>(x.sb[i]));
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const bf16x8 wa = widen8<TA>(x.a[j][s * 2], x.a[j][s * 2 + 1], scale_operand<0>(x.sa[j]));
#pragma unroll
          for (int i = 0; i < NT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[i], wa, acc[i][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.b[i], x.a[j], acc[i][j], TB == T5_E5M2, TA == T5_E5M2, 0, x.sb[i], 0, x.sa[j]);
    }
  };
  for (int t = wave; t < nk; t += IN * NW) {  // (the last blocks, too, are all loaded first: 1 x 5120 x 2048 5.4 us, like this 4.4)
    Block<MT, NT> x[IN];
#pragma unroll
    for (int i = 0; i < IN; ++i)
      if (t + i * NW < nk) load(x[i], t + i * NW);
#pragma unroll
    for (int i = 0; i < IN; ++i)
      if (t + i * NW < nk) add(x[i]);
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) sums[wave][i * MT + j][lane] = acc[i][j];
  __syncthreads();
  for (int at = threadIdx.x; at < NT * MT * 64; at += NW * 64) {
    const int ij = at >> 6, l = at & 63;
    f32x4 s = sums[0][ij][l];
#pragma unroll
    for (int w = 1; w < NW; ++w) s += sums[w][ij][l];
    const int m = m0 + ij % MT * 16 + (l & 15), n = n0 + ij / MT * 16 + (l >> 4) * 4;  // a lane holds four columns of a row
    if (m >= g.M) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i >= g.N) continue;
      if constexpr (F32) {
        float* p = (float*)g.C + (int64_t)m * g.ldc + n + i;
        *p = g.accumulate ? *p + s[i] : s[i];
      } else {
        ((bf16*)g.C)[(int64_t)m * g.ldc + n + i] = (bf16)s[i];
      }
    }
  }
}

template <int TA, int TB, bool F32>
hipError_t launch(const Fp8Gemm& g, hipStream_t st) {
  const int nt = fp8_rows_of_b(g.M, g.N);
  const dim3 grid((unsigned)ceil_div(g.N, 16 * nt), (unsigned)ceil_div(g.M, 16 * g.few));
  // Sixteen wavefronts where each still has several blocks (1 x 2048 x 16384: with eight 15.6 us, 12.0).
  if (g.few == 1) {
    if (nt == 2) gemm_fp8_rows_kernel<TA, TB, F32, 1, 2, 8, 2><<<grid, 512, 0, st>>>(g);
    else if (g.K > 4096) gemm_fp8_rows_kernel<TA, TB, F32, 1, 1, 16, 4><<<grid, 1024, 0, st>>>(g);
    else if (g.K > 1024) gemm_fp8_rows_kernel<TA, TB, F32, 1, 1, 8, 4><<<grid, 512, 0, st>>>(g);
    else gemm_fp8_rows_kernel<TA, TB, F32, 1, 1, 4, 2><<<grid, 256, 0, st>>>(g);
  } else if (g.few == 2) {
    gemm_fp8_rows_kernel<TA, TB, F32, 2, 1, 8, 4><<<grid, 512, 0, st>>>(g);
  } else {
    gemm_fp8_rows_kernel<TA, TB, F32, 4, 1, 8, 2><<<grid, 512, 0, st>>>(g);
  }
  return hipGetLastError();
}
template <int TA, int TB>
hipError_t launch(const Fp8Gemm& g, hipStream_t st) { return g.out_bf16 ? launch<TA, TB, false>(g, st) : launch<TA, TB, true>(g, st); }

}  // namespace

// Two where that leaves two workgroups to a compute unit, as each reads A anew (one row of A, float32, B from memory: 32128 x
// 2048 with one 21.5 us, with two 18.1, with four 20.2; 16384 x 5120 27.3, 20.4, 23.2; 50257 x 768 14.6, 16.2, 20.7).
// More rows of A leave the registers for one (32 x 2048 x 2048: with two 5.4 us, 4.5).
int fp8_rows_of_b(int M, int N) {
  const int n16 = ceil_div(N, 16);
  return M > 16 ? 1 : n16 >= 1024 ? 2 : 1;
}

hipError_t launch_gemm_fp8_rows(const Fp8Gemm& g, int ta, int tb, hipStream_t st) {
  if (ta == T5_E4M3) return tb == T5_E4M3 ? launch<T5_E4M3, T5_E4M3>(g, st) : launch<T5_E4M3, T5_E5M2>(g, st);
  return tb == T5_E4M3 ? launch<T5_E5M2, T5_E4M3>(g, st) : launch<T5_E5M2, T5_E5M2>(g, st);
}

}  // namespace t5mi
