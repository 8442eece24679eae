// Plan of the product of two quantised matrices, and the sum of its slices (kernel: gemm_fp8.h).
#include "gemm_fp8.h"

namespace t5mi {
namespace {

// C (+)= the sum of the slices, in order.  One pass: split * M * N floats in, C out.
__global__ __launch_bounds__(256) void gemm_fp8_sum_kernel(Fp8Gemm g) {
  const int64_t total = (int64_t)g.M * g.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / g.N, n = i - m * g.N;
    float s = 0.f;
    for (int k = 0; k < g.split; ++k) s += g.part[k * total + i];
    if (g.out_bf16) ((bf16*)g.C)[m * g.ldc + n] = (bf16)s;
    else {
      float* p = (float*)g.C + m * g.ldc + n;
      *p = g.accumulate ? *p + s : s;
    }
  }
}

int plan_split(const t5_gemm_fp8_cfg& c, int* slice_tiles) {
  const int64_t tiles = (int64_t)ceil_div(c.M, 128) * ceil_div(c.N, 128);
  const int nk = ceil_div(c.K, 128);
  int split = 1;
  while (tiles * split < 256 && split < 16 && nk / (split * 2) >= 4) split *= 2;
  *slice_tiles = (ceil_div(nk, split) + 3) / 4 * 4;
  return ceil_div(nk, *slice_tiles);
}

}  // namespace

size_t gemm_fp8_ws_bytes(const t5_gemm_fp8_cfg& c) {
  int tiles;
  const int split = plan_split(c, &tiles);
  return split > 1 ? (size_t)split * c.M * c.N * 4 : 0;
}

hipError_t launch_gemm_fp8(const t5_gemm_fp8_cfg& c, const void* A, const uint8_t* sa, const void* B, const uint8_t* sb, void* C,
                           void* ws, hipStream_t st) {
  Fp8Gemm g;
  g.A = (const uint8_t*)A; g.B = (const uint8_t*)B; g.sa = sa; g.sb = sb;
  g.lda = c.lda; g.ldb = c.ldb; g.lsa = c.lsa; g.lsb = c.lsb;
  g.sha = c.a_block_rows == kBlock ? 7 : 0; g.shb = c.b_block_rows == kBlock ? 7 : 0;
  g.M = c.M; g.N = c.N; g.K = c.K;
  g.C = C; g.ldc = c.ldc; g.out_bf16 = c.c_dtype == T5_BF16; g.accumulate = c.accumulate != 0;
  g.part = (float*)ws;
  g.split = plan_split(c, &g.slice_tiles);
  g.big = (int64_t)ceil_div(c.M, 256) * ceil_div(c.N, 256) >= 128;
  hipError_t e;
  if (c.a_dtype == T5_E4M3) e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_44(g, st) : launch_gemm_fp8_45(g, st);
  else e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_54(g, st) : launch_gemm_fp8_55(g, st);
  if (e != hipSuccess || g.split == 1) return e;
  const int64_t total = (int64_t)c.M * c.N;
  gemm_fp8_sum_kernel<<<(unsigned)std::min<int64_t>((total + 255) / 256, 2048), 256, 0, st>>>(g);
  return hipGetLastError();
}

}  // namespace t5mi
