// Plan of the product of two quantised matrices, and the sum of its tiles' parts (kernel: gemm_fp8.h).
#include "gemm_fp8.h"

namespace t5mi {
namespace {

// C (+)= the parts of each shared tile, in the order of k.  A workgroup has 16 rows of a tile; parts are read once.
template <int B>
__global__ __launch_bounds__(256) void gemm_fp8_sum_kernel(Fp8Gemm g) {
  constexpr int PER = B / 16;  // workgroups of a tile
  const int tile = blockIdx.x / PER, r0 = blockIdx.x % PER * 16, units = fp8_units(g);
  const int w0 = fp8_worker(g, (int64_t)tile * units), w1 = fp8_worker(g, (int64_t)(tile + 1) * units - 1);
  if (w0 == w1) return;  // one worker has all of it and has stored it
  int tm, tn;
  fp8_place(g, tile, tm, tn);
  const int m_own = tm * B, n_own = tn * B;
  const int m0 = B == 256 ? min(m_own, g.M - B) : m_own, n0 = B == 256 ? min(n_own, g.N - B) : n_own;
#pragma unroll
  for (int k = 0; k < 16 * B / 1024; ++k) {
    const int at = (k * 256 + threadIdx.x) * 4, m = m0 + r0 + at / B, n = n0 + at % B;
    const float* p = g.part + ((int64_t)w0 + tile) * (B * B) + r0 * B + at;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0; w <= w1; ++w, p += B * B) s += *reinterpret_cast<const f32x4*>(p);
    if (m < m_own || m >= g.M) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i < n_own || n + i >= g.N) continue;
      if (g.out_bf16) ((bf16*)g.C)[(int64_t)m * g.ldc + n + i] = (bf16)s[i];
      else {
        float* c = (float*)g.C + (int64_t)m * g.ldc + n + i;
        *c = g.accumulate ? *c + s[i] : s[i];
      }
    }
  }
}

constexpr int kCus = 256;

void plan(const t5_gemm_fp8_cfg& c, Fp8Gemm* g) {
  const int units = ceil_div(c.K, 512);
  g->big = c.M >= 256 && c.N >= 256 && (int64_t)ceil_div(c.M, 256) * ceil_div(c.N, 256) * units >= 256;
  const int B = g->big ? 256 : 128, slots = g->big ? kCus : 2 * kCus;
  g->tiles_m = ceil_div(c.M, B);
  g->tiles_n = ceil_div(c.N, B);
  const int64_t tiles = (int64_t)g->tiles_m * g->tiles_n, rest = tiles % slots;
  g->shared = g->workers = 0;
  if (rest > 0 && rest <= slots * 7 / 8 && units > 1) {
    g->shared = (int)rest;
    g->workers = (int)std::min<int64_t>(slots, rest * units);
  }
}

}  // namespace

size_t gemm_fp8_ws_bytes(const t5_gemm_fp8_cfg& c) {
  Fp8Gemm g;
  plan(c, &g);
  const size_t B = g.big ? 256 : 128;
  return g.workers > g.shared ? ((size_t)g.workers + g.shared) * B * B * 4 : 0;
}

hipError_t launch_gemm_fp8(const t5_gemm_fp8_cfg& c, const void* A, const uint8_t* sa, const void* B, const uint8_t* sb, void* C,
                           void* ws, hipStream_t st) {
  Fp8Gemm g;
  plan(c, &g);
  g.A = (const uint8_t*)A; g.B = (const uint8_t*)B; g.sa = sa; g.sb = sb;
  g.lda = c.lda; g.ldb = c.ldb; g.lsa = c.lsa; g.lsb = c.lsb;
  g.sha = c.a_block_rows == kBlock ? 7 : 0; g.shb = c.b_block_rows == kBlock ? 7 : 0;
  g.M = c.M; g.N = c.N; g.K = c.K;
  g.C = C; g.ldc = c.ldc; g.out_bf16 = c.c_dtype == T5_BF16; g.accumulate = c.accumulate != 0;
  g.part = (float*)ws;
  hipError_t e;
  if (c.a_dtype == T5_E4M3) e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_44(g, st) : launch_gemm_fp8_45(g, st);
  else e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_54(g, st) : launch_gemm_fp8_55(g, st);
  if (e != hipSuccess || g.workers <= g.shared) return e;
  if (g.big) gemm_fp8_sum_kernel<256><<<(unsigned)g.shared * 16, 256, 0, st>>>(g);
  else gemm_fp8_sum_kernel<128><<<(unsigned)g.shared * 8, 256, 0, st>>>(g);
  return hipGetLastError();
}

}  // namespace t5mi
