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

// Which tiles, and whether those of the last, partly filled round are shared out along k: whatever is estimated to be faster.
// Estimates in us, fitted to the kernels of gemm_fp8.h on shapes of 64 .. 32768 by 300 .. 32128 by 512 .. 32768.  A k-tile of
// a full round (`at_once` tiles: one, two or four workgroups on each of 256 compute units) takes the longer the more of the
// chip is at work, as clocks follow power: `idle` where few tiles run, `busy` more in a full round, rising from a fill of
// `from` on.  A round has `ends` besides.  Sharing costs a launch and the parts' way to memory and back, 3.5 MB a us.
// Small tiles have more loads and conversions to a matrix instruction, large ones fewer workgroups and longer ends.  Measured,
// M x N x K and type of C, us:                tiles of 64, shared      128, shared      256, shared
//   300 x 500 x 1024      f32                  8.5    13.1            13.4    13.3        41      28
//   2048 x 2048 x 2048    bf16                17.4    17.7            13.0    25.8        30      37
//   768 x 2048 x 16384    f32                 85.5    92.3             114      65       279      84
//   4096 x 4096 x 4096    bf16                                          73                65
//   5120 x 2048 x 32768   bf16                                         394     372       353     408
//   5120 x 2048 x 32768   f32                                          609     565       590     549
struct TileCost { int tile, at_once; double idle, busy, from, ends; };
constexpr TileCost kTileCost[2][3] = {
    {{64, 1024, 0.39, 0.6, 0.25, 2.0}, {128, 512, 0.53, 0.55, 0.2, 2.5}, {256, 256, 1.1, 0.6, 0.4, 12.5}},   // bf16 C
    {{64, 1024, 0.55, 0.85, 0.25, 2.0}, {128, 512, 0.83, 0.92, 0.2, 5.0}, {256, 256, 2.05, 1.0, 0.5, 12.5}}};  // float32 C

double round_cost(const TileCost& t, double fill, double nk) {
  return nk * (t.idle + t.busy * std::max(0.0, fill - t.from) / (1.0 - t.from)) + t.ends;
}

// Against few rows of A, B comes from memory (a model's weights pass through the caches between two calls): a k-tile then takes
// longer than the same of operands that many tiles share, and of more than 16 parts of a tile the sum waits for each.  Fitted
// to 1 .. 16 rows against 512 .. 131072 by 384 .. 16384.
constexpr TileCost kFewRowsCost[2] = {{64, 1024, 0.76, 0.71, 0.25, 2.5}, {64, 1024, 0.94, 0.64, 0.2, 2.8}};  // bf16 C, float32 C

// Without tiles, mt * 16 rows of A a workgroup.  Up to 16 rows: a compute unit takes in 18.2 bytes of B a ns, workgroup after
// workgroup.  Measured, B from memory, us (no tiles, tiles of 64):
//   M x N x K               bfloat16         float32                             bfloat16         float32
//   1 x  9216 x 2048       9.6   14.3      10.3   16.8      1 x 50257 x  768   15.3   12.7      16.2   13.5
//   1 x 16384 x 5120      19.9   32.2      20.4   38.6      1 x 50257 x 2048   27.8   23.3      28.9   26.5
//   1 x 32128 x  768       9.4    8.6      10.0   10.5     16 x 50257 x 2048   30.1   24.6      32.0   29.0
//   1 x 32128 x 2048      16.8   16.6      18.1   21.7      1 x 65536 x 2048   33.6   28.3      32.3   30.3
//  16 x 32128 x 2048      18.1   17.6      19.6   22.8      1 x 131072 x 768   31.1   23.4      33.2   26.2
//   1 x 32128 x 5120      36.0   38.2      37.3   49.2      1 x 131072 x 5120   136    119       142    135
// More rows: what a compute unit takes in (37 bytes a ns; widening on top of it), or B's bytes once and what comes again from
// L2 for each workgroup, and the launch.  Measured, us, bfloat16, and in tiles:
//   32 x 2048 x 5120: 7.2, 12.6    64 x 2048 x 5120: 9.3, 12.9       189 x 128 x 2944: 4.4, 8.4       333 x 509 x 1001: 4.7, 5.8
double rows_cost(const t5_gemm_fp8_cfg& c, int mt) {
  const int64_t rb = 16 * fp8_rows_of_b(c.M, c.N), ra = std::min(c.M, 16 * mt), k = c.K;
  const int64_t tm = ceil_div(c.M, 16 * mt), wgs = (c.N + rb - 1) / rb * tm;
  const int64_t taken = rb + 16 * mt;
  const bool f32 = c.c_dtype == T5_F32;
  const int64_t rounds = (wgs + 255) / 256;  // ends and beginnings of workgroups with many registers do not overlap
  if (c.M <= 16) return 2.0 + (double)rounds * (0.5 + ((double)rb + c.M / 8.0) * (double)k / 18.2e3) * (f32 ? 1.0 : 0.95);
  const double unit = (double)(rounds * taken * k) / 37e3 * (f32 ? 1.1 : 1.0) + (mt > 1 ? (double)(rounds - 1) * (f32 ? 1.0 : 0.5) : 0.0);
  return 2.0 + std::max(unit, (double)(c.N * k + (c.N * (tm - 1) + wgs * ra) * k / 8) / 6e6);
}

void plan(const t5_gemm_fp8_cfg& c, Fp8Gemm* g) {
  g->shared = g->workers = 0;
  g->few = 0;
  const int units = ceil_div(c.K, 512);
  const double nk = c.K / 128.0;
  double best = -1.0;
  for (const TileCost& many : kTileCost[c.c_dtype == T5_F32]) {
    if (c.M <= 16 && best >= 0.0) break;  // larger tiles only where these would be too many
    const TileCost& t = c.M <= 16 && many.tile == 64 ? kFewRowsCost[c.c_dtype == T5_F32] : many;
    const int B = t.tile, slots = t.at_once, tm = ceil_div(c.M, B), tn = ceil_div(c.N, B);
    if (B == 256 && (c.M < 256 || c.N < 256)) break;
    const int64_t tiles = (int64_t)tm * tn, rest = tiles % slots;
    if (tiles + slots > kMostWorkgroups && (B == 64 || (B == 128 && c.M >= 256 && c.N >= 256))) continue;  // larger ones are fewer
    const double full = (double)(tiles / slots) * round_cost(t, 1.0, nk), fill = (double)rest / slots;
    const double alone = full + (rest ? round_cost(t, fill, nk) : 0.0);
    const int64_t workers = std::min<int64_t>(slots, rest * units);
    const double run = (double)workers / slots;
    double shared = full + round_cost(t, run, nk * rest / std::max<int64_t>(workers, 1)) + 6.0 + (double)(workers + rest) * B * B * 8 / 3.5e6;
    if (c.M <= 16 && rest > 0) shared += 0.25 * std::max(0.0, (double)workers / (double)rest - 16.0);
    const bool share = rest > 0 && workers > rest && shared < alone;
    const double cost = share ? shared : alone;
    if (best >= 0.0 && cost >= best) continue;
    best = cost;
    g->tile = B; g->tiles_m = tm; g->tiles_n = tn;
    g->shared = share ? (int)rest : 0;
    g->workers = share ? (int)workers : 0;
  }
  for (int mt = 1; mt <= 4; mt *= 2) {
    if (mt > 1 && c.M <= 8 * mt) break;
    const int64_t wgs = (int64_t)ceil_div(c.N, 16 * fp8_rows_of_b(c.M, c.N)) * ceil_div(c.M, 16 * mt);
    if (wgs > (c.M <= 16 ? kMostWorkgroups / 2 : 4096)) continue;
    const double cost = rows_cost(c, mt);
    if (cost > best) continue;
    best = cost;
    g->few = mt;
    g->shared = g->workers = 0;
  }
}

}  // namespace

size_t gemm_fp8_ws_bytes(const t5_gemm_fp8_cfg& c) {
  Fp8Gemm g;
  plan(c, &g);
  if (g.workers <= g.shared) return 0;
  const size_t B = g.tile;
  return ((size_t)g.workers + g.shared) * B * B * 4;
}

int gemm_fp8_path(const t5_gemm_fp8_cfg& c) {
  Fp8Gemm g;
  plan(c, &g);
  if (g.few) {
    const int nt = fp8_rows_of_b(c.M, c.N);
    return T5_FP8_PATH_ROWS | (g.few == 2 ? T5_FP8_PATH_ROWS_A32 : g.few == 4 ? T5_FP8_PATH_ROWS_A64 : 0) |
           (nt == 2 ? T5_FP8_PATH_ROWS_B32 : 0);
  }
  return (g.tile == 64 ? T5_FP8_PATH_TILE64 : g.tile == 128 ? T5_FP8_PATH_TILE128 : T5_FP8_PATH_TILE256) |
         (g.workers > g.shared ? T5_FP8_PATH_SHARED : 0);
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
  if (g.few) return launch_gemm_fp8_rows(g, c.a_dtype, c.b_dtype, st);
  hipError_t e;
  if (c.a_dtype == T5_E4M3) e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_44(g, st) : launch_gemm_fp8_45(g, st);
  else e = c.b_dtype == T5_E4M3 ? launch_gemm_fp8_54(g, st) : launch_gemm_fp8_55(g, st);
  if (e != hipSuccess || g.workers <= g.shared) return e;
  if (g.tile == 256) gemm_fp8_sum_kernel<256><<<(unsigned)g.shared * 16, 256, 0, st>>>(g);
  else if (g.tile == 128) gemm_fp8_sum_kernel<128><<<(unsigned)g.shared * 8, 256, 0, st>>>(g);
  else gemm_fp8_sum_kernel<64><<<(unsigned)g.shared * 4, 256, 0, st>>>(g);
  return hipGetLastError();
}

}  // namespace t5mi
