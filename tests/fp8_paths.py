"""Shapes that reach every kernel of the product of quantised matrices, with the kernel that each is there for, and operands,
values and error bounds on the GPU.  tests/test_fp8_paths_cpu.py holds the choice to this list."""
import torch

import paper_2203_17189_amd as P
from fp8_util import DT, E8M0, FP8, STORE, U

T64, T128, T256, SHARED = P.FP8_PATH_TILE64, P.FP8_PATH_TILE128, P.FP8_PATH_TILE256, P.FP8_PATH_SHARED
ROWS, A32, A64 = P.FP8_PATH_ROWS, P.FP8_PATH_ROWS | P.FP8_PATH_ROWS_A32, P.FP8_PATH_ROWS | P.FP8_PATH_ROWS_A64
B32 = P.FP8_PATH_ROWS | P.FP8_PATH_ROWS_B32

# M, N, K, type of C, kernel.  Sizes off the multiples of a tile, of a block of k and of a piece; tiles of 256 reach back in
# both directions.  ROWS has three forms by K.
SHAPES = [
    *[(3, 200, 330, out, ROWS) for out in DT], *[(16, 259, 3000, out, ROWS) for out in DT], *[(5, 97, 5000, out, ROWS) for out in DT],
    *[(31, 2100, 1100, out, A32) for out in DT], *[(270, 300, 1100, out, A32) for out in DT], *[(515, 257, 330, out, A64) for out in DT],
    *[(7, 16380, 1100, out, B32) for out in DT], *[(1, 50257, 700, out, T64) for out in DT],
    *[(1000, 257, 330, out, T64) for out in DT], *[(700, 2049, 1100, out, T64) for out in DT],
    *[(2100, 3001, 330, out, T128) for out in DT], *[(1500, 3001, 700, out, T128) for out in DT],
    (4097, 3500, 1537, "f32", T256), *[(4100, 2049, 4100, out, T256) for out in DT],
    *[(259, 301, 16400, out, T64 | SHARED) for out in DT], *[(912, 1046, 16390, out, T128 | SHARED) for out in DT],
    *[(1500, 3001, 30010, out, T256 | SHARED) for out in DT],
    # more tiles than run at once: those of whole rounds are stored by themselves, the rest in parts
    *[(5418, 1454, 5001, out, T128 | SHARED) for out in DT], *[(1448, 11030, 8200, out, T256 | SHARED) for out in DT],
]
IDS = ["%dx%dx%d-%s" % s[:4] for s in SHAPES]
# What the list has to reach, for results of both types.
REACHED = [(p, out) for p in (ROWS, A32, A64, B32, T64, T128, T256, T64 | SHARED, T128 | SHARED, T256 | SHARED) for out in DT]
# Tokens, width in and out of a layer, and which of its three products (y, dx, dw) divides its k, on tiles of what size.
LAYERS = [(260, 16400, 301, "y", T64), (301, 260, 16400, "dx", T64), (16400, 301, 259, "dw", T64), (16390, 1046, 912, "dw", T128),
          (30010, 3001, 1500, "dw", T256)]


def path(m, n, k, out):
    return P.t5_gemm_fp8_kernel_path(m, n, k, DT[out])


def layer_products(tokens, d_in, d_out):
    return {"y": (tokens, d_out, d_in, "bf16"), "dx": (tokens, d_in, d_out, "bf16"), "dw": (d_out, d_in, tokens, "f32")}


def operand(gen, rows, k, fmt, block_rows, gap=0):
    """(codes, scales, values in float64), random, of every finite code; rows `gap` bytes further apart than they need be, what
    is between them NaN, of scales too."""
    ld, sr, sk = -(-k // 16) * 16 + gap, -(-rows // block_rows), -(-k // 128)
    lds = -(-sk // 4) * 4 + (4 if gap else 0)
    finite = torch.arange(256, dtype=torch.uint8, device="cuda")
    finite = finite[finite.view(FP8[fmt]).float().isfinite()]
    q = torch.full((rows, ld), 0xFF, dtype=torch.uint8, device="cuda")
    q[:, :k] = finite[torch.randint(len(finite), (rows, k), device="cuda", generator=gen)]
    s = torch.full((sr, lds), 0xFF, dtype=torch.uint8, device="cuda")
    s[:, :sk] = torch.randint(120, 134, (sr, sk), device="cuda", generator=gen).to(torch.uint8)
    q, s = q[:, :k].view(FP8[fmt]), s[:, :sk].view(E8M0)
    return q, s, values(q, s)


def values(q, s):
    e = s.view(torch.uint8).double() - 127
    f = torch.exp2(e).repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.float().double() * (f if s.shape[0] == q.shape[0] else f.repeat_interleave(128, 0)[:q.shape[0]])


def bound(a, b, want, out):
    """fp8_util.product_bound for float64 tensors on the GPU, with two roundings more for each of up to 257 parts of a tile
    that are added (an addend's rounding is among the 20 there)."""
    a, b = a.abs(), b.abs()
    k = a.shape[1]
    far = (k / 16 + 64 + 20 + 257) * U * torch.matmul(a, b.t().contiguous()) + STORE[out] * want.abs() + 1e-30
    if out == "bf16":
        at, bt = a.t().contiguous(), b.t().contiguous()
        big, other = torch.empty_like(want), torch.empty_like(want)
        for g in range(0, k, 8):
            big.zero_()
            for j in range(g, min(g + 8, k)):
                torch.mul(at[j][:, None], bt[j][None], out=other)
                torch.maximum(big, other, out=big)
            far.add_(big, alpha=7 * 2.0 ** -13)
    return far
