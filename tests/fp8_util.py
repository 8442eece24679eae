"""Inputs, views and error bounds of the tests of training in 8 bits."""
import numpy as np
import torch

from oracle import fp8_oracle as O

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
E8M0 = torch.float8_e8m0fnu
STORE = {"f32": U, "bf16": 2.0 ** -8}


def host(t):
    return t.detach().double().cpu().numpy()


def codes(t):
    return t.detach().contiguous().view(torch.uint8).cpu().numpy()


def rough(rng, rows, cols):
    """Rows and columns of unequal size, so that scales differ from block to block."""
    return rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))) * np.exp(0.7 * rng.standard_normal((1, cols)))


def matrix(a, dtype, gap=0, shift=0, fill=float("nan")):
    """a as a view of rows that are gap elements longer, its first element `shift` elements into the buffer."""
    rows, cols = a.shape
    wide = torch.full((rows * (cols + gap) + shift,), fill, dtype=DT[dtype], device="cuda")
    x = wide[shift:].view(rows, cols + gap)[:, :cols]
    x.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda())
    return x


def operand(rng, rows, k, fmt, block_rows, ld=None, lds=None, fill=0xFF):
    """(codes, scales on the GPU, values in float64): every code and a range of scales, rows ld and lds bytes apart, what is
    between them filled (0xFF: NaN in both types, and as a scale)."""
    good = np.flatnonzero(np.isfinite(O.code_values(fmt)))
    c = rng.choice(good, (rows, k)).astype(np.uint8)
    s = rng.integers(120, 134, (-(-rows // block_rows), -(-k // 128))).astype(np.uint8)

    def place(a, step, ld):
        ld = ld or -(-a.shape[1] // step) * step
        wide = torch.full((a.shape[0], ld), fill, dtype=torch.uint8, device="cuda")
        wide[:, :a.shape[1]] = torch.from_numpy(a).cuda()
        return wide[:, :a.shape[1]]

    q, sc = place(c, 16, ld), place(s, 4, lds)
    return q.view(FP8[fmt]), sc.view(E8M0), O.values(c, s, fmt)


def product_bound(a, b, want, out):
    """Largest difference that the arithmetic explains.  Products of two codes are exact.  Each of the K / 64 (or K / 16) matrix
    instructions adds them to an accumulator: at most 64 roundings of partial sums inside it and one of the accumulator, each
    at most u times the sum of the absolute products so far; slices and an addend are a few more.  bfloat16 results: seven of
    eight consecutive products lose what is below 2^-13 of the largest, each at most that much."""
    a, b, want = (torch.from_numpy(np.ascontiguousarray(x)).cuda().abs() for x in (a, b, want))
    k = a.shape[1]
    bound = (k / 16 + 64 + 20) * U * (a @ b.T) + STORE[out] * want + 1e-30
    if out == "bf16":
        for g in range(0, k, 8):
            big = torch.zeros_like(want)
            for j in range(g, min(g + 8, k)):
                torch.maximum(big, a[:, j, None] * b[None, :, j], out=big)
            bound += 7 * 2.0 ** -13 * big
    return bound.cpu().numpy()
