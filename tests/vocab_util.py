"""Inputs and error bounds of the GPU tests of the vocabulary operators."""
import numpy as np
import torch

U = 2.0 ** -24  # half a step of float32, relative
STORE = {"f32": U, "bf16": 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(DT[dtype])


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def rows_with_gap(a, dtype, ld, shift=0, fill=float("nan")):
    """[rows, vocab] as a view of rows ld elements apart whose other elements hold `fill`; shift: first element's offset."""
    rows, vocab = a.shape
    wide = torch.full((rows, ld), fill, dtype=DT[dtype], device="cuda")
    wide[:, shift:shift + vocab] = dev(a, dtype)
    return wide, wide[:, shift:shift + vocab]


def distill_bounds(x, targets, t, ids, tau, soft, z, dtype, row, grad):
    """Largest differences that float32 arithmetic explains, for row losses and gradients of the mean.

    exp2 of a rounded product: relative error |d| log2(e) ln2 u per rounding of d = x - m and of the product (2 |d| u in
    all) and one unit of the exponential (2 u, with slack).  A sum over V in 64-wide lanes and workgroups of 256 is at most
    V / 256 + 16 additions deep.  So log sum exp is off by at most e = (2 R + V / 256 + 24) u absolutely, R the range of
    the finite logits of the row (times 1 / tau), and a softmax value by 2 (e + ...) relatively.  The rest are a few
    roundings of the terms themselves."""
    fin = np.where(np.isfinite(x), x, 0.0)
    R = (fin.max(1) - fin.min(1)) * max(1.0, 1.0 / tau)
    V = x.shape[1]
    on = (ids >= 0) & (ids < V) & np.isfinite(t)
    tf = np.where(on, t, 0.0)
    Rt = (tf.max(1) - tf.min(1)) / tau
    e = (2 * R + V / 256 + 24) * U
    et = (2 * Rt + 32) * U
    size = np.abs(fin).max(1)
    lse = size + np.log(V)
    mag = (1 - soft) * (lse + size) + soft * tau * tau * (lse / min(tau, 1.0) * 2 + Rt + 8) + z * lse ** 2
    row_tol = (1 - soft) * e + 2 * z * lse * e + soft * tau * tau * (e + 2 * et * (1 + R + Rt + np.log(V))) + 8 * U * mag
    # every part of a gradient element is at most k / n in size; parts are off relatively by 2 e (softmax) or 2 et (entries)
    counted = np.ones(len(x), bool) if targets is None else (targets >= 0) & (targets < V)
    n = max(1, int(counted.sum()))
    part = (1 - soft + 2 * z * lse + soft * tau)[:, None] / n
    q = np.exp(fin - fin.max(1, keepdims=True)) if True else None
    q = np.where(np.isfinite(x), q, 0.0)
    q = q / q.sum(1, keepdims=True)
    qt = np.exp((fin - fin.max(1, keepdims=True)) / tau)
    qt = np.where(np.isfinite(x), qt, 0.0)
    qt = qt / qt.sum(1, keepdims=True)
    here = np.zeros_like(x)
    for r in range(len(x)):
        np.add.at(here[r], ids[r][on[r]], 1.0)
        if targets is not None and counted[r]:
            here[r, targets[r]] += 1.0
    grad_tol = part * ((q + qt) * (2 * e[:, None] + 8 * U) + np.minimum(here, 1.0) * (2 * et + 24 * U)[:, None])
    grad_tol = grad_tol + (STORE[dtype] + 2 * U) * np.abs(grad) + 1e-37
    return row_tol, grad_tol
