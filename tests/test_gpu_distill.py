"""Distillation loss and gradient against the float64 definition, with bounds from float32 arithmetic (vocab_util)."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as VO
from vocab_util import dev, distill_bounds, host, ints, rows_with_gap

pytestmark = pytest.mark.gpu


def make(rows, vocab, k, seed, spread=2.5):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, vocab)) * spread
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)])
    t = np.sort(rng.standard_normal((rows, k)) * 2, 1)[:, ::-1].copy()
    tgt = rng.integers(0, vocab, rows)
    if rows > 3:
        tgt[1], tgt[2] = -1, vocab + 3
        ids[0, :] = -1                       # no entry
        ids[3, k // 2:] = vocab + np.arange(k - k // 2)  # a short list
        t[3, k // 2:] = np.nan               # whose rest is never used
    if rows > 6 and k > 2:
        ids[4, 1] = ids[4, 0]                # an id twice
        t[5, 1] = -np.inf                    # an entry of probability 0
        ids[6, 0] = tgt[6]                   # the target among the entries
        t[6, :] = t[6, 0]
    return x, tgt, t, ids


def check(P, x, tgt, t, ids, tau, soft, z, dtype, tx=None, out=None):
    tx = dev(x, dtype) if tx is None else tx
    hx = host(tx)
    loss, row, g = P.t5_distill_loss_and_grad(tx, None if tgt is None else ints(tgt), dev(t), ints(ids), temperature=tau,
                                              soft_weight=soft, z_loss=z, dlogits=out)
    tau, soft, z = (float(np.float32(v)) for v in (tau, soft, z))
    ht = np.float32(t).astype(np.float64)
    wl, wr, wg = VO.distill_loss(hx, tgt, ht, ids, tau, soft, z)
    rt, gt = distill_bounds(hx, tgt, ht, ids, tau, soft, z, dtype, wr, wg)
    assert np.all(np.abs(host(row) - wr) <= rt), np.max(np.abs(host(row) - wr) / rt)
    assert np.all(np.abs(host(g) - wg) <= gt), np.max(np.abs(host(g) - wg) / gt)
    n = max(1, len(wr) if tgt is None else int(((tgt >= 0) & (tgt < hx.shape[1])).sum()))
    depth = len(wr) / 1024 + 32
    assert abs(float(loss) - wl) <= rt.sum() / n + depth * 2.0 ** -24 * np.abs(wr).sum() / n
    return loss, row, g


CASES = [(1, 2, 1), (1, 7, 7), (4, 33, 8), (7, 256, 16), (9, 509, 8), (8, 2048, 64), (8, 2056, 256), (7, 4100, 100),
         (16, 32128, 64), (8, 32776, 32), (8, 65537, 40), (7, 131072, 128), (300, 700, 5), (260, 33001, 9), (1030, 40, 3), (513, 5000, 20)]
MIX = [(1.0, 1.0, 0.0), (2.0, 0.5, 1e-4), (0.7, 0.9, 1e-2), (1.0, 0.0, 1e-3), (4.0, 1.0, 0.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau,soft,z", MIX)
@pytest.mark.parametrize("rows,vocab,k", CASES)
def test_loss_and_gradient(rows, vocab, k, tau, soft, z, dtype):
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(rows, vocab, k, rows + vocab + k)
    args = (x, tgt, t, ids, tau, soft, z, dtype)
    loss, row, g = check(P, *args)
    assert torch.all(row[ints(tgt) < 0] == 0) and torch.all(g[ints(tgt) < 0] == 0)
    more = dict(temperature=tau, soft_weight=soft, z_loss=z)
    tx = dev(x, dtype)
    only = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), want_grads=False, **more)
    assert only[2] is None and torch.equal(only[0], loss) and torch.equal(only[1], row)
    # in place, and the same bits again
    l2, r2, g2 = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), dlogits=tx, **more)
    assert g2 is tx and torch.equal(l2, loss) and torch.equal(r2, row) and torch.equal(g2, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k,mix", [(520, 1600, 7, 0), (520, 1601, 100, 2), (513, 3500, 5, 1), (512, 9001, 33, 2), (512, 17003, 16, 1),
                                              (256, 66001, 8, 4), (300, 131073, 3, 2)])
def test_many_rows(rows, vocab, k, mix, dtype):
    """Rows enough for workgroups that share a compute unit, of every size of theirs."""
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(rows, vocab, k, vocab)
    tx = dev(x, dtype)
    _, _, g = check(P, x, tgt, t, ids, *MIX[mix], dtype, tx=tx.clone())
    tau, soft, z = MIX[mix]
    P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), temperature=tau, soft_weight=soft, z_loss=z, dlogits=tx)
    assert torch.equal(tx, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k", [(5, 40, 3), (12, 5001, 20), (6, 33000, 64)])
def test_without_targets(rows, vocab, k, dtype):
    import paper_2203_17189_amd as P
    x, _, t, ids = make(rows, vocab, k, 7)
    check(P, x, None, t, ids, 1.5, 1.0, 1e-3, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,ld,shift", [(2048, 2056, 0), (2048, 2056, 8), (4000, 4003, 0), (4000, 4100, 3), (333, 1000, 1),
                                            (40000, 40008, 0), (70000, 70001, 1)])
def test_rows_with_a_longer_stride_keep_the_rest(vocab, ld, shift, dtype):
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(8, vocab, 16, ld)
    wide, tx = rows_with_gap(x, dtype, ld, shift)
    before = wide.clone()
    out = torch.full_like(wide, 3.0)
    _, _, g = check(P, x, tgt, t, ids, 2.0, 0.5, 1e-4, dtype, tx=tx, out=out[:, shift:shift + vocab])
    assert torch.equal(wide[~wide.isnan()], before[~before.isnan()])
    assert torch.all(out[:, :shift] == 3) and torch.all(out[:, shift + vocab:] == 3)
    P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), temperature=2.0, soft_weight=0.5, z_loss=1e-4, dlogits=tx)
    assert torch.equal(tx, g)
    assert torch.all(wide[:, :shift].isnan()) and torch.all(wide[:, shift + vocab:].isnan())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [509, 4096, 40000])
def test_masked_logits(vocab, dtype):
    """Columns of -inf and of the type's lowest value: probability 0, gradient 0."""
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(9, vocab, 8, 3)
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    dead = np.unique(np.concatenate([np.arange(0, vocab, 3), [vocab - 1]]))
    x[:, dead] = -np.inf
    x[7, dead] = low
    ids = np.where(np.isin(ids, dead), -1, ids)
    tgt = np.where(np.isin(tgt, dead), -1, tgt)
    tx = dev(x, dtype)
    loss, row, g = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), temperature=0.5, soft_weight=0.5)
    assert torch.all(g[:, torch.from_numpy(dead).cuda()] == 0)
    hx = host(tx)
    wl, wr, wg = VO.distill_loss(np.where(hx <= low, -np.inf, hx), tgt, np.float32(t).astype(float), ids, 0.5, 0.5)
    alive = np.where(hx <= low, -np.inf, hx)
    rt, gt = distill_bounds(alive, tgt, np.float32(t).astype(float), ids, 0.5, 0.5, 0.0, dtype, wr, wg)
    assert np.all(np.abs(host(row) - wr) <= rt) and np.all(np.abs(host(g) - wg) <= gt) and np.isfinite(float(loss))
    # an entry of positive probability on a masked logit: infinitely wrong, with a finite gradient
    ids[8, 0], tgt[8] = dead[0], (dead[0] + 1) % vocab
    loss, row, g = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), soft_weight=0.5)
    assert float(row[8]) == np.inf and bool(torch.isfinite(g[8].float()).all()) and float(loss) == np.inf
    # with soft_weight 0 the teacher does not matter
    loss, row, g = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t * np.nan), ints(ids), soft_weight=0.0)
    assert np.isfinite(float(row[8])) and bool(torch.isfinite(g.float()).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [509, 4096, 40000, 140000])
def test_far_from_zero(vocab, dtype):
    """Rows shifted far from 0, and rows of nothing but the type's lowest value (uniform: loss log V, gradient 1 / V)."""
    import paper_2203_17189_amd as P
    x, _, t, ids = make(6, vocab, 4, 21)
    tgt = np.array([5, 6, 7, 8, 9, 10])
    ids[:] = np.arange(4)
    t[3, 2:] = t[3, 0]
    x[1] += 3000.0
    x[2] -= 3000.0
    x[4] = float(torch.finfo(torch.bfloat16).min)
    x[5] = float(torch.finfo(torch.bfloat16).max)
    for tau, soft in ((1.0, 0.5), (0.5, 0.5), (2.0, 0.5), (2.0, 1.0), (1.0, 0.0)):
        tx = dev(x, dtype)
        _, row, g = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), temperature=tau, soft_weight=soft)
        hx, ht = host(tx), np.float32(t).astype(float)
        _, wr, wg = VO.distill_loss(hx, tgt, ht, ids, tau, soft)
        shifted = hx - hx.max(1, keepdims=True)   # the loss without z does not depend on the shift
        rt, gt = distill_bounds(shifted, tgt, ht, ids, tau, soft, 0.0, dtype, wr, wg)
        assert np.all(np.abs(host(row) - wr) <= rt), (tau, soft, np.abs(host(row) - wr) / rt)
        assert np.all(np.abs(host(g) - wg) <= gt)


@pytest.mark.parametrize("vocab", [100, 4096, 40000])
def test_padding_rows_hide_whatever_they_hold(vocab):
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(6, vocab, 4, 11)
    tgt[:] = [3, -1, 5, -7, vocab, 1]
    x[1], x[3, 5], x[4] = np.nan, np.inf, -np.inf
    t[1], t[3, 0] = np.nan, np.inf
    tx = dev(x, "bf16")
    loss, row, g = P.t5_distill_loss_and_grad(tx, ints(tgt), dev(t), ints(ids), soft_weight=0.5, z_loss=1e-3)
    off = torch.tensor([1, 3, 4], device="cuda")
    assert bool(torch.isfinite(loss)) and torch.all(row[off] == 0) and torch.all(g[off] == 0)
    none, row, g = P.t5_distill_loss_and_grad(tx, ints(np.full(6, -1)), dev(t), ints(ids), soft_weight=0.5)
    assert float(none) == 0 and torch.all(row == 0) and torch.all(g == 0)


@pytest.mark.parametrize("vocab", [100, 4096, 40000])
def test_bad_entries_and_logits_show(vocab):
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(8, vocab, 4, 12)
    tgt[:] = 1
    ids[:] = np.arange(4)
    t[0, 1], t[1, 2], x[2, 9], x[3] = np.nan, np.inf, np.nan, -np.inf
    t[4, :] = -np.inf                       # entries without any probability: no soft term
    t[5, :] = [np.nan] + [-np.inf] * 3
    _, row, g = P.t5_distill_loss_and_grad(dev(x), ints(tgt), dev(t), ints(ids), soft_weight=0.5)
    bad = row.isnan().tolist()
    assert bad == [True, True, True, True, False, True, False, False]
    _, hard, hg = P.t5_distill_loss_and_grad(dev(x), ints(tgt), dev(t), ints(np.full_like(ids, -1)), soft_weight=0.5)
    assert torch.equal(hard[4], row[4]) and torch.equal(hg[4], g[4])


def test_empty():
    import paper_2203_17189_amd as P
    z = torch.zeros(0, 10, device="cuda")
    i = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    loss, row, g = P.t5_distill_loss_and_grad(z, None, torch.zeros(0, 2, device="cuda"), i)
    assert float(loss) == 0 and row.shape == (0,) and g.shape == (0, 10)


@pytest.mark.parametrize("rows,vocab", [(5, 300), (6, 40000)])
def test_gradient_by_differences(rows, vocab):
    """The kernel's own loss, differenced along the kernel's own gradient: float32 row losses are good to about 1e-6, a step
    that moves the loss by about 1e-2 leaves the quotient good to 1e-3."""
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(rows, vocab, 8, 5)
    more = dict(temperature=2.0, soft_weight=0.5, z_loss=1e-3)
    f = lambda a: host(P.t5_distill_loss_and_grad(dev(a), ints(tgt), dev(t), ints(ids), want_grads=False, **more)[1]).sum()  # noqa: E731
    g = host(P.t5_distill_loss_and_grad(dev(x), ints(tgt), dev(t), ints(ids), **more)[2])
    n = int(((tgt >= 0) & (tgt < vocab)).sum())
    g = g * n                                # of the sum of the rows
    h = 5e-3 / np.sum(g * g)
    num = (f(x + h * g) - f(x - h * g)) / (2 * h)
    assert abs(num - np.sum(g * g)) <= 2e-3 * np.sum(g * g)


def test_rows_beyond_32_bit_offsets():
    """520 rows, 2^23 + 8 elements apart, the gradient over the logits."""
    import paper_2203_17189_amd as P
    rows, vocab, k = 520, 1000, 8
    x, tgt, t, ids = make(rows, vocab, k, 4)
    wide, tx = rows_with_gap(x, "bf16", (1 << 23) + 8, fill=7.0)
    args = (ints(tgt), dev(t), ints(ids))
    more = dict(temperature=2.0, soft_weight=0.5)
    want = P.t5_distill_loss_and_grad(tx.contiguous(), *args, **more)
    loss, row, g = P.t5_distill_loss_and_grad(tx, *args, dlogits=tx, **more)
    assert torch.equal(loss, want[0]) and torch.equal(row, want[1]) and torch.equal(g.contiguous(), want[2])
    assert bool((wide[:, vocab:] == 7.0).all())
