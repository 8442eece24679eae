"""Pins of the float64 definitions of the vocabulary operators: closed forms, torch autograd in float64, differences."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as VO

RNG = np.random.default_rng(0)


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    tok = np.array([[3, 0, 3], [7, -2, 9]])  # ids outside [0, 8) are clamped
    table, dx = RNG.standard_normal((8, 5)), RNG.standard_normal((2, 3, 5))
    lhs = np.sum(VO.embed_fwd(tok, table, 0.7) * dx)
    assert np.isclose(lhs, np.sum(table * VO.embed_bwd(tok, dx, 8, 0.7)))
    d = VO.embed_bwd(tok, dx, 8, 0.7)
    assert np.allclose(d[7], 0.7 * (dx[1, 0] + dx[1, 2])) and np.all(d[[1, 2, 4, 5, 6]] == 0)


def test_top_logits_order():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0], [0.0, np.nan, -0.0, np.inf, np.nan]])
    v, i = VO.top_logits(x, 4)
    assert i.tolist() == [[1, 2, 4, 0], [1, 4, 3, 0]]
    assert v[0].tolist() == [3, 3, 2, 1]


def _case(rows=6, vocab=11, k=4):
    x, t = RNG.standard_normal((rows, vocab)) * 2, RNG.standard_normal((rows, k)) * 2
    ids = np.stack([RNG.permutation(vocab)[:k] for _ in range(rows)])
    ids[1, 2], ids[2, :], ids[3, 1] = -1, -1, ids[3, 0]  # a hole, no entry at all, an id twice
    tgt = RNG.integers(0, vocab, rows)
    tgt[4] = -1
    return x, tgt, t, ids


@pytest.mark.parametrize("tau,soft,z", [(1.0, 1.0, 0.0), (2.0, 0.5, 1e-2), (0.7, 0.0, 1e-3)])
def test_distill_gradient_by_differences(tau, soft, z):
    x, tgt, t, ids = _case()
    loss, row, g = VO.distill_loss(x, tgt, t, ids, tau, soft, z)
    assert np.all(g[4] == 0) and row[4] == 0
    for r, v in [(0, 3), (1, ids[1, 0]), (2, 5), (3, ids[3, 0]), (5, tgt[5])]:
        e = np.zeros_like(x)
        e[r, v] = 1e-5
        num = (VO.distill_loss(x + e, tgt, t, ids, tau, soft, z)[0] - VO.distill_loss(x - e, tgt, t, ids, tau, soft, z)[0]) / 2e-5
        assert abs(num - g[r, v]) < 1e-8


def test_distill_against_torch_in_64_bits():
    x, tgt, t, ids = _case()
    keep = np.array([0, 5])  # whole lists, targets present
    loss, _, g = VO.distill_loss(x[keep], tgt[keep], t[keep], ids[keep], 2.0, 0.5, 0.0)
    tx = torch.tensor(x[keep], requires_grad=True)
    p = torch.zeros(2, 11, dtype=torch.float64).scatter_(1, torch.tensor(ids[keep]), torch.softmax(torch.tensor(t[keep]) / 2, 1))
    want = 0.5 * torch.nn.functional.cross_entropy(tx, torch.tensor(tgt[keep])) + \
        0.5 * 4 * torch.nn.functional.kl_div(torch.log_softmax(tx / 2, 1), p, reduction="batchmean")
    want.backward()
    assert np.isclose(loss, want.item()) and np.allclose(g, tx.grad.numpy())


def test_distill_ends():
    x, tgt, t, ids = _case()
    assert VO.distill_loss(x, np.full(6, -1), t, ids, 1.0, 0.5)[0] == 0
    # soft weight 0: plain cross-entropy; a teacher equal to the student over the whole vocabulary: no loss, no gradient
    ce = np.mean([VO._lse(x[r]) - x[r, tgt[r]] for r in range(6) if tgt[r] >= 0])
    assert np.isclose(VO.distill_loss(x, tgt, t, ids, 3.0, 0.0)[0], ce)
    all_ids = np.tile(np.arange(11), (6, 1))
    loss, _, g = VO.distill_loss(x, None, x, all_ids, 2.5)
    assert abs(loss) < 1e-14 and np.abs(g).max() < 1e-15
    # masked logits: probability 0, no gradient; an entry there costs infinitely much
    xm = x.copy()
    xm[:, 7] = -np.inf
    i7 = np.where(ids == 7, -1, ids)
    loss, _, g = VO.distill_loss(xm, None, t, i7)
    assert np.isfinite(loss) and np.all(g[:, 7] == 0)
    i7[0, 0] = 7
    assert VO.distill_loss(xm, None, t, i7)[0] == np.inf
