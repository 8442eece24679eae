"""Distillation loss at the ends of its ranges: temperatures next to nothing, entries on logits of the type's lowest value."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as VO
from vocab_util import U, dev, host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 40000, 140000])
@pytest.mark.parametrize("tau", [0.5, 1e-3, 1e-30, 1e-37, 4.3e-39])
def test_entries_far_below_the_largest_logit(tau, vocab, dtype):
    """One entry a row, so p = 1, on logits 0, 45 and some 3e38 below the row's largest: the row's loss is
    T^2 (log sum exp((x - m) / T) - (x - m) / T) = T (m - x) + T^2 log(count of m), a finite number though (m - x) / T is none.
    Three roundings, and for T below 1.2e-38 steps of 1.4e-45 (2^-149)."""
    import paper_2203_17189_amd as P
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    x = np.full((3, vocab), -50.0)
    x[:, 5], x[:, 9], x[:, vocab - 2] = 3.0, -42.0, low
    ids = np.array([[5], [9], [vocab - 2]])
    t = np.zeros((3, 1))
    _, row, g = P.t5_distill_loss_and_grad(dev(x, dtype), None, dev(t), ints(ids), temperature=tau)
    tau = float(np.float32(tau))
    _, want, wg = VO.distill_loss(host(dev(x, dtype)), None, t, ids, tau)
    assert np.all(np.isfinite(want)) and want[1] == pytest.approx(45 * tau, rel=1e-9)
    assert np.all(np.abs(host(row) - want) <= 4 * U * want + 4 * 2.0 ** -149), (host(row), want)
    # the gradient, T (q - [v = id]) / rows: q is 1 at the largest logit alone (exp(-45 / 0.5) is 1e-39)
    tol = (2.0 ** -8 if dtype == "bf16" else 4 * U) * np.abs(wg) + 1e-37
    assert np.all(np.abs(host(g) - wg) <= tol)
