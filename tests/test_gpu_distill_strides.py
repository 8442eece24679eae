"""Gradients of the distillation loss whose rows are not as far apart as those of the logits, or lie elsewhere against
16-byte boundaries: the same bits as in a gradient with the logits' strides, and nothing written between the rows."""
import numpy as np
import pytest
import torch

from test_gpu_distill import make
from vocab_util import dev, ints, rows_with_gap

pytestmark = pytest.mark.gpu
MORE = dict(temperature=2.0, soft_weight=0.5, z_loss=1e-4)


def _same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [500, 1003, 40000])
def test_last_positions_of_sequences(vocab, dtype):
    """Rows of [batch, seq, vocab] that are a sequence apart: the gradient takes memory for its own rows alone."""
    import paper_2203_17189_amd as P
    batch, seq = 6, 50
    x, tgt, t, ids = make(batch, vocab, 8, vocab)
    whole = torch.zeros(batch, seq, vocab, dtype=dev(x[:1, :1], dtype).dtype, device="cuda")
    whole[:, -1] = dev(x, dtype)
    args = (ints(tgt), dev(t), ints(ids))
    want = P.t5_distill_loss_and_grad(whole[:, -1], *args, dlogits=torch.empty_like(whole)[:, -1], **MORE)
    got = P.t5_distill_loss_and_grad(whole[:, -1], *args, **MORE)
    assert _same(got, want)
    assert got[2].untyped_storage().nbytes() < batch * (vocab + 8) * whole.element_size()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,ld,out_ld,out_shift", [(500, 500, 512, 0), (500, 516, 501, 0), (1003, 1003, 1011, 0), (40000, 40000, 40003, 3),
                                                      (40000, 40016, 40008, 8), (140001, 140001, 140001, 1), (140001, 140008, 140002, 0)])
def test_a_row_stride_of_its_own(vocab, ld, out_ld, out_shift, dtype):
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(9, vocab, 16, ld)
    _, tx = rows_with_gap(x, dtype, ld)
    args = (ints(tgt), dev(t), ints(ids))
    want = P.t5_distill_loss_and_grad(tx, *args, dlogits=torch.empty(9, ld, dtype=tx.dtype, device="cuda")[:, :vocab], **MORE)
    buf = torch.full((9 * out_ld + out_shift + vocab,), 3.0, dtype=tx.dtype, device="cuda")
    out = buf[out_shift:out_shift + 9 * out_ld].view(9, out_ld)[:, :vocab]
    got = P.t5_distill_loss_and_grad(tx, *args, dlogits=out, **MORE)
    assert got[2] is out and _same(got, want)
    out.fill_(3.0)
    assert torch.all(buf == 3)


def test_refusals():
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(4, 64, 4, 1)
    wide = torch.zeros(4, 80, device="cuda")
    args = (ints(tgt), dev(t), ints(ids))
    over = wide.flatten()[:4 * 64].view(4, 64)  # starts with the logits, its rows elsewhere
    with pytest.raises(P.T5Error):
        P.t5_distill_loss_and_grad(wide[:, :64], *args, dlogits=over, **MORE)
    for bad in (wide[:, :63], wide[:3, :64], wide[:, :64].bfloat16(), wide[:, :64].cpu(), wide[:, ::2][:, :40]):
        with pytest.raises(ValueError):
            P.t5_distill_loss_and_grad(dev(x), *args, dlogits=bad, **MORE)
