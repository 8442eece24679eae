"""Vocabulary operators on tensors that lie anywhere against 16-byte boundaries: the same bits as on aligned ones, with
guards around what is written."""
import numpy as np
import pytest
import torch

from test_gpu_distill import make
from test_gpu_embed_sorted import _tokens
from vocab_util import DT, dev, ints, rows_with_gap

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,ld,shift", [(9, 500, 600, 3), (9, 1003, 1016, 1), (530, 5000, 5008, 5), (9, 40000, 40016, 3), (140, 33000, 33040, 7),
                                                 (9, 140000, 140016, 1)])
def test_gradient_of_a_shifted_view(rows, vocab, ld, shift, dtype):
    """The gradient that is made by default lies at another phase than the logits; rows without a target among them."""
    import paper_2203_17189_amd as P
    x, tgt, t, ids = make(rows, vocab, 16, ld)
    wide, tx = rows_with_gap(x, dtype, ld, shift)
    args, more = (ints(tgt), dev(t), ints(ids)), dict(temperature=2.0, soft_weight=0.5, z_loss=1e-4)
    want = P.t5_distill_loss_and_grad(tx, *args, dlogits=torch.empty_like(wide)[:, shift:shift + vocab], **more)
    got = P.t5_distill_loss_and_grad(tx, *args, **more)
    assert got[2].data_ptr() % 16 == 0 and tx.data_ptr() % 16 != 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool(torch.all(got[2][ints(tgt) < 0] == 0))


# forms of the gradient: no sort, blocks merged, by digits of ten and of eight bits; widths odd, even, and below four
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out_at", [1, 2, 3])
@pytest.mark.parametrize("n,vocab,d", [(333, 100, 64), (333, 101, 67), (9001, 777, 64), (9001, 1001, 33), (9000, 333, 3), (16384, 12345, 7),
                                       (20000, 777, 64), (20000, 1001, 33), (20000, 31, 2), (40000, 300000, 5), (70001, 70000, 9)])
def test_gradient_of_a_table(n, vocab, d, out_at, dtype):
    import paper_2203_17189_amd as P
    rng = np.random.default_rng(n + d)
    tok = ints(_tokens(n, vocab, "two" if n % 2 else "skewed", rng))
    dx = dev(rng.standard_normal(n * d + 4), dtype)
    dx_at = out_at if dtype == "f32" else 2 * out_at - 1
    odd = torch.empty(n * d + 8, dtype=DT[dtype], device="cuda")[dx_at:dx_at + n * d].view(n, d)
    odd.copy_(dx[:n * d].view(n, d))
    want = P.t5_embed_bwd(tok, dx[:n * d].view(n, d), vocab, scale=0.5)
    buf = torch.full((vocab * d + 8,), 7.0, device="cuda")
    out = buf[out_at:out_at + vocab * d].view(vocab, d)
    P.t5_embed_bwd(tok, odd, vocab, scale=0.5, dtable=out)
    assert torch.equal(out, want)
    P.t5_embed_bwd(tok, odd, vocab, scale=0.5, dtable=out, accumulate=True)
    assert torch.equal(out, 2 * want)
    out.fill_(7.0)
    assert bool(torch.all(buf == 7.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 3, 7, 8, 33, 64, 770])
def test_lookup(d, dtype):
    import paper_2203_17189_amd as P
    rng = np.random.default_rng(d)
    n, vocab = 501, 97
    tok = ints(rng.integers(-3, vocab + 3, n))
    table = dev(rng.standard_normal((vocab, d)), dtype)
    for at in (1, 3):
        odd = torch.empty(vocab * d + 8, dtype=DT[dtype], device="cuda")[at:at + vocab * d].view(vocab, d)
        odd.copy_(table)
        buf = torch.full((n * d + 8,), 7.0, dtype=DT[dtype], device="cuda")
        x = buf[at + 1:at + 1 + n * d].view(n, d)
        P.t5_embed_fwd(tok, odd, scale=1.5, x=x)
        assert torch.equal(x, P.t5_embed_fwd(tok, table, scale=1.5))
        x.fill_(7.0)
        assert bool(torch.all(buf == 7.0))
