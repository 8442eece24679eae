"""The vocabulary operators captured into a graph and replayed, on a stream of their own, two at a time with a workspace
each, and refusals that need device tensors."""
import numpy as np
import pytest
import torch

from vocab_util import dev, ints

pytestmark = pytest.mark.gpu


def _inputs(seed, n, vocab, d, rows, lvocab, k, dtype):
    rng = np.random.default_rng(seed)
    return dict(tok=ints(vocab * rng.random(n) ** 2), dx=dev(rng.standard_normal((n, d)), dtype),
                x=dev(rng.standard_normal((rows, lvocab)) * 3, dtype), tgt=ints(rng.integers(-1, lvocab, rows)),
                t=dev(rng.standard_normal((rows, k))), ids=ints(rng.integers(-1, lvocab, (rows, k))))


# forms of the gradient: no sort, blocks merged, by digits (twice); forms of the rows: one wavefront, one workgroup, parts
SHAPES = [(500, 700, 40, 300, 700, 9), (3000, 700, 520, 20, 40000, 64), (17000, 300, 24, 5, 140000, 33), (70000, 40000, 8, 1100, 5000, 16)]


def _run(P, s, vocab, k, out):
    g = P.t5_embed_bwd(s["tok"], s["dx"], vocab, scale=0.5, dtable=out.get("g"), workspace=out.get("w1"))
    v, i = P.t5_top_logits(s["x"], k, values=out.get("v"), ids=out.get("i"))
    l, r, dl = P.t5_distill_loss_and_grad(s["x"], s["tgt"], s["t"], s["ids"], temperature=1.5, soft_weight=0.5, z_loss=1e-3,
                                          loss=out.get("l"), row_loss=out.get("r"), dlogits=out.get("dl"), workspace=out.get("w2"))
    e = P.t5_embed_fwd(s["tok"], g, scale=2.0, x=out.get("e"))
    return dict(g=g, v=v, i=i, l=l, r=r, dl=dl, e=e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,rows,lvocab,k", SHAPES)
def test_replays_equal_eager_calls(n, vocab, d, rows, lvocab, k, dtype):
    import paper_2203_17189_amd as P
    s = _inputs(0, n, vocab, d, rows, lvocab, k, dtype)
    bytes_ = lambda: torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")  # (nothing may rely on zeros)
    out = dict(_run(P, s, vocab, k, {}), w1=bytes_(), w2=bytes_())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(P, s, vocab, k, out)
    for rep in range(3):
        other = _inputs(rep + 1, n, vocab, d, rows, lvocab, k, dtype)
        for name in s:
            s[name].copy_(other[name])
        for name in ("g", "v", "l", "r", "dl", "e"):
            out[name].fill_(7.0)
        graph.replay()
        want = _run(P, s, vocab, k, {})
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(out[name], want[name]), (rep, name)


def test_two_streams_at_once():
    import paper_2203_17189_amd as P
    n, vocab, d, rows, lvocab, k = SHAPES[2]
    ss = [_inputs(q, n, vocab, d, rows, lvocab, k, "bf16") for q in range(2)]
    want = [_run(P, s, vocab, k, {}) for s in ss]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ss]
    for _ in range(3):
        got = []
        for s, q in zip(ss, streams):
            with torch.cuda.stream(q):
                got.append(_run(P, s, vocab, k, {}))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for name in b:
                assert torch.equal(a[name], b[name]), name


def test_refusals_of_the_wrappers():
    import paper_2203_17189_amd as P
    x = torch.zeros(6, 16, device="cuda")
    i32 = torch.zeros(6, dtype=torch.int32, device="cuda")
    ids, t = torch.zeros(6, 2, dtype=torch.int32, device="cuda"), torch.zeros(6, 2, device="cuda")
    bad = [lambda: P.t5_top_logits(x.t(), 2), lambda: P.t5_top_logits(x[:, ::2], 2), lambda: P.t5_top_logits(x[:1].expand(6, 16), 2),
           lambda: P.t5_top_logits(x.half(), 2), lambda: P.t5_top_logits(x, 2, ids=ids.long()), lambda: P.t5_top_logits(x[0], 2),
           lambda: P.t5_embed_fwd(i32.long(), x), lambda: P.t5_embed_fwd(i32, x.t()), lambda: P.t5_embed_fwd(i32.cpu(), x),
           lambda: P.t5_embed_bwd(i32[:5], x, 9), lambda: P.t5_embed_bwd(i32, x, 9, dtable=x),
           lambda: P.t5_distill_loss_and_grad(x, i32[:5], t, ids), lambda: P.t5_distill_loss_and_grad(x, i32, t[:, :1], ids),
           lambda: P.t5_distill_loss_and_grad(x, i32, t.double(), ids), lambda: P.t5_distill_loss_and_grad(x, i32, t, ids, dlogits=x[:, :8]),
           lambda: P.t5_distill_loss_and_grad(x, i32, t, ids, dlogits=x.bfloat16())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: P.t5_top_logits(x, 17), lambda: P.t5_distill_loss_and_grad(x, None, t, ids, soft_weight=0.5),
              lambda: P.t5_distill_loss_and_grad(x, i32, t, ids, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
              lambda: P.t5_embed_bwd(i32, x, 9, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
              lambda: P.t5_embed_fwd(i32, x, scale=float("nan")), lambda: P.t5_embed_bwd(i32, x, 2 ** 32 + 8),
              lambda: P.t5_embed_bwd(i32, x, 0), lambda: P.t5_top_logits(x, 2 ** 32 + 2), lambda: P.t5_top_logits(x, 0),
              lambda: P.t5_top_logits(x, -3)):
        with pytest.raises(P.T5Error):
            f()


def test_numbers_of_other_kinds():
    """numpy's numbers are taken as Python's; a fraction is no size."""
    import paper_2203_17189_amd as P
    x = torch.arange(96.0, device="cuda").view(6, 16) / 50
    i32 = torch.arange(6, dtype=torch.int32, device="cuda")
    v, i = P.t5_top_logits(x, np.int64(3))
    assert torch.equal(i, P.t5_top_logits(x, 3)[1])
    two = np.float32(2.0)
    a = P.t5_distill_loss_and_grad(x, i32, v, i, temperature=two, soft_weight=np.float64(0.5), z_loss=0)
    b = P.t5_distill_loss_and_grad(x, i32, v, i, temperature=2.0, soft_weight=0.5)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert torch.equal(P.t5_embed_fwd(i32, x, scale=two), 2 * x)
    assert torch.equal(P.t5_embed_bwd(i32, x, np.int32(9), scale=two), P.t5_embed_bwd(i32, x, 9, scale=2.0))
    for f in (lambda: P.t5_top_logits(x, 2.5), lambda: P.t5_embed_bwd(i32, x, 9.5)):
        with pytest.raises(TypeError):
            f()
