"""A linear layer trained in 8 bits, as the operators are used together: activations and weights quantised, the forward
product, both gradients, the optimizer's step with 8-bit states; eager, on a stream of its own, and captured."""
import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
from oracle import fp8_oracle as O
from fp8_util import E8M0, codes, host, product_bound

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def value(q, s, fmt):
    return O.values(codes(q), codes(s), fmt)


def layer(tokens, d_in, d_out, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    n = d_out * d_in
    zeros = lambda k, dt: torch.zeros(k, dtype=torch.uint8, device="cuda").view(dt)  # noqa: E731
    return dict(x=rn(tokens, d_in).bfloat16(), target=rn(tokens, d_out), w=rn(d_out, d_in) * d_in ** -0.5, dw=torch.zeros(d_out, d_in, device="cuda"),
                m=zeros(n, torch.float8_e4m3fn), v=zeros(n, torch.float8_e4m3fn), ms=zeros(-(-n // 128), E8M0), vs=zeros(-(-n // 128), E8M0),
                copy=torch.zeros(d_out, d_in, dtype=torch.bfloat16, device="cuda"))


def train_step(s, step, workspace=None):
    """One step of the layer; every tensor it made on the way."""
    xq, xs, xt, xts = P.t5_quantize_fp8(s["x"], "e4m3", transposed=True)
    wq, ws, wt, wts = P.t5_quantize_fp8(s["w"], "e4m3", block_rows=128, transposed=True)
    y = P.t5_gemm_fp8(xq, xs, wq, ws, workspace=workspace)
    dy = ((y.float() - s["target"]) * (1.0 / y.shape[0])).bfloat16()
    gq, gs, gt, gts = P.t5_quantize_fp8(dy, "e5m2", transposed=True)
    dx = P.t5_gemm_fp8(gq, gs, wt, wts, workspace=workspace)
    P.t5_gemm_fp8(gt, gts, xt, xts, out=s["dw"], accumulate=True, workspace=workspace)
    P.adamw_step_multi([dict(param=s["w"], grad=s["dw"], m=s["m"], v=s["v"], m_scale=s["ms"], v_scale=s["vs"], bf16_copy_out=s["copy"],
                             weight_decay=0.1)], step=step, seed=77, **HP)
    return dict(xq=xq, xs=xs, xt=xt, xts=xts, wq=wq, ws=ws, wt=wt, wts=wts, y=y, dy=dy, gq=gq, gs=gs, gt=gt, gts=gts, dx=dx)


@pytest.mark.parametrize("tokens,d_in,d_out", [(1, 64, 48), (33, 130, 257), (300, 512, 384), (2049, 300, 200)])
def test_steps_against_float64(tokens, d_in, d_out):
    s = layer(tokens, d_in, d_out)
    for step in (1, 2, 3):
        s["dw"].zero_()
        w, state = host(s["w"]), [s[k].clone() for k in ("m", "v", "ms", "vs")]
        o = train_step(s, step)
        for m, q, sc, fmt, rows in ((host(s["x"]), "xq", "xs", "e4m3", 1), (host(s["x"]).T, "xt", "xts", "e4m3", 1), (w, "wq", "ws", "e4m3", 128),
                                    (w.T, "wt", "wts", "e4m3", 128), (host(o["dy"]), "gq", "gs", "e5m2", 1), (host(o["dy"]).T, "gt", "gts", "e5m2", 1)):
            wq, wsc = O.quantize(m, fmt, rows)
            assert (codes(o[q]) == wq).all() and (codes(o[sc]) == wsc).all()
        for got, a, sa, fa, b, sb, out in ((o["y"], "xq", "xs", "e4m3", "wq", "ws", "bf16"), (o["dx"], "gq", "gs", "e5m2", "wt", "wts", "bf16"),
                                           (s["dw"], "gt", "gts", "e5m2", "xt", "xts", "f32")):
            va, vb = value(o[a], o[sa], fa), value(o[b], o[sb], "e4m3")
            assert (np.abs(host(got) - va @ vb.T) <= product_bound(va, vb, va @ vb.T, out)).all()
        n = w.size
        m, r = (O.code_values("e4m3")[codes(q)] * np.repeat(2.0 ** (codes(sc) - 127.0), 128)[:n] for q, sc in ((state[0], state[2]), (state[1], state[3])))
        want, _, _ = O.adamw(w.reshape(-1), host(s["dw"]).reshape(-1), m, r * r, step=step, weight_decay=0.1, **HP)
        np.testing.assert_allclose(host(s["w"]).reshape(-1), want, rtol=4 * 2.0 ** -24, atol=HP["lr"] * 40 * 2.0 ** -24)
        assert torch.equal(s["copy"], s["w"].bfloat16())


def test_gradients_are_the_layers():
    """Values that 8 bits hold exactly: the three products are the layer's forward pass and its gradients, by differences of
    L = sum(y * g) in float64."""
    rng = np.random.default_rng(5)
    pick = lambda *shape: rng.choice([0.0, 1.0, -1.0, 0.5, -2.0, 3.0], shape)  # noqa: E731
    x, w, g = pick(130, 70), pick(90, 70), pick(130, 90)
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    xq, xs, xt, xts = P.t5_quantize_fp8(dev(x), transposed=True)
    wq, ws, wt, wts = P.t5_quantize_fp8(dev(w), block_rows=128, transposed=True)
    gq, gs, gt, gts = P.t5_quantize_fp8(dev(g), "e5m2", transposed=True)
    f32 = torch.float32
    assert (host(P.t5_gemm_fp8(xq, xs, wq, ws, out_dtype=f32)) == x @ w.T).all()
    dx = host(P.t5_gemm_fp8(gq, gs, wt, wts, out_dtype=f32))
    dw = host(P.t5_gemm_fp8(gt, gts, xt, xts, out_dtype=f32))
    loss = lambda x, w: float(((x @ w.T) * g).sum())  # noqa: E731
    for _ in range(30):
        i, j, o = rng.integers(130), rng.integers(70), rng.integers(90)
        dxe, dwe = np.zeros_like(x), np.zeros_like(w)
        dxe[i, j] = dwe[o, j] = 0.25
        assert abs((loss(x + dxe, w) - loss(x - dxe, w)) / 0.5 - dx[i, j]) < 1e-9
        assert abs((loss(x, w + dwe) - loss(x, w - dwe)) / 0.5 - dw[o, j]) < 1e-9


def snapshot(s, o):
    out = {k: v.clone() for k, v in o.items()}
    out.update({k: s[k].clone() for k in ("w", "dw", "m", "v", "ms", "vs", "copy")})
    return out


def same(a, b):
    for k in a:
        assert torch.equal(a[k].contiguous().view(torch.uint8) if a[k].element_size() == 1 else a[k],
                           b[k].contiguous().view(torch.uint8) if b[k].element_size() == 1 else b[k]), k


# few rows; tiles with shared rounds (a workspace); many tiles
SHAPES = [(7, 200, 136), (520, 3100, 330), (2100, 520, 1100)]


@pytest.mark.parametrize("tokens,d_in,d_out", SHAPES)
def test_replays_equal_eager_steps(tokens, d_in, d_out):
    """A captured step, replayed on other inputs, with eager steps between; workspaces that held something else before."""
    s, e = layer(tokens, d_in, d_out), layer(tokens, d_in, d_out)
    work = torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")
    train_step(s, 4, work)
    train_step(e, 4)
    torch.cuda.synchronize()
    keep = {k: v.clone() for k, v in s.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = train_step(s, 4, work)
    for k, v in keep.items():
        s[k].copy_(v)
    for rep in range(4):
        new = layer(tokens, d_in, d_out, seed=rep + 1)
        for t in (s, e):
            for k in ("x", "target"):
                t[k].copy_(new[k])
        work.fill_(0xFF if rep % 2 else 0x7F)
        graph.replay()
        eager = snapshot(e, train_step(e, 4))
        same(snapshot(s, o), eager)


def test_two_graphs_with_a_workspace_each_and_a_stream_each():
    sets = [layer(520, 3100, 330, seed=k) for k in range(2)]
    eager = [layer(520, 3100, 330, seed=k) for k in range(2)]
    works = [torch.zeros(1 << 28, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for t in sets:
        train_step(t, 2, works[0])
    for t in eager:
        train_step(t, 2)
    torch.cuda.synchronize()
    keep = [{k: v.clone() for k, v in t.items()} for t in sets]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for t, w in zip(sets, works):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(train_step(t, 2, w))
        graphs.append(graph)
    for t, k in zip(sets, keep):
        for name in t:
            t[name].copy_(k[name])
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for t, o, e in zip(sets, outs, eager):
            same(snapshot(t, o), snapshot(e, train_step(e, 2)))


def test_on_another_stream():
    s, e = layer(520, 3100, 330), layer(520, 3100, 330)
    want = snapshot(e, train_step(e, 1))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        o = train_step(s, 1)
        got = snapshot(s, o)
    stream.synchronize()
    same(got, want)
