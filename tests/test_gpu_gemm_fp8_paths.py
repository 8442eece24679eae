"""Every kernel of the product of quantised matrices (tests/fp8_paths.py) with every pair of types, values that are not finite,
scales from end to end, rows with NaN between them, workspaces that held something else, captured and on streams."""
import ctypes as C

import pytest
import torch

import paper_2203_17189_amd as P
from paper_2203_17189_amd import binding as B
from fp8_paths import IDS, LAYERS, SHAPES, SHARED, bound, layer_products, operand, path
from fp8_util import DT
from test_gpu_train8_layer import layer, same, snapshot, train_step

pytestmark = pytest.mark.gpu
PARTS = [s for s in SHAPES if s[4] & SHARED]
every = pytest.mark.parametrize("m,n,k,out,kernel", SHAPES, ids=IDS)
in_parts = pytest.mark.parametrize("m,n,k,out,kernel", PARTS, ids=["%dx%dx%d-%s" % s[:4] for s in PARTS])


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def workspace(m, n, k, out, fill):
    ld, lds = -(-k // 16) * 16, -(-k // 512) * 4
    need = P.lib().t5_gemm_fp8_workspace_bytes(C.byref(B._GemmFp8Cfg(m, n, k, ld, ld, n, lds, lds, 2, 2, 1, 1, 0 if out == "f32" else 1, 0)))
    assert need > 0
    return torch.full((need,), fill, dtype=torch.uint8, device="cuda")


@every
@pytest.mark.parametrize("ta,tb,ra,rb", [("e4m3", "e4m3", 1, 128), ("e4m3", "e5m2", 128, 1), ("e5m2", "e4m3", 1, 1), ("e5m2", "e5m2", 128, 128)])
def test_types_and_strides(m, n, k, out, kernel, ta, tb, ra, rb):
    assert path(m, n, k, out) == kernel
    g = gen(m + n + k)
    a, sa, va = operand(g, m, k, ta, ra, gap=48)
    b, sb, vb = operand(g, n, k, tb, rb, gap=48)
    want = torch.matmul(va, vb.t().contiguous())
    far = bound(va, vb, want, out)
    wide = torch.full((m, n + 3), 7.0, dtype=DT[out], device="cuda")
    c = wide[:, :n]
    assert P.t5_gemm_fp8(a, sa, b, sb, out=c) is c
    assert bool(((c.double() - want).abs() <= far).all()) and bool((wide[:, n:] == 7.0).all())
    if out == "f32":
        c0 = torch.randn(m, n, device="cuda", generator=g) * want.abs().max().float()
        c.copy_(c0)
        P.t5_gemm_fp8(a, sa, b, sb, out=c, accumulate=True)
        # (the sum is rounded once more, to float32)
        assert bool(((c.double() - want - c0.double()).abs() <= far + 2.0 ** -24 * (want + c0.double()).abs() * 2).all())
        assert bool((wide[:, n:] == 7.0).all())


@every
def test_what_is_not_finite_stays_in_its_row_or_column(m, n, k, out, kernel):
    g = gen(1)
    a, sa, _ = operand(g, m, k, "e4m3", 1)
    b, sb, _ = operand(g, n, k, "e5m2", 1)
    u8 = lambda t: t.view(torch.uint8)  # noqa: E731
    one, two = min(1, m - 1), min(2, m - 1)
    u8(a)[one, k - 1] = 0x7F            # NaN, in the last block
    u8(sa)[two, (k - 1) // 128] = 255
    u8(b)[5, 0] = 0x7C                  # infinity
    u8(b)[n - 1, k // 2] = 0xFE         # NaN
    u8(sb)[n - 2, 0] = 255
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[[one, two]] = True
    bad[:, [5, n - 2, n - 1]] = True
    c = P.t5_gemm_fp8(a, sa, b, sb, out_dtype=DT[out])
    assert torch.equal(~c.isfinite(), bad)
    assert bool(c[[one, two]].isnan().all()) and bool(c[:, n - 2:].isnan().all())


@every
def test_scales_from_end_to_end(m, n, k, out, kernel):
    """Ones with powers far apart.  Sums of ones are exact; with float32 results an element below 2^-126 may count as zero."""
    one = lambda rows: torch.full((rows, -(-k // 16) * 16), 0x38, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :k]  # noqa: E731
    byte = lambda rows, e: torch.full((rows, -(-k // 512) * 4), e, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)[:, :-(-k // 128)]  # noqa: E731
    a, b = one(m), one(n)
    for ea, eb in ((0, 254), (254, 0), (1, 254), (254, 1), (127, 127), (100, 60), (254, 130)):
        want = (torch.tensor(float(k), dtype=torch.float64) * 2.0 ** (ea + eb - 254)).to(DT[out]).item()
        c = P.t5_gemm_fp8(a, byte(m, ea), b, byte(n, eb), out_dtype=DT[out])
        assert bool((c == want).all()) or (out == "f32" and min(ea, eb) == 0 and bool((c == 0).all())), (ea, eb, c[0, 0].item(), want)


@in_parts
def test_parts_from_workspaces_that_held_something_else(m, n, k, out, kernel):
    g = gen(3)
    a, sa, _ = operand(g, m, k, "e4m3", 1)
    b, sb, _ = operand(g, n, k, "e4m3", 128)
    first = P.t5_gemm_fp8(a, sa, b, sb, out_dtype=DT[out])
    for fill in (0x7F, 0xFF, 0x00):
        assert torch.equal(P.t5_gemm_fp8(a, sa, b, sb, out_dtype=DT[out], workspace=workspace(m, n, k, out, fill)), first)


@in_parts
def test_parts_in_graphs_and_on_streams(m, n, k, out, kernel):
    """Two graphs that share a workspace, replayed in turn, and two that have one each, on a stream each; other inputs in the
    same buffers and another content of the workspace at every replay."""
    def inputs(seed):
        g = gen(seed)
        a, sa, _ = operand(g, m, k, "e5m2", 1)
        b, sb, _ = operand(g, n, k, "e4m3", 1)
        return [a, sa, b, sb]

    sets = [inputs(10), inputs(11)]
    eager = lambda s: P.t5_gemm_fp8(*s, out_dtype=DT[out])  # noqa: E731
    for s in sets:
        eager(s)
    for shared in (True, False):
        works = [workspace(m, n, k, out, 0xFF)] * 2 if shared else [workspace(m, n, k, out, 0xFF) for _ in range(2)]
        graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for s, w in zip(sets, works):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                outs.append(P.t5_gemm_fp8(*s, out_dtype=DT[out], workspace=w))
            graphs.append(graph)
        for rep in range(3):
            for i, s in enumerate(sets):
                for t, u in zip(s, inputs(100 * rep + 20 + i)):
                    t.view(torch.uint8).copy_(u.view(torch.uint8))
            for w in works:
                w.fill_(0x7F if rep % 2 else 0xFF)
            torch.cuda.synchronize()
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(torch.cuda.current_stream() if shared else stream):
                    graph.replay()
            torch.cuda.synchronize()
            for s, c in zip(sets, outs):
                assert torch.equal(c, eager(s))


@pytest.mark.parametrize("tokens,d_in,d_out,which,tile", LAYERS)
def test_layers_with_products_in_parts(tokens, d_in, d_out, which, tile):
    """A captured step, replayed on other inputs, and a step on another stream, equal eager ones."""
    assert path(*layer_products(tokens, d_in, d_out)[which]) == tile | SHARED
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
    for rep in range(3):
        new = layer(tokens, d_in, d_out, seed=rep + 1)
        for t in (s, e):
            for k in ("x", "target"):
                t[k].copy_(new[k])
        work.fill_(0xFF if rep % 2 else 0x7F)
        graph.replay()
        same(snapshot(s, o), snapshot(e, train_step(e, 4)))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = snapshot(s, train_step(s, 5))
    stream.synchronize()
    same(got, snapshot(e, train_step(e, 5)))
