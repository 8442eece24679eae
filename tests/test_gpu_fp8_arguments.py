"""Arguments of the operators of training in 8 bits that are no rows of memory, or not where the others are."""
import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
from paper_2203_17189_amd import binding as B
from oracle import fp8_oracle as O
from fp8_util import codes, host

pytestmark = pytest.mark.gpu


def not_strided(x):
    return [x.to_sparse_csr(), x.to_sparse_csc(), x.to_sparse_bsr((2, 2)), x.to_sparse(), torch.nested.nested_tensor([x[:1], x[1:]]),
            torch.nested.nested_tensor([x[:1], x[1:]], layout=torch.jagged)]


@pytest.mark.filterwarnings("ignore")
def test_sparse_and_nested_tensors_are_refused():
    """Asked for its strides or its memory, such a tensor throws: that has to become an exception of Python's."""
    x = torch.randn(4, 512, device="cuda")
    q, s, _, _ = P.t5_quantize_fp8(x)
    out = torch.zeros(4, 4, device="cuda")
    flat = lambda: torch.zeros(8, device="cuda")  # noqa: E731
    for t in not_strided(x):
        with pytest.raises(ValueError):
            P.t5_quantize_fp8(t)
        for at in range(4):
            args = [q, s, q, s]
            args[at] = t
            with pytest.raises(ValueError):
                P.t5_gemm_fp8(*args)
        for name in ("param", "grad", "m", "v"):
            entry = dict(param=flat(), grad=flat(), m=flat(), v=flat())
            entry[name] = t
            with pytest.raises(ValueError):
                P.adamw_step_multi([entry], step=1, lr=1e-3)
    for t in not_strided(out):
        with pytest.raises(ValueError):
            P.t5_gemm_fp8(q, s, q, s, out=t)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("cols", [1, 2, 3, 4])
def test_few_columns_of_rows_of_four(cols, block_rows):
    """A matrix whose memory ends with its last element."""
    rows = 130
    x = torch.zeros(4 * (rows - 1) + cols, device="cuda").as_strided((rows, cols), (4, 1))
    x.copy_(torch.from_numpy(np.random.default_rng(cols).standard_normal((rows, cols)).astype(np.float32)))
    out = P.t5_quantize_fp8(x, block_rows=block_rows, transposed=True)
    for a, q, s in ((host(x), *out[:2]), (host(x).T, *out[2:])):
        wq, ws = O.quantize(a, "e4m3", block_rows)
        assert (codes(q) == wq).all() and (codes(s) == ws).all()
    if block_rows == 1:
        assert (codes(P.t5_quantize_fp8(x)[0]) == codes(out[0])).all()


def _calls():
    """Calls of every kind, right and wrong, as functions of nothing."""
    u8, e4, e8 = torch.uint8, torch.float8_e4m3fn, torch.float8_e8m0fnu
    x = torch.randn(130, 300, device="cuda")
    wide = torch.randn(130, 307, device="cuda")
    unclear = torch.zeros(2, dtype=torch.bool)
    tight = torch.zeros(4 * 3 + 1, device="cuda").as_strided((4, 1), (4, 1))
    quant = [x, x.bfloat16(), wide[:, :300], wide[:, 5:], x.t(), x[::2], x[:1], x[:0], x[:, :1], x[:, :0], x[0], x[None], x.double(), x.half(), x[:1].expand(5, 300),
             x[:, ::2], x.cpu(), tight, torch.zeros(0, device="cuda"), torch.nn.Parameter(x)]
    for t in quant:
        for kw in ({}, dict(q_dtype="e5m2", block_rows=128, transposed=True), dict(rows=False), dict(rows=0, transposed=1, q_dtype=torch.float8_e5m2)):
            yield lambda t=t, kw=kw: P.t5_quantize_fp8(t, **kw)
    for kw in (dict(block_rows=2), dict(block_rows=1.0), dict(block_rows=np.int64(128)), dict(block_rows="1"), dict(rows=unclear), dict(transposed=unclear), dict(q_dtype="e3m4"),
               dict(q_dtype=torch.uint8), dict(rows=None)):
        yield lambda kw=kw: P.t5_quantize_fp8(x, **kw)
    (a, sa), (b, sb) = P.t5_quantize_fp8(x)[:2], P.t5_quantize_fp8(x[:70], block_rows=128)[:2]
    one, s1 = P.t5_quantize_fp8(x[:1])[:2]
    loose = torch.zeros(130, 320, dtype=u8, device="cuda").view(e4)[:, :300]
    tight_q = torch.zeros(130 * 304 - 4, dtype=u8, device="cuda").as_strided((130, 300), (304, 1)).view(e4)
    tight_s = torch.zeros(130 * 4 - 1, dtype=u8, device="cuda").as_strided((130, 3), (4, 1)).view(e8)
    short = torch.zeros(300, dtype=u8, device="cuda").view(e4)[None]  # a row that ends inside a piece
    pairs = [(a, sa), (b, sb), (one, s1), (loose, sa), (a, sa[:2]), (a, sa[:3]), (a, sa[:, :2]), (a[:, :299], sa), (a[:0], sa[:0]), (a.view(u8), sa), (a, sa.view(u8)), (a.cpu(), sa),
             (a, sa.cpu()), (a.t(), sa), (a[0], sa), (tight_q, sa), (a, tight_s), (short, s1), (a[:, 1:], sa), (a[:, :256], sa[:, :2]), (a[::2], sa[::2]), (a[:128], sb)]
    for p in pairs:
        yield lambda p=p: P.t5_gemm_fp8(*p, b, sb)
        yield lambda p=p: P.t5_gemm_fp8(a, sa, *p, out_dtype=torch.float32)
    f, h = torch.zeros(130, 70, device="cuda"), torch.zeros(130, 70, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(130, 75, device="cuda")
    for out in (f, h, w[:, :70], w[:, 5:], w, f[:129], f.t(), f.half(), f.cpu(), f[0], f.view(-1), w.view(-1)[1:].as_strided((130, 70), (69, 1)), torch.zeros(70, 130, device="cuda").t(),
                f.to_sparse(), None):
        for kw in ({}, dict(accumulate=True), dict(out_dtype=torch.float32), dict(out_dtype=torch.float16)):
            yield lambda out=out, kw=kw: P.t5_gemm_fp8(a, sa, b, sb, out=out, **kw)
    for kw in (dict(accumulate=unclear, out=f), dict(accumulate=1, out=f.clone()), dict(accumulate=0, out=f), dict(accumulate=None)):
        yield lambda kw=kw: P.t5_gemm_fp8(a, sa, b, sb, **kw)


def _outcome(call):
    try:
        out = call()
    except Exception as e:
        return type(e), getattr(e, "status", None)
    out = out if isinstance(out, tuple) else (out,)
    return [None if t is None else (t.dtype, tuple(t.shape), tuple(t.stride()), codes(t) if t.element_size() == 1 else host(t.clone())) for t in out]


@pytest.mark.filterwarnings("ignore")
def test_native_and_python_checks_agree(monkeypatch):
    """Ordinary calls are read by native code, what that leaves by the binding: the same calls pass, with the same results, and
    the same are refused, with the same errors, when the native readers leave everything."""
    native = [_outcome(c) for c in _calls_seeded()]
    real = B._LISTS
    left = []
    nothing = lambda *a: left.append(a) or None  # noqa: E731
    monkeypatch.setattr(B, "_LISTS", (nothing, real[1], nothing, *real[3:]))
    python = [_outcome(c) for c in _calls_seeded()]
    assert len(native) == len(python) == 20 * 4 + 9 + 22 * 2 + 15 * 4 + 4 and len(left) > 100
    passed = 0
    for i, (n, p) in enumerate(zip(native, python)):
        assert type(n) is type(p), (i, n, p)
        if isinstance(n, tuple):
            assert n == p, (i, n, p)
            continue
        passed += 1
        for u, v in zip(n, p):
            assert (u is None) == (v is None) and (u is None or u[:2] == v[:2] and (u[1][0] <= 1 or u[2][0] == v[2][0]) and np.array_equal(u[3], v[3], equal_nan=True)), i
    assert 60 < passed < len(native) - 60


def _calls_seeded():
    torch.manual_seed(7)
    return list(_calls())
