"""Refusals of the vocabulary operators: every one precedes device work, so they run on a host without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2203_17189_amd as P
from paper_2203_17189_amd import binding as B

D = C.c_void_p(4096)  # never dereferenced
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


def _embed(**kw):
    return B._EmbedCfg(*{**dict(n_tokens=8, vocab=16, d_model=4, dtype=1, scale=1.0), **kw}.values())


def _top(**kw):
    return B._TopCfg(*{**dict(rows=8, ld=16, vocab=16, top_k=4, dtype=1), **kw}.values())


def _distill(**kw):
    return B._DistillCfg(*{**dict(rows=8, ld=16, vocab=16, top_k=4, dtype=1, temperature=1.0, soft_weight=0.5, z_loss=0.0), **kw}.values())


EMBED_BAD = [(dict(n_tokens=-1), SHAPE), (dict(vocab=0), SHAPE), (dict(d_model=0), SHAPE), (dict(scale=float("nan")), SHAPE),
             (dict(scale=float("inf")), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(n_tokens=1 << 24), UNSUPPORTED),
             (dict(vocab=(1 << 22) + 1), UNSUPPORTED), (dict(d_model=(1 << 16) + 1), UNSUPPORTED)]
ROWS_BAD = [(dict(rows=-1), SHAPE), (dict(vocab=1), SHAPE), (dict(ld=15), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=17), SHAPE),
            (dict(dtype=7), UNSUPPORTED), (dict(rows=1 << 24), UNSUPPORTED), (dict(ld=1000, vocab=1000, top_k=257), UNSUPPORTED),
            (dict(ld=1 << 23, vocab=(1 << 22) + 1), UNSUPPORTED), (dict(ld=(1 << 32) + 1), UNSUPPORTED)]
nan, inf = float("nan"), float("inf")
DISTILL_BAD = [(dict(temperature=v), SHAPE) for v in (0.0, -1.0, nan, inf, 1e-39)] + \
              [(dict(soft_weight=v), SHAPE) for v in (-0.1, 1.1, nan)] + [(dict(z_loss=v), SHAPE) for v in (-1e-4, nan, inf)]


@pytest.mark.parametrize("kw,rc", EMBED_BAD, ids=str)
def test_embed_refusals(kw, rc):
    L, c = P.lib(), _embed(**kw)
    assert L.t5_embed_fwd(C.byref(c), D, D, D, None) == rc
    assert L.t5_embed_bwd(C.byref(c), D, D, D, 0, D, 1 << 40, None) == rc
    assert L.t5_embed_bwd_workspace_bytes(C.byref(c)) == 0


def test_embed_nulls_empty_and_workspace():
    L, c, e = P.lib(), _embed(), _embed(n_tokens=0)
    assert L.t5_embed_fwd(None, D, D, D, None) == NULL
    for i in range(3):
        a = [D, D, D]
        a[i] = None
        assert L.t5_embed_fwd(C.byref(c), *a, None) == NULL
        assert L.t5_embed_bwd(C.byref(c), *a, 0, D, 1 << 40, None) == NULL
    assert L.t5_embed_bwd(C.byref(c), D, D, D, 0, None, 1 << 40, None) == NULL
    need = L.t5_embed_bwd_workspace_bytes(C.byref(c))
    assert need > 0 and L.t5_embed_bwd(C.byref(c), D, D, D, 0, D, need - 1, None) == WORKSPACE
    assert L.t5_embed_bwd(C.byref(c), D, D, D, 0, C.c_void_p(4096 + 128), 1 << 40, None) == WORKSPACE
    assert L.t5_embed_fwd(C.byref(e), None, None, None, None) == 0  # nothing to do
    assert L.t5_embed_bwd(C.byref(e), None, None, None, 1, None, 0, None) == 0


@pytest.mark.parametrize("kw,rc", ROWS_BAD, ids=str)
def test_row_refusals(kw, rc):
    L, t, d = P.lib(), _top(**kw), _distill(**kw)
    assert L.t5_top_logits(C.byref(t), D, D, D, None) == rc
    assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, 1 << 40, None) == rc
    assert L.t5_distill_workspace_bytes(C.byref(d)) == 0


@pytest.mark.parametrize("kw,rc", DISTILL_BAD, ids=str)
def test_distill_refusals(kw, rc):
    L, d = P.lib(), _distill(**kw)
    assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, 1 << 40, None) == rc
    assert L.t5_distill_workspace_bytes(C.byref(d)) == 0


def test_top_and_distill_nulls_and_workspace():
    L, t, d = P.lib(), _top(), _distill()
    assert L.t5_top_logits(None, D, D, D, None) == NULL
    for i in range(3):
        a = [D, D, D]
        a[i] = None
        assert L.t5_top_logits(C.byref(t), *a, None) == NULL
    assert L.t5_top_logits(C.byref(_top(rows=0)), None, None, None, None) == 0
    assert L.t5_distill_loss_and_grad(None, D, D, D, D, D, D, D, D, 1 << 40, None) == NULL
    for i in (0, 1, 2, 3, 4, 7):  # row losses and the gradient may be absent; targets only with soft_weight 1
        a = [D] * 8
        a[i] = None
        assert L.t5_distill_loss_and_grad(C.byref(d), *a, 1 << 40, None) == NULL, i
    need = L.t5_distill_workspace_bytes(C.byref(d))
    assert need > 0 and L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, need - 1, None) == WORKSPACE
    assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, C.c_void_p(4096 + 8), 1 << 40, None) == WORKSPACE


def test_wrappers_refuse_host_tensors_types_and_shapes():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 8)
    with pytest.raises(ValueError):
        P.t5_embed_fwd(i, f)
    with pytest.raises(ValueError):
        P.t5_embed_fwd(i, f.double())
    with pytest.raises(ValueError):
        P.t5_embed_bwd(i, f, 8)
    with pytest.raises(ValueError):
        P.t5_top_logits(f, 2)
    with pytest.raises(ValueError):
        P.t5_distill_loss_and_grad(f, None, f[:, :2], i.reshape(4, 1))


def test_model_refusals():
    import synth_inputs as SI
    from dataclasses import replace
    L = P.lib()
    sc = SI.StackConfig("r", replace(SI.CONFIGS["c1_tiny_f32"], causal=True), n_layers=1, vocab=300)
    ec = SI._encdec("r", 1, 2, 8, 8, 32, 2, 8, 48, 1, 1, 300)
    cs, ce = B._stack_cfg_struct(sc), B._encdec_cfg_struct(ec)
    ok = B._DistillOpts(8, 1.0, 0.5)
    lw = (B._Weights * 1)(B._Weights(*[4096] * 10))
    xw = (B._CrossWeights * 1)(B._CrossWeights(*[4096] * 5))
    ws, we = B._StackWeights(4096, 4096, lw, 4096, 4096), B._EncDecWeights(4096, 4096, lw, 4096, 4096, lw, xw, 4096, 4096)
    top_s = lambda k, tok=D, v=D, w=D, n=1 << 40, W=ws: L.t5_stack_top_logits(C.byref(cs), tok, C.byref(W), k, v, D, w, n, None)
    top_e = lambda k, tok=D, v=D, w=D, n=1 << 40, W=we: L.t5_encdec_top_logits(C.byref(ce), tok, D, C.byref(W), k, v, D, w, n, None)
    for top, q in ((top_s, lambda k: L.t5_stack_top_logits_workspace_bytes(C.byref(cs), k)),
                   (top_e, lambda k: L.t5_encdec_top_logits_workspace_bytes(C.byref(ce), k))):
        for k, rc in ((0, SHAPE), (301, SHAPE), (257, UNSUPPORTED)):
            assert top(k) == rc and q(k) == 0
        assert top(8, tok=None) == top(8, v=None) == top(8, w=None) == NULL
        assert q(8) > 0 and top(8, n=q(8) - 1) == WORKSPACE
    dis_s = lambda o, t=D, tl=D, n=1 << 40: L.t5_stack_distill_loss_and_grad(C.byref(cs), o and C.byref(o), D, t, tl, D, C.byref(ws), D, None, 0, D, n, None)
    dis_e = lambda o, t=D, tl=D, n=1 << 40: L.t5_encdec_distill_loss_and_grad(C.byref(ce), o and C.byref(o), D, D, t, tl, D, C.byref(we), D, None, 0, D, n, None)
    for dis, q in ((dis_s, lambda o: L.t5_stack_distill_workspace_bytes(C.byref(cs), o and C.byref(o))),
                   (dis_e, lambda o: L.t5_encdec_distill_workspace_bytes(C.byref(ce), o and C.byref(o)))):
        for o, rc in ((None, NULL), (B._DistillOpts(0, 1.0, 0.5), SHAPE), (B._DistillOpts(301, 1.0, 0.5), SHAPE),
                      (B._DistillOpts(257, 1.0, 0.5), UNSUPPORTED), (B._DistillOpts(8, 0.0, 0.5), SHAPE),
                      (B._DistillOpts(8, nan, 0.5), SHAPE), (B._DistillOpts(8, 1.0, 1.5), SHAPE)):
            assert dis(o) == rc and q(o) == 0
        assert dis(ok, t=None) == dis(ok, tl=None) == NULL
        assert dis(ok, n=q(ok) - 1) == WORKSPACE
        # the teacher's loss and the sorted embedding gradient need room of their own
    assert L.t5_stack_distill_workspace_bytes(C.byref(cs), C.byref(ok)) > L.t5_stack_workspace_bytes(C.byref(cs))
    assert L.t5_stack_top_logits_workspace_bytes(C.byref(cs), 8) < L.t5_stack_workspace_bytes(C.byref(cs))
