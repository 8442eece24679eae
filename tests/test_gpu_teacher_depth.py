"""Top logits of models of more layers than the forward pass keeps outputs of, against the oracle, with whatever the workspace held before."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth_inputs as SI
from oracle import t5_oracle as O
from parity_util import TOL_F32, to_np
from test_gpu_parity_stack import _ec_upload, _upload

pytestmark = pytest.mark.gpu
K = 6


def _check(logits, v, i):
    tol = TOL_F32[0] * np.maximum(np.abs(logits).max(-1, keepdims=True), 1.0)
    assert np.all(np.abs(np.take_along_axis(logits, i.cpu().numpy(), -1) - to_np(v)) <= tol)
    assert np.all(np.abs(-np.sort(-logits, -1)[..., :K] - to_np(v)) <= tol)


def _junk(nbytes):
    return torch.full((nbytes,), 0x7F, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("layers", [1, 2, 5])
def test_stack(layers, tied):
    import ctypes as C
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    b = SI.BlockConfig("depth", 190 + layers, batch=2, seq=19, d_model=32, n_heads=2, d_kv=8, d_ff=48, dtype="f32", causal=True)
    sc = SI.StackConfig("depth", b, n_layers=layers, vocab=64, tied_logits=tied)
    w = SI.make_stack_weights(sc)
    SI.make_stack_random_scales(sc, w)
    tokens, targets = SI.make_tokens(sc)
    _, saved = O.stack_loss(sc, tokens, targets, w)
    dw, tt, _ = _upload(sc, w, tokens, targets)
    need = B.lib().t5_stack_top_logits_workspace_bytes(C.byref(B._stack_cfg_struct(sc)), K)
    ws = _junk(need + 4096)
    v, i = P.t5_stack_top_logits(sc, tt, dw, K, workspace=ws[:need])
    _check(saved["logits"], v, i)
    assert bool((ws[need:] == 0x7F).all())


@pytest.mark.parametrize("enc,dec,tied", [(1, 4, False), (4, 1, True), (3, 3, False)])
def test_pair(enc, dec, tied):
    import ctypes as C
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    ec = replace(SI._encdec("depth", 196, 2, 20, 13, 32, 2, 8, 48, enc, dec, 64, block=dict(dtype="f32")), tied_logits=tied)
    w = SI.make_encdec_weights(ec)
    SI.make_encdec_random_scales(ec, w)
    et, dt, tg = SI.make_encdec_tokens(ec)
    _, saved = O.encdec_loss(ec, et, dt, tg, w)
    dw, det, ddt, _ = _ec_upload(ec, w, et, dt, tg)
    need = B.lib().t5_encdec_top_logits_workspace_bytes(C.byref(B._encdec_cfg_struct(ec)), K)
    ws = _junk(need + 4096)
    v, i = P.t5_encdec_top_logits(ec, det, ddt, dw, K, workspace=ws[:need])
    _check(saved["logits"], v, i)
    assert bool((ws[need:] == 0x7F).all())
