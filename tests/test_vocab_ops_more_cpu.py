"""Further refusals and sizes of the vocabulary operators and of the models that call them; no device work."""
import ctypes as C
from dataclasses import replace

import pytest
import torch

import paper_2203_17189_amd as P
import synth_inputs as SI
from paper_2203_17189_amd import binding as B
from test_vocab_ops_cpu import D, SHAPE, WORKSPACE, _distill


@pytest.mark.parametrize("t,ok", [(4e-39, False), (4.2e-39, False), (4.3e-39, True), (1e-37, True), (3e38, True)])
def test_temperatures_whose_exponentials_overflow(t, ok):
    """Exponentials are powers of two of log2(e) x / T: that factor has to be a number, not only 1 / T (below 2.9e-39 even
    that is none)."""
    L, d = P.lib(), _distill(temperature=t)
    if ok:
        assert L.t5_distill_workspace_bytes(C.byref(d)) > 0
    else:
        assert L.t5_distill_workspace_bytes(C.byref(d)) == 0
        assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, 1 << 40, None) == SHAPE


@pytest.mark.parametrize("out_ld,rc", [(-1, SHAPE), (15, SHAPE), ((1 << 32) + 1, 3)])
def test_strides_of_the_gradient(out_ld, rc):
    L, d = P.lib(), _distill(dlogits_ld=out_ld)
    assert L.t5_distill_workspace_bytes(C.byref(d)) == 0
    assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, 1 << 40, None) == rc


def test_a_gradient_over_the_logits_keeps_their_stride():
    L, d = P.lib(), _distill(dlogits_ld=17)
    assert L.t5_distill_workspace_bytes(C.byref(d)) > 0
    assert L.t5_distill_loss_and_grad(C.byref(d), D, D, D, D, D, D, D, D, 1 << 40, None) == SHAPE


def _stack(n_layers, tied=False):
    sc = SI.StackConfig("m", SI.BlockConfig("m", 1, 2, 64, 128, 2, 64, 256, causal=True), n_layers=n_layers, vocab=1024, tied_logits=tied)
    return P.lib().t5_stack_top_logits_workspace_bytes(C.byref(B._stack_cfg_struct(sc)), 8)


def _pair(n_enc, n_dec, tied=False):
    ec = replace(SI._encdec("m", 1, 2, 64, 32, 128, 2, 64, 256, n_enc, n_dec, 1024), tied_logits=tied)
    return P.lib().t5_encdec_top_logits_workspace_bytes(C.byref(B._encdec_cfg_struct(ec)), 8)


def test_a_teacher_needs_room_for_one_layer():
    """However deep the teacher is; and for no copy of its output matrix where that is the embedding, which the logits' GEMM
    reads as it lies."""
    assert _stack(1) == _stack(2) == _stack(24) > 0
    assert _pair(1, 1) == _pair(24, 1) == _pair(1, 24) == _pair(24, 24) > 0
    assert _stack(2) - _stack(2, tied=True) == _pair(2, 2) - _pair(2, 2, tied=True) == 1024 * 128 * 2


def test_model_workspaces_off_256_bytes():
    L, odd, n = P.lib(), C.c_void_p(4096 + 128), 1 << 40
    sc = SI.StackConfig("r", replace(SI.CONFIGS["c1_tiny_f32"], causal=True), n_layers=1, vocab=300)
    ec = SI._encdec("r", 1, 2, 8, 8, 32, 2, 8, 48, 1, 1, 300)
    cs, ce, o = B._stack_cfg_struct(sc), B._encdec_cfg_struct(ec), B._DistillOpts(8, 1.0, 0.5)
    lw = (B._Weights * 1)(B._Weights(*[4096] * 10))
    xw = (B._CrossWeights * 1)(B._CrossWeights(*[4096] * 5))
    ws, we = B._StackWeights(4096, 4096, lw, 4096, 4096), B._EncDecWeights(4096, 4096, lw, 4096, 4096, lw, xw, 4096, 4096)
    assert L.t5_stack_top_logits(C.byref(cs), D, C.byref(ws), 8, D, D, odd, n, None) == WORKSPACE
    assert L.t5_encdec_top_logits(C.byref(ce), D, D, C.byref(we), 8, D, D, odd, n, None) == WORKSPACE
    assert L.t5_stack_distill_loss_and_grad(C.byref(cs), C.byref(o), D, D, D, D, C.byref(ws), D, None, 0, odd, n, None) == WORKSPACE
    assert L.t5_encdec_distill_loss_and_grad(C.byref(ce), C.byref(o), D, D, D, D, D, C.byref(we), D, None, 0, odd, n, None) == WORKSPACE


def test_tensors_of_a_model_on_another_device():
    t, other = torch.zeros(2), torch.device("cpu", 7)  # (two devices of one kind, as two GPUs are)
    for tree in (t, dict(a=t), dict(layers=[dict(b=None), dict(b=t)])):
        with pytest.raises(ValueError):
            B._check_devices(other, tree, "weights")
        B._check_devices(t.device, tree, "weights")
    # what a caller keeps beside its weights: nothing, names, numbers, tensors on the host
    B._check_devices(torch.device("cuda", 0), dict(name="model", step=3, note=None, host=t, more=(1, "x")), "weights")
    B._check_devices(other, None, "grads")
