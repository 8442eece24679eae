"""Students whose rows of logits are cut into parts, whose statistics and picked logits lie in the model's workspace: short
batches, and a last chunk of logits that is cut where the chunks before it are not.  What the workspace held before and what
lies behind it play no part."""
import ctypes as C
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth_inputs as SI
from oracle import t5_oracle as O
from oracle import vocab_oracle as VO
from parity_util import TOL_F32
from test_gpu_parity_stack import _ec_errs, _ec_upload, _grads_np, _stack_errs, _upload
from vocab_util import dev, ints

pytestmark = pytest.mark.gpu
K, TAU, SOFT = 12, 2.0, 0.5


def _entries(tokens, vocab, seed):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, vocab, (*tokens.shape, K))
    ids[..., -1] = np.where(rng.random(tokens.shape) < 0.3, -1, ids[..., -1])
    return np.float32(rng.standard_normal(ids.shape) * 2).astype(np.float64), ids


def _guarded(need):
    return torch.full((need + (1 << 20),), 0x7F, dtype=torch.uint8, device="cuda")


def _compare(errs, loss, want):
    assert abs(float(loss) - want) <= 1e-5 * max(1.0, abs(want)), (float(loss), want)
    for name, e in errs.items():
        assert e[0] <= TOL_F32[0], (name, e)


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("vocab", [16385, 20000])
def test_few_tokens(vocab, tied):
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    b = SI.BlockConfig("parts", 210, batch=3, seq=21, d_model=32, n_heads=2, d_kv=8, d_ff=48, dtype="f32", causal=True)
    sc = SI.StackConfig("parts", b, n_layers=1, vocab=vocab, tied_logits=tied, z_loss=1e-3)
    w = SI.make_stack_weights(sc)
    SI.make_stack_random_scales(sc, w)
    tokens, targets = SI.make_tokens(sc, ignore_fraction=0.15)
    t, ids = _entries(tokens, vocab, vocab)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    cs, o = B._stack_cfg_struct(sc), B._DistillOpts(K, TAU, SOFT)
    need = P.lib().t5_stack_distill_workspace_bytes(C.byref(cs), C.byref(o))
    ws = _guarded(need)
    loss, g = P.t5_stack_distill_loss_and_grad(sc, tt, tg, dev(t), ints(ids), dw, temperature=TAU, soft_weight=SOFT, workspace=ws[:need])
    _, saved = O.stack_loss(sc, tokens, targets, w)
    want, _, dl = VO.distill_loss(saved["logits"].reshape(-1, vocab), targets.reshape(-1), t.reshape(-1, K), ids.reshape(-1, K),
                                  TAU, SOFT, sc.z_loss)
    _compare(_stack_errs(sc, _grads_np(g), O.stack_loss_grad(sc, w, saved, dl.reshape(saved["logits"].shape)), tokens, targets), loss, want)
    assert bool((ws[need:] == 0x7F).all())


def test_only_the_last_chunk_is_cut():
    """16400 tokens: 16384 whole rows, then 16 in parts.  Loss and gradients come from the positions with a target alone, so the
    oracle takes the sequences that hold one, some of either chunk."""
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    b = SI.BlockConfig("parts_chunk", 212, batch=1025, seq=16, d_model=8, n_heads=1, d_kv=8, d_ff=8, dtype="f32", causal=True)
    vocab, some = 17000, [0, 517, 1023, 1024]
    sc = SI.StackConfig("parts_chunk", b, n_layers=1, vocab=vocab, z_loss=1e-3)
    w = SI.make_stack_weights(sc)
    SI.make_stack_random_scales(sc, w)
    tokens, targets = SI.make_tokens(sc, ignore_fraction=0.15)
    targets[[q for q in range(1025) if q not in some]] = -1
    t, ids = _entries(tokens, vocab, 5)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    cs, o = B._stack_cfg_struct(sc), B._DistillOpts(K, TAU, SOFT)
    need = P.lib().t5_stack_distill_workspace_bytes(C.byref(cs), C.byref(o))
    ws = _guarded(need)
    loss, g = P.t5_stack_distill_loss_and_grad(sc, tt, tg, dev(t), ints(ids), dw, temperature=TAU, soft_weight=SOFT, workspace=ws[:need])
    few = replace(sc, block=replace(b, batch=len(some)))
    ftok, ftgt, ft, fids = tokens[some], targets[some], t[some].reshape(-1, K), ids[some].reshape(-1, K)
    _, saved = O.stack_loss(few, ftok, ftgt, w)
    want, _, dl = VO.distill_loss(saved["logits"].reshape(-1, vocab), ftgt.reshape(-1), ft, fids, TAU, SOFT, sc.z_loss)
    got = _grads_np(g)
    _compare(_stack_errs(few, got, O.stack_loss_grad(few, w, saved, dl.reshape(saved["logits"].shape)), ftok, ftgt), loss, want)
    assert np.all(got["embedding"][np.setdiff1d(np.arange(vocab), ftok)] == 0)
    assert bool((ws[need:] == 0x7F).all())


def test_pair():
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    vocab = 18001
    ec = SI._encdec("parts_ed", 214, 2, 20, 12, 32, 2, 8, 48, 1, 1, vocab, z_loss=1e-3, block=dict(dtype="f32"))
    w = SI.make_encdec_weights(ec)
    SI.make_encdec_random_scales(ec, w)
    et, dt, tg = SI.make_encdec_tokens(ec, ignore_fraction=0.15)
    t, ids = _entries(dt, vocab, 6)
    dw, det, ddt, dtg = _ec_upload(ec, w, et, dt, tg)
    ce, o = B._encdec_cfg_struct(ec), B._DistillOpts(K, TAU, SOFT)
    need = P.lib().t5_encdec_distill_workspace_bytes(C.byref(ce), C.byref(o))
    ws = _guarded(need)
    loss, g = P.t5_encdec_distill_loss_and_grad(ec, det, ddt, dtg, dev(t), ints(ids), dw, temperature=TAU, soft_weight=SOFT, workspace=ws[:need])
    _, saved = O.encdec_loss(ec, et, dt, tg, w)
    want, _, dl = VO.distill_loss(saved["logits"].reshape(-1, vocab), tg.reshape(-1), t.reshape(-1, K), ids.reshape(-1, K),
                                  TAU, SOFT, ec.z_loss)
    _compare(_ec_errs(ec, _grads_np(g), O.encdec_loss_grad(ec, w, saved, dl.reshape(saved["logits"].shape)), et, dt, tg), loss, want)
    assert bool((ws[need:] == 0x7F).all())
