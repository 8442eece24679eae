"""Teacher and student in bfloat16, stack and encoder-decoder pair: every logit and gradient against the float64 oracle, held to
bounds from the floor of ideal bf16-operand arithmetic for the very case (tests/bf16_model.py, its head with this loss)."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import bf16_model as M
import synth_inputs as SI
from oracle import t5_oracle as O
from oracle import vocab_oracle as VO
from parity_util import check_bf16, general_mlp_path, rel_err, to_np
from test_gpu_parity_stack import _ec_errs, _ec_upload, _grads_np, _stack_errs, _upload
from vocab_util import dev, ints

pytestmark = pytest.mark.gpu
TAU, SOFT = 2.0, 0.5

BLK = SI.BlockConfig("distill_bf16", 220, batch=2, seq=128, d_model=128, n_heads=2, d_kv=64, d_ff=256, causal=True, attn_scale=64 ** -0.5)
STACKS = [SI.StackConfig("distill_bf16", BLK, n_layers=2, vocab=256, z_loss=1e-3),
          SI.StackConfig("distill_bf16_tied", replace(BLK, index=222, causal=False), n_layers=2, vocab=256, tied_logits=True),
          SI.StackConfig("distill_bf16_ragged", SI.BlockConfig("distill_bf16_ragged", 224, batch=1, seq=50, d_model=72, n_heads=3, d_kv=24,
                                                               d_ff=136, causal=True, attn_scale=24 ** -0.5), n_layers=2, vocab=251),
          # rows in parts, two tokens fewer than a tile
          SI.StackConfig("distill_bf16_parts", replace(BLK, index=226, batch=1, seq=126, d_model=64, n_heads=1, d_ff=128), n_layers=1, vocab=40000)]
PAIRS = [SI._encdec("distill_ed_bf16", 230, 2, 256, 128, 128, 2, 64, 256, 2, 2, 256, block=dict(attn_scale=64 ** -0.5)),
         replace(SI._encdec("distill_ed_bf16_tied", 232, 1, 128, 128, 128, 2, 64, 256, 1, 2, 256, block=dict(attn_scale=64 ** -0.5)), tied_logits=True),
         SI._encdec("distill_ed_bf16_ragged", 234, 1, 70, 33, 72, 3, 24, 136, 2, 1, 251, block=dict(attn_scale=24 ** -0.5))]


def _entries(shape, vocab, seed, k=16):
    """Some entries of each position; sharp and flat distributions, holes."""
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, vocab, (*shape, k))
    t = np.float32(rng.standard_normal(ids.shape) * rng.choice([0.5, 4.0], (*shape, 1))).astype(np.float64)
    return t, np.where(rng.random(ids.shape) < 0.1, -1, ids)


def _head(t, ids, kept):
    """The model's head with the distillation loss in place of the cross-entropy: the same tensors rounded."""
    def head(cfg, x_last, final_scale, emb_or_w, tied, targets, z_loss, site):
        s = cfg.d_model ** -0.5 if tied else 1.0
        gf = M.rb(final_scale * s) if tied else final_scale
        nf, rf = O.rmsnorm_fwd(x_last, gf, cfg.rms_eps)
        nf = M.rb(nf)
        wmat = emb_or_w.T if tied else emb_or_w
        kept["logits"] = logits = M.rb(nf @ wmat)
        k = ids.shape[-1]
        loss, _, dl = VO.distill_loss(logits.reshape(-1, logits.shape[-1]), targets.reshape(-1), t.reshape(-1, k), ids.reshape(-1, k),
                                      TAU, SOFT, z_loss)
        dlogits = M.rb(dl.reshape(logits.shape))
        dw = M._flat(nf).T @ M._flat(dlogits)
        dx, dgf = O.rmsnorm_bwd(x_last, gf, rf, dlogits @ wmat.T)
        return loss, M.rb(dx), dgf * s, (dw.T if tied else dw)
    return head


def _whole(v, i, vocab):
    """[positions, vocab] from entries that hold every logit."""
    out = np.full((v.shape[0] * v.shape[1], vocab), np.nan)
    np.put_along_axis(out, i.cpu().numpy().reshape(len(out), -1), to_np(v).reshape(len(out), -1), 1)
    return out


def _oracle(saved, targets, t, ids, z):
    flat, k = saved["logits"].reshape(-1, saved["logits"].shape[-1]), ids.shape[-1]
    loss, _, dl = VO.distill_loss(flat, targets.reshape(-1), t.reshape(-1, k), ids.reshape(-1, k), TAU, SOFT, z)
    return loss, dl.reshape(saved["logits"].shape)


def _check(label, loss, want, errs, floors, logits, saved, kept):
    """The loss: the cross-entropy's bound (5e-4), by how much further the same errors of the logits move this one: a row's
    gradient over its logits is at most 2 (1 - a + a T) in sum instead of 2."""
    assert abs(float(loss) - want) <= 5e-4 * (1 - SOFT + SOFT * TAU) * max(1.0, abs(want)), (float(loss), want)
    if logits is not None:
        ref = saved["logits"].reshape(logits.shape)
        errs, floors = dict(errs, logits=rel_err(logits, ref)), dict(floors, logits=rel_err(kept["logits"].reshape(logits.shape), ref))
    check_bf16(label, errs, floors)


@pytest.mark.parametrize("sc", STACKS, ids=[c.name for c in STACKS])
def test_stack(sc, monkeypatch):
    import paper_2203_17189_amd as P
    w = SI.make_stack_weights(sc)
    SI.make_stack_random_scales(sc, w)
    tokens, targets = SI.make_tokens(sc, ignore_fraction=0.15)
    t, ids = _entries(tokens.shape, sc.vocab, sc.block.index)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    logits = None
    if sc.vocab <= 256:
        logits = _whole(*P.t5_stack_top_logits(sc, tt, dw, sc.vocab), sc.vocab)
    loss, g = P.t5_stack_distill_loss_and_grad(sc, tt, tg, dev(t), ints(ids), dw, temperature=TAU, soft_weight=SOFT)
    _, saved = O.stack_loss(sc, tokens, targets, w)
    want, dl = _oracle(saved, targets, t, ids, sc.z_loss)
    wg = O.stack_loss_grad(sc, w, saved, dl)
    kept = {}
    monkeypatch.setattr(M, "_head", _head(t, ids, kept))
    _, mg = M.stack_model(sc, tokens, targets, w, round_uw=general_mlp_path(sc.block))
    _check(sc.name, loss, want, _stack_errs(sc, _grads_np(g), wg, tokens, targets), _stack_errs(sc, mg, wg, tokens, targets), logits, saved, kept)


@pytest.mark.parametrize("ec", PAIRS, ids=[c.name for c in PAIRS])
def test_pair(ec, monkeypatch):
    import paper_2203_17189_amd as P
    w = SI.make_encdec_weights(ec)
    SI.make_encdec_random_scales(ec, w)
    et, dt, tg = SI.make_encdec_tokens(ec, ignore_fraction=0.15)
    t, ids = _entries(dt.shape, ec.vocab, ec.enc_block.index)
    dw, det, ddt, dtg = _ec_upload(ec, w, et, dt, tg)
    logits = _whole(*P.t5_encdec_top_logits(ec, det, ddt, dw, ec.vocab), ec.vocab)
    loss, g = P.t5_encdec_distill_loss_and_grad(ec, det, ddt, dtg, dev(t), ints(ids), dw, temperature=TAU, soft_weight=SOFT)
    _, saved = O.encdec_loss(ec, et, dt, tg, w)
    want, dl = _oracle(saved, tg, t, ids, ec.z_loss)
    wg = O.encdec_loss_grad(ec, w, saved, dl)
    kept = {}
    monkeypatch.setattr(M, "_head", _head(t, ids, kept))
    _, mg = M.encdec_model(ec, et, dt, tg, w, round_uw=general_mlp_path(ec.enc_block) or general_mlp_path(ec.dec_block))
    _check(ec.name, loss, want, _ec_errs(ec, _grads_np(g), wg, et, dt, tg), _ec_errs(ec, mg, wg, et, dt, tg), logits, saved, kept)
