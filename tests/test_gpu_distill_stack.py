"""A student trained from a teacher, whole models: the teacher's top logits, the student's loss and gradients against them
(float64 oracle), a few training steps as a program runs them, and the same captured into a graph."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth_inputs as SI
from oracle import t5_oracle as O
from oracle import vocab_oracle as VO
from parity_util import TOL_F32, rel_err, to_dev, to_np
from test_gpu_parity_stack import _ec_errs, _ec_upload, _grads_np, _stack_errs, _upload

pytestmark = pytest.mark.gpu

BLK = SI.BlockConfig("distill_f32", 160, batch=2, seq=24, d_model=32, n_heads=2, d_kv=8, d_ff=48, dtype="f32", causal=True)
STUDENTS = [
    SI.StackConfig("distill_f32", BLK, n_layers=2, vocab=61, z_loss=1e-2),
    SI.StackConfig("distill_f32_tied", replace(BLK, index=161, causal=False), n_layers=2, vocab=64, tied_logits=True, z_loss=1e-3),
    SI.StackConfig("distill_f32_remat", replace(BLK, index=162), n_layers=3, vocab=200, remat=True, z_loss=0.0),
    SI.StackConfig("distill_f32_dropout", replace(BLK, index=163, dropout_rate=0.1, dropout_seed=5), n_layers=1, vocab=1500),
    # more tokens than the logits exist for at a time, and a last chunk that is not whole
    SI.StackConfig("distill_f32_chunks", SI.BlockConfig("distill_chunks", 164, batch=1025, seq=16, d_model=8, n_heads=1, d_kv=8,
                                                        d_ff=8, dtype="f32", causal=True), n_layers=1, vocab=50),
]


def _teacher(sc, k):
    """A wider, deeper model over the same vocabulary: (configuration, weights, top values, ids) from the device."""
    import paper_2203_17189_amd as P
    b = replace(sc.block, index=sc.block.index + 100, d_model=48, n_heads=3, d_ff=64, dropout_rate=0.0)
    tc = SI.StackConfig("teacher", b, n_layers=2, vocab=sc.vocab)
    w = SI.make_stack_weights(tc)
    SI.make_stack_random_scales(tc, w)
    tokens, targets = SI.make_tokens(sc, ignore_fraction=0.15)
    dw, tt, _ = _upload(tc, w, tokens, targets)
    v, i = P.t5_stack_top_logits(tc, tt, dw, k)
    torch.cuda.synchronize()
    return tc, w, tokens, targets, v, i


def _student_oracle(sc, w, tokens, targets, v, i, tau, soft):
    _, saved = O.stack_loss(sc, tokens, targets, w)
    flat = saved["logits"].reshape(-1, sc.vocab)
    loss, _, dl = VO.distill_loss(flat, targets.reshape(-1), to_np(v).reshape(len(flat), -1).astype(np.float64),
                                  i.cpu().numpy().reshape(len(flat), -1), tau, soft, sc.z_loss)
    return loss, O.stack_loss_grad(sc, w, saved, dl.reshape(saved["logits"].shape))


@pytest.mark.parametrize("k,tau,soft", [(8, 2.0, 0.5), (1, 1.0, 1.0), (50, 1.5, 0.9)])
@pytest.mark.parametrize("sc", STUDENTS, ids=[c.name for c in STUDENTS])
def test_teacher_then_student(sc, k, tau, soft):
    import paper_2203_17189_amd as P
    tc, tw, tokens, targets, v, i = _teacher(sc, k)
    # the teacher's entries: the oracle's logits at the ids, none of the others larger by more than the same tolerance
    _, saved = O.stack_loss(tc, tokens, targets, tw)
    lg = saved["logits"]
    tol = TOL_F32[0] * np.maximum(np.abs(lg).max(-1, keepdims=True), 1.0)
    ids = i.cpu().numpy()
    assert v.shape == (*tokens.shape, k) and np.all(np.diff(to_np(v), axis=-1) <= 0)
    assert np.all(np.abs(np.take_along_axis(lg, ids, -1) - to_np(v)) <= tol)
    assert np.all(-np.sort(-lg, -1)[..., :k] - to_np(v) <= tol)
    assert np.all(np.diff(np.sort(ids, -1), axis=-1) > 0)
    # the student's loss and every gradient
    w = SI.make_stack_weights(sc)
    SI.make_stack_random_scales(sc, w)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    loss, g = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=tau, soft_weight=soft)
    want, wg = _student_oracle(sc, w, tokens, targets, v, i, tau, soft)
    assert abs(float(loss) - want) <= 1e-5 * max(1.0, abs(want))
    for name, e in _stack_errs(sc, _grads_np(g), wg, tokens, targets).items():
        assert e[0] <= TOL_F32[0], (name, e)
    only, none = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=tau, soft_weight=soft, want_grads=False)
    assert none is None and torch.equal(only, loss)
    # accumulating once more doubles them; the embedding's has the same bits every time
    _, g2 = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=tau, soft_weight=soft)
    if not sc.tied_logits:
        assert torch.equal(g2["embedding"], g["embedding"])
    P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=tau, soft_weight=soft, grads=g2, accumulate=True)
    for name in ("embedding", "rel_table", "final_scale"):
        np.testing.assert_allclose(to_np(g2[name]), 2 * to_np(g[name]), rtol=2e-5, atol=1e-7)


def test_without_soft_targets_it_is_the_cross_entropy():
    """soft_weight 0 against t5_stack_loss_and_grad, float32 (to rounding) and bf16 (two roundings of the same numbers to
    bfloat16 and what the layers below make of them: each within 2^-8 of the exact ones, so 2 * 2^-8 of each other)."""
    import paper_2203_17189_amd as P
    for dtype, tol in (("f32", 2e-5), ("bf16", 2.0 ** -7)):
        b = replace(BLK, index=170, dtype=dtype, d_model=128, n_heads=2, d_kv=64, d_ff=128, seq=64, attn_scale=0.125)
        sc = SI.StackConfig("distill_ce", b, n_layers=2, vocab=512, z_loss=1e-3)
        w = SI.make_stack_weights(sc)
        tokens, targets = SI.make_tokens(sc, ignore_fraction=0.15)
        dw, tt, tg = _upload(sc, w, tokens, targets)
        v, i = P.t5_stack_top_logits(sc, tt, dw, 16)
        loss, g = P.t5_stack_loss_and_grad(sc, tt, tg, dw)
        l2, g2 = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, soft_weight=0.0)
        assert abs(float(l2) - float(loss)) <= 1e-6 * float(loss)
        for name in ("embedding", "logits_w", "final_scale", "rel_table"):
            a, c = to_np(g[name]), to_np(g2[name])
            assert np.linalg.norm(a - c) <= tol * np.linalg.norm(a), (dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_teacher_that_is_the_student_teaches_nothing(dtype):
    """All logits as entries and the student's own: p = q, so the loss is 0 but for float32 rounding of sums of 256 terms
    (log p and log q are good to 1e-6) and the gradient over the logits cancels to the same degree."""
    import paper_2203_17189_amd as P
    b = replace(BLK, index=171, dtype=dtype, d_model=128, n_heads=2, d_kv=64, d_ff=128, seq=64, attn_scale=0.125)
    sc = SI.StackConfig("distill_self", b, n_layers=2, vocab=256, z_loss=0.0)
    w = SI.make_stack_weights(sc)
    tokens, targets = SI.make_tokens(sc)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    v, i = P.t5_stack_top_logits(sc, tt, dw, 256)
    assert np.array_equal(np.sort(i.cpu().numpy(), -1), np.broadcast_to(np.arange(256), (*tokens.shape, 256)))
    loss, g = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=2.0)
    ref = P.t5_stack_loss_and_grad(sc, tt, tg, dw)[1]
    assert abs(float(loss)) <= 4 * 2e-6
    for name in ("embedding", "logits_w", "final_scale"):
        assert float(g[name].norm()) <= 1e-4 * float(ref[name].norm())


ECS = [SI._encdec("distill_ed", 180, 2, 20, 12, 32, 2, 8, 48, 2, 2, 61, z_loss=1e-3, block=dict(dtype="f32")),
       SI._encdec("distill_ed_tied", 182, 2, 9, 17, 32, 2, 8, 48, 1, 2, 300, tied_logits=True, block=dict(dtype="f32"))]


@pytest.mark.parametrize("ec", ECS, ids=[c.name for c in ECS])
def test_encoder_decoder(ec):
    import paper_2203_17189_amd as P
    w = SI.make_encdec_weights(ec)
    SI.make_encdec_random_scales(ec, w)
    et, dt, tg = SI.make_encdec_tokens(ec, ignore_fraction=0.15)
    dw, det, ddt, dtg = _ec_upload(ec, w, et, dt, tg)
    tw = SI.make_encdec_weights(ec)  # a teacher of the same shape with other scales
    v, i = P.t5_encdec_top_logits(ec, det, ddt, _ec_upload(ec, tw, et, dt, tg)[0], 7)
    _, saved = O.encdec_loss(ec, et, dt, tg, tw)
    tol = TOL_F32[0] * np.maximum(np.abs(saved["logits"]).max(-1, keepdims=True), 1.0)
    assert np.all(np.abs(np.take_along_axis(saved["logits"], i.cpu().numpy(), -1) - to_np(v)) <= tol)
    assert np.all(np.abs(-np.sort(-saved["logits"], -1)[..., :7] - to_np(v)) <= tol)
    loss, g = P.t5_encdec_distill_loss_and_grad(ec, det, ddt, dtg, v, i, dw, temperature=2.0, soft_weight=0.7)
    _, saved = O.encdec_loss(ec, et, dt, tg, w)
    flat = saved["logits"].reshape(-1, ec.vocab)
    want, _, dl = VO.distill_loss(flat, tg.reshape(-1), to_np(v).reshape(len(flat), 7).astype(np.float64),
                                  i.cpu().numpy().reshape(len(flat), 7), 2.0, float(np.float32(0.7)), ec.z_loss)
    wg = O.encdec_loss_grad(ec, w, saved, dl.reshape(saved["logits"].shape))
    assert abs(float(loss) - want) <= 1e-5 * max(1.0, abs(want))
    for name, e in _ec_errs(ec, _grads_np(g), wg, et, dt, tg).items():
        assert e[0] <= TOL_F32[0], (name, e)


def test_training_steps_and_refusals():
    """Three steps as a program runs them: the teacher's pass, the student's, Adafactor on every tensor.  The first step's
    update is checked against the oracle's gradients elsewhere; here every parameter stays finite and moves."""
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    sc = STUDENTS[0]
    tc, tw, tokens, targets, _, _ = _teacher(sc, 8)
    tdw, tt, tg = _upload(tc, tw, tokens, targets)
    w = SI.make_stack_weights(sc)
    dw = _upload(sc, w, tokens, targets)[0]
    grads = B.alloc_stack_grads(sc, dw)
    flat = lambda d: [d[n] for n in ("embedding", "rel_table", "final_scale", "logits_w")] + [t for l in d["layers"] for t in l.values()]
    before = [p.clone() for p in flat(dw)]
    state = [dict(param=p, grad=g, factored=False, v_full=torch.zeros_like(p)) for p, g in zip(flat(dw), flat(grads))]
    for step in range(1, 4):
        v, i = P.t5_stack_top_logits(tc, tt, tdw, 8)
        P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, temperature=2.0, soft_weight=0.8, grads=grads)
        P.adafactor_step_multi(state, step=step, lr=1e-2)
    assert all(bool(torch.isfinite(p).all()) and not torch.equal(p, q) for p, q in zip(flat(dw), before))
    for bad in (dict(temperature=0.0), dict(soft_weight=1.5)):
        with pytest.raises(P.T5Error):
            P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, **bad)
    for k in (0, 62, 257):
        with pytest.raises(P.T5Error):
            P.t5_stack_top_logits(tc, tt, tdw, k)
    with pytest.raises(P.T5Error) as e:
        P.t5_stack_top_logits(tc, tt, tdw, 8, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 4
    with pytest.raises(ValueError):
        P.t5_stack_distill_loss_and_grad(sc, tt, tg, v[..., :4].contiguous(), i, dw)


def test_teacher_and_student_in_a_graph():
    import paper_2203_17189_amd as P
    from paper_2203_17189_amd import binding as B
    b = replace(BLK, index=172, dtype="bf16", d_model=128, n_heads=2, d_kv=64, d_ff=256, seq=128, attn_scale=0.125)
    sc = SI.StackConfig("distill_graph", b, n_layers=2, vocab=512)
    w = SI.make_stack_weights(sc)
    tokens, targets = SI.make_tokens(sc)
    dw, tt, tg = _upload(sc, w, tokens, targets)
    tw = SI.make_stack_weights(replace(sc, block=replace(b, index=272)))
    tdw = _upload(sc, tw, tokens, targets)[0]
    opts = dict(temperature=2.0, soft_weight=0.5)
    from paper_2203_17189_amd.binding import _DistillOpts, _stack_cfg_struct, lib
    import ctypes as C
    cs, o = _stack_cfg_struct(sc), _DistillOpts(16, 2.0, 0.5)
    mk = lambda: dict(grads=B.alloc_stack_grads(sc, dw), loss=torch.zeros(1, device="cuda"),
                      v=torch.empty(*tokens.shape, 16, device="cuda"),
                      i=torch.empty(*tokens.shape, 16, dtype=torch.int32, device="cuda"),
                      ws=torch.empty(lib().t5_stack_distill_workspace_bytes(C.byref(cs), C.byref(o)), dtype=torch.uint8, device="cuda"),
                      tws=torch.empty(lib().t5_stack_top_logits_workspace_bytes(C.byref(cs), 16), dtype=torch.uint8, device="cuda"))
    eager, graph = mk(), mk()

    def step(s):
        P.t5_stack_top_logits(sc, tt, tdw, 16, values=s["v"], ids=s["i"], workspace=s["tws"])
        P.t5_stack_distill_loss_and_grad(sc, tt, tg, s["v"], s["i"], dw, grads=s["grads"], loss=s["loss"], workspace=s["ws"], **opts)

    step(graph)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graph)
    for rep in range(3):
        tok2, tgt2 = SI.make_tokens(sc, seed_offset=rep + 1)
        tt.copy_(torch.from_numpy(tok2).cuda())
        tg.copy_(torch.from_numpy(tgt2).cuda())
        graph["loss"].zero_()
        g.replay()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(graph["v"], eager["v"]) and torch.equal(graph["i"], eager["i"])
        assert torch.equal(graph["loss"], eager["loss"])
        for k in ("embedding", "logits_w", "final_scale", "rel_table"):
            a = to_np(eager["grads"][k])
            assert np.abs(to_np(graph["grads"][k]) - a).max() <= 1e-4 * (np.abs(a).max() + 1e-30), (rep, k)
