"""What the wrappers of a student's step refuse before anything is launched."""
import pytest
import torch

import synth_inputs as SI
from test_gpu_distill_stack import ECS, STUDENTS
from test_gpu_parity_stack import _ec_upload, _upload

pytestmark = pytest.mark.gpu
# (on the host, of another type, of no or several elements, strided)
LOSSES = [torch.zeros(1), torch.zeros(1, dtype=torch.float64), "f64", "empty", "two", "strided"]


def _loss(kind):
    if isinstance(kind, torch.Tensor):
        return kind
    return dict(f64=lambda: torch.zeros(1, dtype=torch.float64, device="cuda"), empty=lambda: torch.zeros(0, device="cuda"),
                two=lambda: torch.zeros(2, device="cuda"), strided=lambda: torch.zeros(2, 2, device="cuda").t())[kind]()


@pytest.mark.parametrize("kind", LOSSES, ids=["host", "host_f64", "f64", "empty", "two", "strided"])
def test_loss(kind):
    import paper_2203_17189_amd as P
    sc = STUDENTS[0]
    dw, tt, tg = _upload(sc, SI.make_stack_weights(sc), *SI.make_tokens(sc))
    v, i = P.t5_stack_top_logits(sc, tt, dw, 4)
    with pytest.raises(ValueError):
        P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, loss=_loss(kind))
    mine = torch.full((3,), 7.0, device="cuda")
    loss, _ = P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, loss=mine[1:2])
    assert torch.equal(loss, P.t5_stack_distill_loss_and_grad(sc, tt, tg, v, i, dw, want_grads=False)[0])
    assert float(mine[0]) == float(mine[2]) == 7.0
    ec = ECS[0]
    dw, et, dt, tg = _ec_upload(ec, SI.make_encdec_weights(ec), *SI.make_encdec_tokens(ec))
    v, i = P.t5_encdec_top_logits(ec, et, dt, dw, 4)
    with pytest.raises(ValueError):
        P.t5_encdec_distill_loss_and_grad(ec, et, dt, tg, v, i, dw, loss=_loss(kind))


def test_tokens_weights_and_gradients_on_the_host():
    import paper_2203_17189_amd as P
    ec = ECS[0]
    dw, et, dt, tg = _ec_upload(ec, SI.make_encdec_weights(ec), *SI.make_encdec_tokens(ec))
    v, i = P.t5_encdec_top_logits(ec, et, dt, dw, 4)
    for bad in (lambda: P.t5_encdec_top_logits(ec, et.cpu(), dt, dw, 4),
                lambda: P.t5_encdec_top_logits(ec, et, dt, dict(dw, embedding=dw["embedding"].cpu()), 4),
                lambda: P.t5_encdec_distill_loss_and_grad(ec, et, dt, tg, v, i.cpu(), dw),
                lambda: P.t5_encdec_distill_loss_and_grad(ec, et, dt, tg.cpu(), v, i, dw)):
        with pytest.raises(ValueError):
            bad()
