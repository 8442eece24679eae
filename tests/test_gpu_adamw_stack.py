"""Models trained through the library's own calls: loss and gradients of a whole stack, then one AdamW call over all of its
tensors, with states in 32 bits and in 8, float32 and bfloat16 models; every tensor, state and copy against float64."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
import test_gpu_parity_stack as TS
from paper_2203_17189_amd import binding as B
from test_gpu_adamw import E8M0, step_and_check
from test_gpu_train_steps import SC, _flat

pytestmark = pytest.mark.gpu
HP = dict(lr=2e-3, beta1=0.9, beta2=0.98, eps=1e-8)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sc", [SC, replace(TS.BF16_CASES[0], n_layers=2)], ids=["f32", "bf16"])
def test_three_steps_of_a_stack(sc, bits):
    w, tokens, targets = TS._case(sc)
    dw, ttok, ttgt = TS._upload(sc, w, tokens, targets)
    grads = B.alloc_stack_grads(sc, dw)
    zeros = lambda n, dt: torch.zeros(n, dtype=torch.uint8, device="cuda").view(dt)  # noqa: E731
    opt = []
    for _, wt, gt in _flat(dw, grads):
        n = wt.numel()
        t = dict(param=wt.view(-1) if wt.dtype == torch.float32 else wt.float().view(-1), grad=gt.view(-1), weight_decay=0.1 if wt.dim() == 2 else 0.0,
                 bf16_copy_out=wt.view(-1) if wt.dtype == torch.bfloat16 else None)
        if bits == 32:
            t.update(m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
        else:
            t.update(m=zeros(n, torch.float8_e4m3fn), v=zeros(n, torch.float8_e4m3fn), m_scale=zeros(-(-n // 128), E8M0), v_scale=zeros(-(-n // 128), E8M0))
        opt.append(t)
    losses = []
    for step in (1, 2, 3):
        loss, _ = P.t5_stack_loss_and_grad(sc, ttok, ttgt, dw, grads=grads)
        losses.append(loss.item())
        step_and_check(opt, step, seed=3, hp=HP)
    assert np.isfinite(losses).all()
    for (_, wt, _), t in zip(_flat(dw, grads), opt):  # the model holds what the optimizer wrote
        assert torch.equal(wt.view(-1), t["param"].to(wt.dtype))
