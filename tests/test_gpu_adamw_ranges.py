"""AdamW at the ends of float32's range: gradients and states whose squares leave it, against float64."""
import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
from oracle import fp8_oracle as O
from fp8_util import U, codes, host
from test_gpu_adamw import make, state

pytestmark = pytest.mark.gpu
HP = dict(lr=2e-3, beta1=0.9, beta2=0.99, eps=1e-30)
TINY = 2.0 ** -149  # a step of float32's subnormal values


def scaled(t, k):
    """The tensors of t with gradients, first moments and roots of second ones times 2^k, exactly."""
    t["grad"].mul_(2.0 ** k)
    if t["m"].dtype == torch.float32:
        t["m"].mul_(2.0 ** k)
        t["v"].mul_(2.0 ** k).mul_(2.0 ** k)
    else:
        for key in ("m_scale", "v_scale"):
            b = t[key].view(torch.uint8)
            b.copy_((b.int() + k).clamp(0, 254).to(torch.uint8))
    return t


def step_and_check(t, step, seed=0, hp=HP):
    p, g, (m, v) = host(t["param"]), host(t["grad"]), state(t)
    eight = t["m"].dtype != torch.float32
    v = v * v if eight else v
    wp, wm, wv = O.adamw(p, g, m, v, step=step, weight_decay=t["weight_decay"], **hp)
    P.adamw_step_multi([t], step=step, seed=seed, **hp)
    # m: three roundings and the factors' (values below float32's normal range: half a step each)
    bm = 6 * U * (np.abs(hp["beta1"] * m) + np.abs((1 - hp["beta1"]) * g)) + 3 * TINY
    # root of v: 8 bits: two factors and products, two squares, a sum and the root: 5 U at most; 32 bits: half of v's own error
    bv = 8 * U * wv + 4 * TINY
    root = np.sqrt(wv)
    with np.errstate(divide="ignore", invalid="ignore"):
        br = 5 * U * root + 4 * TINY if eight else np.where(wv > 0, 0.5 * bv / root + 2 * U * root, 0.0)
    factor = 1 / np.sqrt(1 - hp["beta2"] ** step)
    below = root * factor + hp["eps"]
    known = br * factor < 0.01 * below  # (a second moment of a few steps of float32's last place says little of its root)
    # (32 bits, k = -62, first step: v is 33 steps of float32's last place where |g| = 0.01 2^k, and 200 of them are known to 1 %:
    # |g| 2.5 times that, which is a fifth of normal numbers of sizes spread by exp of another)
    assert known.mean() > (0.9 if eight else 0.1)
    upd = np.abs(wp - p * (1 - hp["lr"] * t["weight_decay"]))
    bp = 3 * U * (np.abs(p) + upd) + 16 * U * upd + hp["lr"] / (1 - hp["beta1"] ** step) * bm / below + 1.02 * upd * br * factor / below
    far = np.abs(host(t["param"]) - wp)
    assert (far <= bp)[known].all(), (far[known] / bp[known]).max()
    if not eight:
        assert (np.abs(host(t["m"]) - wm) <= bm).all() and (np.abs(host(t["v"]) - wv) <= bv).all()
        return
    um, ur = O.random_parts(p.size, 0, step, seed)
    for key, want, u, bound in (("m", wm, um, bm), ("v", root, ur, br)):
        s, steps, width = O.steps_of(want)
        got_s = codes(t[key + "_scale"])
        pad = np.pad(np.abs(want), (0, -want.size % 128)).reshape(-1, 128).max(1)
        # A largest value within float32's rounding of 448 times a power of two may have either scale.  With s the float64
        # one, its share of s' largest value is then 1 (it came out at or below the border) or 1/2 (above: s is twice as large).
        share = pad / (2.0 ** (s - 127.0) * 448)
        near = (np.abs(share - 1) < 1e-5) | (np.abs(share - 0.5) < 1e-5)
        assert (got_s[~near] == s[~near]).all()
        x = steps + u
        k = np.floor(x)
        if key == "v":
            k = np.where(want > 0, np.maximum(k, 1), k)
        got = O.code_values("e4m3")[codes(t[key])] * np.repeat(2.0 ** (got_s - 127.0), 128)[:p.size]
        slack = bound / width + 16 * U * (1 + x)
        clear = np.repeat(~near, 128)[:p.size] & (np.abs(x - np.round(x)) > slack)
        assert clear.mean() > 0.9
        assert (got[clear] == np.copysign(k * width, want)[clear]).all(), key
        if key == "v":
            assert (codes(t[key])[want > 2.0 ** -130] != 0).all()


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("k", [-105, -90, -75, -60, -45, 0, 40, 60, 90, 118])
def test_states_in_8_bits_over_the_range_of_float32(k, grad):
    """Roots are held, not squares: second moments far below and above float32 are as good as any."""
    for step, zero in ((1, True), (3, False)):
        step_and_check(scaled(make(np.random.default_rng(200 + k), 3001, 8, grad, zero_state=zero), k), step, seed=5)


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("k", [-62, -60, -55, -45, 0, 40, 55])
def test_states_in_32_bits_down_to_subnormal_second_moments(k, grad):
    for step, zero in ((1, True), (3, False)):
        step_and_check(scaled(make(np.random.default_rng(300 + k), 3001, 32, grad, zero_state=zero), k), step)


def test_roots_far_from_the_gradient():
    """States that are far larger or smaller than the gradient, in one block with ordinary ones and zeros."""
    for k in (-70, -30, 30, 70):
        for beta2 in (0.0, 0.5, 0.999):
            t = make(np.random.default_rng(400 + k), 1024, 8)
            t["grad"].mul_(2.0 ** k)
            t["grad"][::7] = 0.0
            t["v"].view(torch.uint8)[::11] = 0
            step_and_check(t, 2, seed=8, hp={**HP, "beta2": beta2, "eps": 1e-25})


def test_many_steps_of_large_gradients_stay_finite():
    t = make(np.random.default_rng(5), 1000, 8, zero_state=True, decay=0.0)
    t["grad"].copy_(t["grad"].sign() * 2.0 ** 124)
    p = t["param"].clone()
    for step in range(1, 31):
        P.adamw_step_multi([t], step=step, seed=3, **HP)
    m, r = state(t)
    assert np.isfinite(m).all() and np.isfinite(r).all() and torch.isfinite(t["param"]).all()
    # (each step's m and root are off by a step of the type, an eighth, at most, and by as much again from the steps before)
    move = host(p - t["param"]) / host(t["grad"].sign()) / (30 * HP["lr"])
    assert (move > 0.5).all() and (move < 2.0).all()
