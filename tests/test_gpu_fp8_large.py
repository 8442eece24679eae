"""Operators of training in 8 bits on data beyond 32-bit offsets: the same as on the end of that data alone."""
import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
from oracle import fp8_oracle as O
from fp8_util import E8M0, codes, host

pytestmark = pytest.mark.gpu


def need(gb):
    if torch.cuda.get_device_properties(0).total_memory < gb << 30:
        pytest.skip(f"needs {gb} GB")


def tile_copies(t, rows):
    """rows rows, those of t again and again."""
    return t.repeat(-(-rows // t.shape[0]), 1)[:rows].contiguous()


def test_quantise_and_multiply_beyond_4_gb():
    need(64)
    rows, cols, last = 70000, 65536, 69888  # codes of 4.6 GB; `last` is a multiple of 128
    g = torch.Generator(device="cuda").manual_seed(1)
    x = tile_copies(torch.randn(1000, cols, device="cuda", generator=g).bfloat16(), rows)
    q, s, qt, st = P.t5_quantize_fp8(x, transposed=True)
    eq, es, eqt, est = P.t5_quantize_fp8(x[last:], transposed=True)
    u8 = lambda t: t.view(torch.uint8)  # noqa: E731
    assert torch.equal(u8(q)[last:], u8(eq)) and torch.equal(u8(s)[last:], u8(es))
    assert torch.equal(u8(qt)[:, last:], u8(eqt)) and torch.equal(u8(st)[:, last // 128:], u8(est))
    square = P.t5_quantize_fp8(x, block_rows=128)[:2]
    esq = P.t5_quantize_fp8(x[last:], block_rows=128)[:2]
    assert torch.equal(u8(square[0])[last:], u8(esq[0])) and torch.equal(u8(square[1])[last // 128:], u8(esq[1]))
    rowwise = P.t5_quantize_fp8(x)[:2]
    assert torch.equal(u8(rowwise[0]), u8(q)) and torch.equal(u8(rowwise[1]), u8(s))
    del square, rowwise, x
    b, sb = eq[:70], es[:70]
    va, vb = O.values(codes(q[-100:]), codes(s[-100:]), "e4m3"), O.values(codes(b), codes(sb), "e4m3")
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    c = P.t5_gemm_fp8(q, s, b, sb, out_dtype=torch.float32)
    assert (np.abs(host(c[-100:]) - want) <= (cols / 16 + 84) * 2.0 ** -24 * size).all()
    c = P.t5_gemm_fp8(q, s, b, sb)
    # each product loses less than 2^-13 of its group's sum
    assert (np.abs(host(c[-100:]) - want) <= 2.0 ** -8 * np.abs(want) + (8 * 2.0 ** -13 + (cols / 64 + 84) * 2.0 ** -24) * size).all()
    # as the second operand, and in few rows
    c = P.t5_gemm_fp8(b, sb, q, s)
    assert (np.abs(host(c[:, -100:]) - want.T) <= 2.0 ** -8 * np.abs(want.T) + (8 * 2.0 ** -13 + (cols / 64 + 84) * 2.0 ** -24) * size.T).all()
    few = P.t5_gemm_fp8(b[:3], sb[:3], q, s, out_dtype=torch.float32)
    assert (np.abs(host(few[:, -100:]) - want.T[:3]) <= (cols / 16 + 84) * 2.0 ** -24 * size.T[:3]).all()


def test_result_beyond_4_g_elements():
    need(64)
    m, n, k = 70000, 65536, 128
    g = torch.Generator(device="cuda").manual_seed(2)
    a, sa, _, _ = P.t5_quantize_fp8(torch.randn(m, k, device="cuda", generator=g))
    b, sb, _, _ = P.t5_quantize_fp8(torch.randn(n, k, device="cuda", generator=g))
    va, vb = O.values(codes(a[-40:]), codes(sa[-40:]), "e4m3"), O.values(codes(b[-300:]), codes(sb[-300:]), "e4m3")
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    c = P.t5_gemm_fp8(a, sa, b, sb)
    assert (np.abs(host(c[-40:, -300:]) - want) <= 2.0 ** -8 * np.abs(want) + (8 * 2.0 ** -13 + 90 * 2.0 ** -24) * size).all()
    del c
    c = P.t5_gemm_fp8(a, sa, b, sb, out_dtype=torch.float32)
    assert (np.abs(host(c[-40:, -300:]) - want) <= 92 * 2.0 ** -24 * size).all()


def test_adamw_beyond_4_g_elements():
    need(96)
    n, tail = (1 << 32) + 5000, 9000
    hp = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)
    zeros = lambda k, dt: torch.zeros(k, dtype=torch.uint8, device="cuda").view(dt)  # noqa: E731
    t = dict(param=torch.full((n,), 0.5, device="cuda"), grad=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), m=zeros(n, torch.float8_e4m3fn),
             v=zeros(n, torch.float8_e4m3fn), m_scale=zeros(-(-n // 128), E8M0), v_scale=zeros(-(-n // 128), E8M0))
    g = torch.Generator(device="cuda").manual_seed(3)
    t["grad"][-tail:] = torch.randn(tail, device="cuda", generator=g).bfloat16()
    grad = host(t["grad"][-tail:])
    P.adamw_step_multi([t], step=3, seed=(9 << 32) + 5, **hp)
    wp, wm, wv = O.adamw(np.full(tail, 0.5), grad, np.zeros(tail), np.zeros(tail), step=3, weight_decay=0.0, **hp)
    np.testing.assert_allclose(host(t["param"][-tail:]), wp, rtol=4 * 2.0 ** -24, atol=hp["lr"] * 30 * 2.0 ** -24)
    assert (t["param"][:-tail] == 0.5).all()
    first = n - tail + (-(n - tail)) % 128  # whole blocks
    um, ur = O.random_parts(n - first, 0, 3, (9 << 32) + 5, first)
    for key, want, u in (("m", wm, um), ("v", np.sqrt(wv), ur)):
        want = want[first - (n - tail):]
        s, steps, width = O.steps_of(want)
        x = steps + u
        clear = np.abs(x - np.round(x)) > 32 * 2.0 ** -24 * (1 + x)
        k = np.maximum(np.floor(x), 1) if key == "v" else np.floor(x)
        got = O.code_values("e4m3")[codes(t[key][first:])] * np.repeat(2.0 ** (codes(t[key + "_scale"][first // 128:]) - 127.0), 128)[:n - first]
        assert (got[clear] == np.copysign(k * width, want)[clear]).all() and clear.mean() > 0.9


def test_hundreds_of_millions_of_rows():
    """As many rows as the arguments allow: workgroups of a launch are counted in 24 bits."""
    need(128)
    rows = 1 << 30
    a = torch.full((rows, 16), 0x38, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    sa = torch.full((rows // 128, 4), 127, dtype=torch.uint8, device="cuda").view(E8M0)[:, :1]
    b = torch.full((3, 16), 0x40, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    sb = torch.full((1, 4), 128, dtype=torch.uint8, device="cuda").view(E8M0)[:, :1]
    a.view(torch.uint8)[-1, 3] = 0x40
    c = P.t5_gemm_fp8(a, sa, b, sb)
    assert (c[:-1] == 64).all() and (c[-1] == 68).all()
    del c
    c = P.t5_gemm_fp8(b, sb, a, sa)  # the few rows against them
    assert (c[:, :-1] == 64).all() and (c[:, -1] == 68).all()
    del c, a, sa
    x = torch.ones((1 << 26) - 7, 5, dtype=torch.bfloat16, device="cuda")
    x[-1] = 2.0
    q, s, _, _ = P.t5_quantize_fp8(x)
    assert (q.view(torch.uint8) == 0x78).all() and (s.view(torch.uint8)[:-1] == 119).all() and s.view(torch.uint8)[-1, 0] == 120
