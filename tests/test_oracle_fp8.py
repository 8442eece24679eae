"""Pins of the definitions of training in 8 bits: torch's 8-bit types and optimizer, closed forms."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as O

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_codes_are_torchs(fmt):
    v = torch.arange(256, dtype=torch.uint8).view(TYPES[fmt]).double().numpy()
    np.testing.assert_array_equal(O.code_values(fmt), v)
    g = torch.Generator().manual_seed(1)
    most = O.FORMATS[fmt][2]
    x = torch.cat([torch.randn(20000, generator=g) * 2.0 ** torch.randint(-18, 7, (20000,), generator=g), torch.linspace(-most, most, 3001)])
    x = x.clamp(-most, most)
    np.testing.assert_array_equal(O.encode(x.double().numpy(), fmt), x.to(TYPES[fmt]).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt,biggest,e", [("e4m3", 448.0, 0), ("e4m3", 448.1, 1), ("e4m3", 224.0, -1), ("e4m3", 1.0, -8), ("e4m3", 1.76, -7),
                                           ("e5m2", 57344.0, 0), ("e5m2", 57345.0, 1), ("e5m2", 1.0, -15), ("e4m3", 1e-40, -127), ("e4m3", 0.0, 0),
                                           ("e4m3", 3.4e38, 120), ("e5m2", 3.4e38, 113)])
def test_scale_by_hand(fmt, biggest, e):
    assert O.scale_bytes(np.array([[biggest]]), fmt)[0, 0] == e + 127


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantised_values_are_near(fmt, block_rows):
    x = np.random.default_rng(0).standard_normal((200, 300))
    q, s = O.quantize(x, fmt, block_rows)
    v = O.values(q, s, fmt)
    half = {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}[fmt]
    floor = {"e4m3": 2.0 ** -10, "e5m2": 2.0 ** -17}[fmt] * O.spread(s, 200, 300)
    assert (np.abs(v - x) <= np.maximum(half * np.abs(x), floor)).all()
    if block_rows == 128:  # a square's codes are those of the transposed matrix
        qt, st = O.quantize(x.T, fmt, 128)
        np.testing.assert_array_equal(qt, q.T)
        np.testing.assert_array_equal(st, s.T)


def test_adamw_is_torchs():
    rng = np.random.default_rng(2)
    p, g = torch.tensor(rng.standard_normal(50), requires_grad=True), rng.standard_normal((5, 50))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.9, 0.98), eps=1e-6, weight_decay=0.2)
    w, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(5):
        p.grad = torch.tensor(g[t])
        opt.step()
        w, m, v = O.adamw(w, g[t], m, v, step=t + 1, lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-6, weight_decay=0.2)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_random_parts_are_spread_evenly():
    a, b = O.random_parts(1 << 17, 3, 7, 0x1234567800000001)
    for u in (a, b):
        assert 0 <= u.min() and u.max() < 1 and abs(u.mean() - 0.5) < 6 * (1 / 12) ** 0.5 / 2 ** 8.5
        assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 6 / 2 ** 8.5
    assert abs(np.corrcoef(a, b)[0, 1]) < 6 / 2 ** 8.5
    # one hash by hand in whole numbers
    M = 0xFFFFFFFF

    def mix(x):
        x ^= x >> 16
        x = x * 0x7FEB352D & M
        x ^= x >> 15
        x = x * 0x846CA68B & M
        return x ^ (x >> 16)

    i = 130
    h = mix(mix(mix(mix(1 ^ 7) ^ (3 * 0x9E3779B9 & M)) ^ (i >> 7) ^ 0x12345678) ^ (i & 127))
    assert (a[i], b[i]) == ((h & 0xFFFF) / 65536, (h >> 16) / 65536)


def test_a_step_of_the_random_rounding_is_unbiased():
    """Mean over the fractions of floor(t + u) is t, and never more than one step away."""
    s, t, width = O.steps_of(np.array([3.0, 448.0, 0.013, 2.0 ** -9 * 0.3, 0.0]))
    assert s[0] == 127
    u = np.arange(65536) / 65536
    for k in range(5):
        f = np.floor(t[k] + u)
        assert abs(f.mean() - t[k]) <= 2.0 ** -16 and np.abs(f - t[k]).max() < 1
    np.testing.assert_allclose(t * width, [3.0, 448.0, 0.013, 2.0 ** -9 * 0.3, 0.0], rtol=1e-15)
