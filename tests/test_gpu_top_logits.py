"""Top logits of each row: values and ids are exactly those of a stable descending sort."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as VO
from vocab_util import dev, host, rows_with_gap

pytestmark = pytest.mark.gpu


def _check(x, k, values, ids):
    v, i = VO.top_logits(host(x), k)
    assert ids.dtype == torch.int32 and values.dtype == torch.float32
    assert np.array_equal(ids.cpu().numpy(), i)
    assert np.array_equal(host(values), v, equal_nan=True)


def _rows(rows, vocab, kind, rng):
    if kind == "equal":      # nothing but ties
        return np.full((rows, vocab), 1.5)
    if kind == "coarse":     # a handful of values
        return np.round(rng.standard_normal((rows, vocab)))
    if kind == "rising":     # the largest side by side, at the end
        return np.tile(np.arange(vocab) / 64.0, (rows, 1))
    if kind == "falling":
        return np.tile(-np.arange(vocab) / 64.0, (rows, 1))
    if kind == "stripes":    # the largest all belong to the pieces of a few threads
        x = rng.standard_normal((rows, vocab))
        return np.where(np.arange(vocab) // 8 % 256 < 3, 50 + x, x)
    if kind == "masked":     # all but a few are -inf; some rows have fewer finite values than are asked for
        x = rng.standard_normal((rows, vocab))
        x[rng.random((rows, vocab)) < 0.9] = -np.inf
        x[0, 1:] = -np.inf
        return x
    if kind == "odd":        # every special value
        x = rng.standard_normal((rows, vocab))
        for val in (np.nan, np.inf, -np.inf, 0.0, -0.0, np.finfo(np.float32).min):
            x[rng.random((rows, vocab)) < 0.1] = val
        return x
    return rng.standard_normal((rows, vocab)) * 3


CASES = [(1, 2, 1), (3, 2, 2), (5, 17, 17), (2, 255, 100), (2, 256, 256), (3, 300, 256), (4, 1000, 8), (2, 2047, 64),
         (3, 2048, 256), (2, 2049, 33), (5, 5000, 1), (40, 32128, 64), (2, 32128, 256), (1, 100003, 100), (3, 131072, 16),
         (300, 509, 12)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["random", "equal", "coarse", "rising", "falling", "stripes", "masked", "odd"])
@pytest.mark.parametrize("rows,vocab,k", CASES)
def test_top(rows, vocab, k, kind, dtype):
    import paper_2203_17189_amd as P
    x = dev(_rows(rows, vocab, kind, np.random.default_rng(vocab + k)), dtype)
    _check(x, k, *P.t5_top_logits(x, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,ld,shift", [(2048, 2056, 0), (2048, 2056, 8), (4000, 4001, 0), (4000, 4100, 3), (333, 1000, 1)])
def test_rows_with_a_longer_stride(vocab, ld, shift, dtype):
    import paper_2203_17189_amd as P
    rng = np.random.default_rng(ld)
    _, x = rows_with_gap(rng.standard_normal((9, vocab)), dtype, ld, shift, fill=float("inf"))
    _check(x, 32, *P.t5_top_logits(x, 32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["random", "equal", "coarse", "stripes", "odd"])
@pytest.mark.parametrize("rows,vocab,k", [(600, 100, 32), (600, 1024, 32), (600, 1025, 33), (700, 4096, 20), (700, 8200, 128), (513, 20000, 200), (300, 70000, 100),
                                          (600, 250, 200), (600, 300, 90), (600, 3000, 31), (550, 8000, 90), (550, 16000, 40), (520, 8000, 12), (600, 200, 60), (700, 1030, 40)])
def test_many_rows(rows, vocab, k, kind, dtype):
    """Rows enough for workgroups that share a compute unit; long rows of the few-rows kernel are above."""
    import paper_2203_17189_amd as P
    x = dev(_rows(rows, vocab, kind, np.random.default_rng(vocab + k)), dtype)
    values, ids = P.t5_top_logits(x, k)
    some = np.r_[0:40, rows - 40:rows]
    _check(x[torch.from_numpy(some).cuda()], k, values[torch.from_numpy(some).cuda()], ids[torch.from_numpy(some).cuda()])
    v2, i2 = P.t5_top_logits(x.flip(0).contiguous(), k)
    assert torch.equal(i2.flip(0), ids) and torch.equal(v2.flip(0).nan_to_num(9e9), values.nan_to_num(9e9))


def test_thousands_of_ties_next_to_the_bound():
    """A few values above, thousands equal to the K-th: the first of those, by id, in rows of one and of several chunks."""
    import paper_2203_17189_amd as P
    for vocab in (900, 4000, 33000, 200000):
        for dtype in ("f32", "bf16"):
            rng = np.random.default_rng(vocab)
            x = np.where(rng.random((4, vocab)) < 0.7, 2.0, -1.0)
            x[:, rng.permutation(vocab)[:20]] = 3.0 + np.arange(20) % 3
            x[1] = np.where(np.arange(vocab) < vocab - 30, -np.inf, 0.0)
            x[2, :] = -np.inf
            for k in (20, 21, 31, 100):
                _check(dev(x, dtype), k, *P.t5_top_logits(dev(x, dtype), k))


@pytest.mark.parametrize("vocab", [900, 4000, 8000, 16000])
def test_ties_in_many_rows(vocab):
    """The same, in the forms that give many rows a wavefront or two each."""
    import paper_2203_17189_amd as P
    for dtype in ("f32", "bf16"):
        rng = np.random.default_rng(vocab)
        x = np.where(rng.random((4, vocab)) < 0.7, 2.0, -1.0)
        x[:, rng.permutation(vocab)[:20]] = 3.0 + np.arange(20) % 3
        x[1] = np.where(np.arange(vocab) < vocab - 30, -np.inf, 0.0)
        x[2, :] = -np.inf
        x[3] = rng.integers(0, 40, vocab)
        rows = dev(x, dtype)
        for k in (20, 31, 60, 96):
            v, i = P.t5_top_logits(rows.repeat(130, 1), k)
            _check(rows, k, v[:4], i[:4])
            assert torch.equal(i.view(130, 4, k), i[:4].expand(130, 4, k)) and torch.equal(v.view(130, 4, k), v[:4].expand(130, 4, k))


def test_empty():
    import paper_2203_17189_amd as P
    v, i = P.t5_top_logits(torch.zeros(0, 10, device="cuda"), 3)
    assert v.shape == i.shape == (0, 3)


def test_rows_beyond_32_bit_offsets():
    """520 rows, 2^23 + 8 elements apart."""
    import paper_2203_17189_amd as P
    rng = np.random.default_rng(8)
    _, x = rows_with_gap(rng.standard_normal((520, 1000)), "bf16", (1 << 23) + 8, fill=float("inf"))
    values, ids = P.t5_top_logits(x, 20)
    want = P.t5_top_logits(x.contiguous(), 20)
    assert torch.equal(values, want[0]) and torch.equal(ids, want[1])
    _check(x[-3:], 20, values[-3:], ids[-3:])
