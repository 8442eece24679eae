"""Arguments of the operators of training in 8 bits that are no rows of memory, or not where the others are."""
import numpy as np
import pytest
import torch

import paper_2203_17189_amd as P
from oracle import fp8_oracle as O
from fp8_util import codes, host

pytestmark = pytest.mark.gpu


def not_strided(x):
    return [x.to_sparse_csr(), x.to_sparse_csc(), x.to_sparse_bsr((2, 2)), x.to_sparse(), torch.nested.nested_tensor([x[:1], x[1:]]),
            torch.nested.nested_tensor([x[:1], x[1:]], layout=torch.jagged)]


@pytest.mark.filterwarnings("ignore")
def test_sparse_and_nested_tensors_are_refused():
    """Asked for its strides or its memory, such a tensor throws: that has to become an exception of Python's."""
    x = torch.randn(4, 512, device="cuda")
    q, s, _, _ = P.t5_quantize_fp8(x)
    out = torch.zeros(4, 4, device="cuda")
    flat = lambda: torch.zeros(8, device="cuda")  # noqa: E731
    for t in not_strided(x):
        with pytest.raises(ValueError):
            P.t5_quantize_fp8(t)
        for at in range(4):
            args = [q, s, q, s]
            args[at] = t
            with pytest.raises(ValueError):
                P.t5_gemm_fp8(*args)
        for name in ("param", "grad", "m", "v"):
            entry = dict(param=flat(), grad=flat(), m=flat(), v=flat())
            entry[name] = t
            with pytest.raises(ValueError):
                P.adamw_step_multi([entry], step=1, lr=1e-3)
    for t in not_strided(out):
        with pytest.raises(ValueError):
            P.t5_gemm_fp8(q, s, q, s, out=t)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("cols", [1, 2, 3, 4])
def test_few_columns_of_rows_of_four(cols, block_rows):
    """A matrix whose memory ends with its last element."""
    rows = 130
    x = torch.zeros(4 * (rows - 1) + cols, device="cuda").as_strided((rows, cols), (4, 1))
    x.copy_(torch.from_numpy(np.random.default_rng(cols).standard_normal((rows, cols)).astype(np.float32)))
    out = P.t5_quantize_fp8(x, block_rows=block_rows, transposed=True)
    for a, q, s in ((host(x), *out[:2]), (host(x).T, *out[2:])):
        wq, ws = O.quantize(a, "e4m3", block_rows)
        assert (codes(q) == wq).all() and (codes(s) == ws).all()
    if block_rows == 1:
        assert (codes(P.t5_quantize_fp8(x)[0]) == codes(out[0])).all()
