"""Arguments of the operators of training in 8 bits that are no rows of memory, or not where the others are."""
import pytest
import torch

import paper_2203_17189_amd as P

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
