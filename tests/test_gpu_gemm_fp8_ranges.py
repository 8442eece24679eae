"""Ends of the range of the 8-bit product's operands, on every kernel (tests/fp8_paths.py): what the two types of results take."""
import pytest
import torch

import paper_2203_17189_amd as P
from fp8_paths import IDS, SHAPES
from fp8_util import DT

pytestmark = pytest.mark.gpu


def whole(rows, k, code, byte):
    """A matrix of one code under one scale."""
    q = torch.full((rows, -(-k // 16) * 16), code, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :k]
    return q, torch.full((rows, -(-k // 512) * 4), byte, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)[:, :-(-k // 128)]


@pytest.mark.parametrize("m,n,k,out,kernel", SHAPES, ids=IDS)
def test_elements_of_2_to_the_128_and_more(m, n, k, out, kernel):
    """Finite products with bfloat16 results, whose scales stay apart; infinite ones with float32 results, for which elements
    are widened.  Below, both are exact: 240 K is a whole number of at most 24 bits."""
    assert path_of(m, n, k, out) == kernel
    for code, byte, value in ((0x78, 247, 2.0 ** 128), (0x7E, 254, 448 * 2.0 ** 127), (0x77, 247, 240 * 2.0 ** 120)):
        for small in (37, 60):  # of B: 2^-90, 2^-67
            for turned in (False, True):
                a, b = whole(m, k, *((0x38, small) if turned else (code, byte))), whole(n, k, *((code, byte) if turned else (0x38, small)))
                want = torch.tensor(value * 2.0 ** (small - 127) * k, dtype=torch.float64).to(DT[out]).item()
                if out == "f32" and value >= 2.0 ** 128:
                    want = float("inf")
                c = P.t5_gemm_fp8(*a, *b, out_dtype=DT[out])
                assert bool((c == want).all()), (hex(code), byte, small, turned, c[0, 0].item(), want)


def path_of(m, n, k, out):
    return P.t5_gemm_fp8_kernel_path(m, n, k, DT[out])


def test_the_largest_float32_quantises_to_2_to_the_128():
    x = torch.full((3, 256), torch.finfo(torch.float32).max, device="cuda")
    q, s, _, _ = P.t5_quantize_fp8(x)
    assert bool((q.view(torch.uint8) == 0x78).all()) and bool((s.view(torch.uint8) == 247).all())
    one = whole(40, 256, 0x38, 100)
    assert bool((P.t5_gemm_fp8(q, s, *one) == 2.0 ** (128 + 100 - 127 + 8)).all())
    assert bool(P.t5_gemm_fp8(q, s, *one, out_dtype=torch.float32).isinf().all())
    # the largest that stays below
    x.fill_(247 * 2.0 ** 120)
    q, s, _, _ = P.t5_quantize_fp8(x)
    assert bool((P.t5_gemm_fp8(q, s, *one, out_dtype=torch.float32) == 240 * 2.0 ** (120 - 27 + 8)).all())
