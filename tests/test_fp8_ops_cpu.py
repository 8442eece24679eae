"""Refusals of the operators of training in 8 bits: every one precedes device work, so they run on a host without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2203_17189_amd as P
from paper_2203_17189_amd import binding as B

D = C.c_void_p(4096)  # never dereferenced
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4
nan, inf = float("nan"), float("inf")


def _quant(**kw):
    return B._QuantizeCfg(*{**dict(rows=8, cols=130, ld=130, dtype=1, q_dtype=2, block_rows=1), **kw}.values())


def _gemm(**kw):
    return B._GemmFp8Cfg(*{**dict(M=8, N=16, K=200, lda=208, ldb=208, ldc=16, lsa=4, lsb=4, a_dtype=2, b_dtype=3, a_block_rows=1,
                                  b_block_rows=128, c_dtype=1, accumulate=0), **kw}.values())


def _tensor(**kw):
    return B._AdamTensor(*{**dict(param=4096, grad=4096, m=4096, v=4096, m_scale=4096, v_scale=4096, bf16_copy_out=None, n=10, grad_dtype=0,
                                  state_bits=8, weight_decay=0.1), **kw}.values())


def _adam(**kw):
    return B._AdamCfg(*{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed_lo=0, seed_hi=0, grad_scale=None), **kw}.values())


@pytest.mark.parametrize("kw,rc", [(dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(ld=129), SHAPE), (dict(block_rows=0), SHAPE),
                                   (dict(block_rows=64), SHAPE), (dict(rows=(1 << 31) - 128), UNSUPPORTED),
                                   (dict(cols=(1 << 23) + 1, ld=1 << 24), UNSUPPORTED), (dict(ld=(1 << 32) + 1), UNSUPPORTED),
                                   (dict(rows=1 << 30, cols=1, ld=1), UNSUPPORTED),
                                   (dict(dtype=2), UNSUPPORTED), (dict(q_dtype=1), UNSUPPORTED), (dict(q_dtype=4), UNSUPPORTED)], ids=str)
def test_quantize_refusals(kw, rc):
    assert P.lib().t5_quantize_fp8(C.byref(_quant(**kw)), D, D, D, D, D, None) == rc


def test_quantize_nulls_and_alignment():
    L, c = P.lib(), C.byref(_quant())
    f = L.t5_quantize_fp8
    assert f(None, D, D, D, D, D, None) == NULL
    for args in ((None, D, D, D, D), (D, None, None, None, None), (D, D, None, None, None), (D, None, D, None, None), (D, None, None, D, None),
                 (D, D, D, None, D)):
        assert f(c, *args, None) == NULL
    odd = C.c_void_p(4096 + 8)
    assert f(c, D, odd, D, D, D, None) == UNSUPPORTED and f(c, D, D, D, odd, D, None) == UNSUPPORTED
    odd = C.c_void_p(4096 + 2)
    assert f(c, D, D, odd, D, D, None) == UNSUPPORTED and f(c, D, D, D, D, odd, None) == UNSUPPORTED
    assert f(c, C.c_void_p(4097), D, D, D, D, None) == UNSUPPORTED
    assert f(C.byref(_quant(rows=0)), None, None, None, None, None, None) == 0
    many = C.byref(_quant(rows=1 << 29, cols=1, ld=1))  # threads of one launch
    assert f(many, D, D, D, None, None, None) == UNSUPPORTED
    assert [L.t5_fp8_ld(n) for n in (1, 16, 17, 128)] == [16, 16, 32, 128]
    assert [L.t5_fp8_scale_ld(n) for n in (1, 128, 512, 513)] == [4, 4, 4, 8]


@pytest.mark.parametrize("kw,rc", [(dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(lda=192), SHAPE), (dict(ldb=192), SHAPE),
                                   (dict(ldc=15), SHAPE), (dict(K=513, lda=528, ldb=528), SHAPE), (dict(lsa=1), SHAPE), (dict(a_block_rows=2), SHAPE),
                                   (dict(b_block_rows=0), SHAPE), (dict(a_dtype=1), UNSUPPORTED), (dict(b_dtype=4), UNSUPPORTED),
                                   (dict(c_dtype=2), UNSUPPORTED), (dict(accumulate=1), UNSUPPORTED), (dict(lda=200), UNSUPPORTED),
                                   (dict(ldb=(1 << 23) + 16), UNSUPPORTED), (dict(lsa=6), UNSUPPORTED), (dict(lsb=(1 << 20) + 4), UNSUPPORTED),
                                   (dict(ldc=(1 << 32) + 1), UNSUPPORTED), (dict(M=(1 << 30) + 1), UNSUPPORTED)], ids=str)
def test_gemm_refusals(kw, rc):
    L, c = P.lib(), C.byref(_gemm(**kw))
    assert L.t5_gemm_fp8(c, D, D, D, D, D, D, 1 << 40, None) == rc
    assert L.t5_gemm_fp8_workspace_bytes(c) == 0


def test_gemm_nulls_alignment_and_workspace():
    L = P.lib()
    f, c = L.t5_gemm_fp8, C.byref(_gemm())
    assert f(None, D, D, D, D, D, D, 1 << 40, None) == NULL
    for i in range(5):
        a = [D] * 5
        a[i] = None
        assert f(c, *a, D, 1 << 40, None) == NULL
        a[i] = C.c_void_p(4096 + (8 if i in (0, 2) else 2 if i in (1, 3) else 1))
        assert f(c, *a, D, 1 << 40, None) == UNSUPPORTED
    long = C.byref(_gemm(M=300, N=300, ldc=300, K=40000, lda=40000, ldb=40000, lsa=316, lsb=316, c_dtype=0))
    need = L.t5_gemm_fp8_workspace_bytes(long)
    assert need > 0
    assert f(long, D, D, D, D, D, None, 1 << 40, None) == NULL
    assert f(long, D, D, D, D, D, D, need - 1, None) == WORKSPACE
    assert f(long, D, D, D, D, D, C.c_void_p(4096 + 128), need, None) == WORKSPACE
    assert f(C.byref(_gemm(M=0)), None, None, None, None, None, None, 0, None) == 0


@pytest.mark.parametrize("kw,rc", [(dict(lr=-1e-3), SHAPE), (dict(lr=nan), SHAPE), (dict(lr=inf), SHAPE), (dict(beta1=1.0), SHAPE), (dict(beta1=-0.1), SHAPE),
                                   (dict(beta2=1.0), SHAPE), (dict(beta2=nan), SHAPE), (dict(eps=0.0), SHAPE), (dict(eps=1e-31), SHAPE),
                                   (dict(eps=inf), SHAPE), (dict(eps=nan), SHAPE), (dict(step=0), SHAPE), (dict(grad_scale=4098), UNSUPPORTED)], ids=str)
def test_adamw_refusals(kw, rc):
    t = (B._AdamTensor * 1)(_tensor())
    assert P.lib().adamw_step_multi(t, 1, C.byref(_adam(**kw)), None) == rc


@pytest.mark.parametrize("kw,rc", [(dict(n=0), SHAPE), (dict(weight_decay=-0.1), SHAPE), (dict(weight_decay=inf), SHAPE), (dict(n=(1 << 34) + 1), UNSUPPORTED),
                                   (dict(state_bits=16), UNSUPPORTED), (dict(grad_dtype=2), UNSUPPORTED), (dict(param=None), NULL), (dict(grad=None), NULL),
                                   (dict(m=None), NULL), (dict(v=None), NULL), (dict(m_scale=None), NULL), (dict(v_scale=None), NULL),
                                   (dict(param=4098), UNSUPPORTED), (dict(grad=4098), UNSUPPORTED), (dict(grad=4097, grad_dtype=1), UNSUPPORTED),
                                   (dict(state_bits=32, m=4097), UNSUPPORTED), (dict(bf16_copy_out=4097), UNSUPPORTED)], ids=str)
def test_adamw_tensor_refusals(kw, rc):
    """One bad entry anywhere in a list refuses the whole call."""
    L, c = P.lib(), C.byref(_adam())
    good = [_tensor(param=(1 << 20) + 4096 * i) for i in range(70)]
    for at in (0, 45, 69):
        ts = list(good)
        ts[at] = _tensor(**{"param": (1 << 20) + 4096 * at, **kw})
        assert L.adamw_step_multi((B._AdamTensor * 70)(*ts), 70, c, None) == rc


def test_adamw_lists():
    L, c = P.lib(), C.byref(_adam())
    t = (B._AdamTensor * 1)(_tensor())
    assert L.adamw_step_multi(None, 1, c, None) == NULL and L.adamw_step_multi(t, 1, None, None) == NULL
    assert L.adamw_step_multi(t, 0, c, None) == SHAPE and L.adamw_step_multi(t, (1 << 16) + 1, c, None) == UNSUPPORTED


@pytest.mark.parametrize("second", [4096, 4096 + 36, 4096 - 36])
def test_adamw_parameters_that_overlap_are_refused(second):
    ts = [_tensor(param=(1 << 20) + 4096 * i) for i in range(50)] + [_tensor(param=4096), _tensor(param=second)]
    assert P.lib().adamw_step_multi((B._AdamTensor * 52)(*ts), 52, C.byref(_adam()), None) == SHAPE


def test_binding_refuses_what_it_can_see():
    x = torch.zeros(4, 256)
    with pytest.raises(ValueError):
        P.t5_quantize_fp8(x)
    with pytest.raises(ValueError):
        P.t5_quantize_fp8(x.to(torch.float16))
    q, s = torch.zeros(4, 256, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(4, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError):
        P.t5_gemm_fp8(q, s, q, s)
    with pytest.raises(ValueError):
        P.t5_gemm_fp8(x, s, q, s)
    with pytest.raises(P.T5Error):
        P.adamw_step_multi([], step=1, lr=1e-3)
    for step in (0, -3, 1 << 31, 1 << 40):
        with pytest.raises(P.T5Error):
            P.adamw_step_multi([{}], step=step, lr=1e-3)
    z = torch.zeros(8)
    with pytest.raises(ValueError):
        P.adamw_step_multi([dict(param=z, grad=z, m=z, v=z)], step=1, lr=1e-3)
