"""ctypes binding of libt5mi.so.  Argument marshalling only; torch supplies device memory and
streams.  There is no CPU fallback: a missing library raises."""
from __future__ import annotations

import ctypes as C
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

WEIGHT_NAMES = ("ln1_scale", "wq", "wk", "wv", "wo", "rel_table", "ln2_scale", "wi0", "wi1", "wo_ff")
CROSS_WEIGHT_NAMES = ("lnx_scale", "xq", "xk", "xv", "xo")
T5_F32, T5_BF16, T5_E4M3, T5_E5M2 = 0, 1, 2, 3
MLP_KINDS = {"geglu_tanh": 0, "relu": 1, "geglu_erf": 2}


class T5Error(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({t5_status_string(status)})")
        self.status = status


class _Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "seq", "d_model", "n_heads", "d_kv", "d_ff", "num_buckets",
                                         "max_distance", "causal", "dtype")] + \
               [("rms_eps", C.c_float), ("attn_scale", C.c_float), ("mlp_kind", C.c_int32),
                ("dropout_rate", C.c_float), ("dropout_seed_lo", C.c_uint32), ("dropout_seed_hi", C.c_uint32),
                ("deterministic", C.c_int32)]


class _Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES]


class _Grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES]


class _CrossWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in CROSS_WEIGHT_NAMES]


class _CrossGrads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in CROSS_WEIGHT_NAMES]


class _StackCfg(C.Structure):
    _fields_ = [("block", _Cfg), ("n_layers", C.c_int32), ("vocab", C.c_int32), ("tied_logits", C.c_int32),
                ("remat", C.c_int32), ("z_loss", C.c_float)]


class _StackWeights(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("rel_table", C.c_void_p), ("layers", C.POINTER(_Weights)),
                ("final_scale", C.c_void_p), ("logits_w", C.c_void_p)]


class _StackGrads(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("rel_table", C.c_void_p), ("layers", C.POINTER(_Grads)),
                ("final_scale", C.c_void_p), ("logits_w", C.c_void_p)]


class _EncDecCfg(C.Structure):
    _fields_ = [("enc_block", _Cfg), ("dec_block", _Cfg), ("n_enc_layers", C.c_int32), ("n_dec_layers", C.c_int32),
                ("vocab", C.c_int32), ("tied_logits", C.c_int32), ("remat", C.c_int32), ("z_loss", C.c_float)]


class _EncDecWeights(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("enc_rel_table", C.c_void_p), ("enc_layers", C.POINTER(_Weights)),
                ("enc_final_scale", C.c_void_p), ("dec_rel_table", C.c_void_p), ("dec_layers", C.POINTER(_Weights)),
                ("dec_cross", C.POINTER(_CrossWeights)), ("dec_final_scale", C.c_void_p), ("logits_w", C.c_void_p)]


class _EncDecGrads(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("enc_rel_table", C.c_void_p), ("enc_layers", C.POINTER(_Grads)),
                ("enc_final_scale", C.c_void_p), ("dec_rel_table", C.c_void_p), ("dec_layers", C.POINTER(_Grads)),
                ("dec_cross", C.POINTER(_CrossGrads)), ("dec_final_scale", C.c_void_p), ("logits_w", C.c_void_p)]


class _EmbedCfg(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("vocab", C.c_int32), ("d_model", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float)]


class _TopCfg(C.Structure):
    _fields_ = [("rows", C.c_int64), ("ld", C.c_int64), ("vocab", C.c_int32), ("top_k", C.c_int32), ("dtype", C.c_int32)]


class _DistillCfg(C.Structure):
    _fields_ = _TopCfg._fields_ + [("temperature", C.c_float), ("soft_weight", C.c_float), ("z_loss", C.c_float),
                                 ("dlogits_ld", C.c_int64)]


class _DistillOpts(C.Structure):
    _fields_ = [("top_k", C.c_int32), ("temperature", C.c_float), ("soft_weight", C.c_float)]


class _QuantizeCfg(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("dtype", C.c_int32), ("q_dtype", C.c_int32),
                ("block_rows", C.c_int32)]


class _GemmFp8Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("M", "N", "K")] + [(n, C.c_int64) for n in ("lda", "ldb", "ldc", "lsa", "lsb")] + \
               [(n, C.c_int32) for n in ("a_dtype", "b_dtype", "a_block_rows", "b_block_rows", "c_dtype", "accumulate")]


class _AdamTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "bf16_copy_out")] + \
               [("n", C.c_int64), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("weight_decay", C.c_double)]


class _AdamCfg(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps")] + \
               [("step", C.c_int32), ("seed_lo", C.c_uint32), ("seed_hi", C.c_uint32), ("grad_scale", C.c_void_p)]


class _AfTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("v_row", C.c_void_p), ("v_col", C.c_void_p),
                ("v_full", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("factored", C.c_int32),
                ("bf16_copy_out", C.c_void_p), ("m", C.c_void_p)]


class _AfCfg(C.Structure):
    _fields_ = [("lr", C.c_float), ("decay_pow", C.c_float), ("eps1", C.c_float), ("eps2", C.c_float),
                ("clip", C.c_float), ("scale_by_param", C.c_int32), ("step", C.c_int32), ("beta1", C.c_float),
                ("weight_decay", C.c_float)]


def lib_path() -> str:
    return os.path.join(_HERE, "libt5mi.so")


def lib() -> C.CDLL:
    """Load libt5mi.so (building it first if it is not there).  Raises if that fails."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        from . import build as _build
        _build.build(verbose=False)
    L = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
    L.t5_status_string.restype = C.c_char_p
    L.t5_status_string.argtypes = [i32]
    L.t5_relpos_bucket.restype = i32
    L.t5_relpos_bucket.argtypes = [vp, vp, i64, i32, i32, i32, vp]
    L.t5_dropout_keep.restype = i32
    L.t5_dropout_keep.argtypes = [C.c_uint64, i32, C.c_float, i64, i64, vp, vp]
    L.t5_block_kernel_path.restype = i32
    L.t5_block_kernel_path.argtypes = [C.POINTER(_Cfg), i32]
    L.t5_block_stash_bytes.restype = sz
    L.t5_block_stash_bytes.argtypes = [C.POINTER(_Cfg)]
    L.t5_block_workspace_bytes.restype = sz
    L.t5_block_workspace_bytes.argtypes = [C.POINTER(_Cfg)]
    L.t5_block_fwd.restype = i32
    L.t5_block_fwd.argtypes = [C.POINTER(_Cfg), vp, C.POINTER(_Weights), vp, vp, vp, sz, vp]
    L.t5_block_bwd.restype = i32
    L.t5_block_bwd.argtypes = [C.POINTER(_Cfg), vp, vp, C.POINTER(_Weights), vp, vp, C.POINTER(_Grads), i32,
                               vp, sz, vp]
    L.t5_decoder_block_stash_bytes.restype = sz
    L.t5_decoder_block_stash_bytes.argtypes = [C.POINTER(_Cfg), C.c_int32]
    L.t5_decoder_block_workspace_bytes.restype = sz
    L.t5_decoder_block_workspace_bytes.argtypes = [C.POINTER(_Cfg), C.c_int32]
    L.t5_decoder_block_fwd.restype = i32
    L.t5_decoder_block_fwd.argtypes = [C.POINTER(_Cfg), C.c_int32, vp, vp, C.POINTER(_Weights),
                                       C.POINTER(_CrossWeights), vp, vp, vp, sz, vp]
    L.t5_decoder_block_bwd.restype = i32
    L.t5_decoder_block_bwd.argtypes = [C.POINTER(_Cfg), C.c_int32, vp, vp, vp, C.POINTER(_Weights),
                                       C.POINTER(_CrossWeights), vp, vp, vp, C.POINTER(_Grads),
                                       C.POINTER(_CrossGrads), i32, vp, sz, vp]
    L.t5_stack_workspace_bytes.restype = sz
    L.t5_stack_workspace_bytes.argtypes = [C.POINTER(_StackCfg)]
    L.t5_stack_loss_and_grad.restype = i32
    L.t5_stack_loss_and_grad.argtypes = [C.POINTER(_StackCfg), vp, vp, C.POINTER(_StackWeights), vp,
                                         C.POINTER(_StackGrads), i32, vp, sz, vp]
    L.t5_encdec_workspace_bytes.restype = sz
    L.t5_encdec_workspace_bytes.argtypes = [C.POINTER(_EncDecCfg)]
    L.t5_encdec_loss_and_grad.restype = i32
    L.t5_encdec_loss_and_grad.argtypes = [C.POINTER(_EncDecCfg), vp, vp, vp, C.POINTER(_EncDecWeights), vp,
                                          C.POINTER(_EncDecGrads), i32, vp, sz, vp]
    L.t5_stack_top_logits_workspace_bytes.restype = sz
    L.t5_stack_top_logits_workspace_bytes.argtypes = [C.POINTER(_StackCfg), C.c_int32]
    L.t5_stack_top_logits.restype = i32
    L.t5_stack_top_logits.argtypes = [C.POINTER(_StackCfg), vp, C.POINTER(_StackWeights), C.c_int32, vp, vp, vp, sz, vp]
    L.t5_encdec_top_logits_workspace_bytes.restype = sz
    L.t5_encdec_top_logits_workspace_bytes.argtypes = [C.POINTER(_EncDecCfg), C.c_int32]
    L.t5_encdec_top_logits.restype = i32
    L.t5_encdec_top_logits.argtypes = [C.POINTER(_EncDecCfg), vp, vp, C.POINTER(_EncDecWeights), C.c_int32, vp, vp, vp, sz, vp]
    L.t5_stack_distill_workspace_bytes.restype = sz
    L.t5_stack_distill_workspace_bytes.argtypes = [C.POINTER(_StackCfg), C.POINTER(_DistillOpts)]
    L.t5_stack_distill_loss_and_grad.restype = i32
    L.t5_stack_distill_loss_and_grad.argtypes = [C.POINTER(_StackCfg), C.POINTER(_DistillOpts), vp, vp, vp, vp,
                                                 C.POINTER(_StackWeights), vp, C.POINTER(_StackGrads), i32, vp, sz, vp]
    L.t5_encdec_distill_workspace_bytes.restype = sz
    L.t5_encdec_distill_workspace_bytes.argtypes = [C.POINTER(_EncDecCfg), C.POINTER(_DistillOpts)]
    L.t5_encdec_distill_loss_and_grad.restype = i32
    L.t5_encdec_distill_loss_and_grad.argtypes = [C.POINTER(_EncDecCfg), C.POINTER(_DistillOpts), vp, vp, vp, vp, vp,
                                                  C.POINTER(_EncDecWeights), vp, C.POINTER(_EncDecGrads), i32, vp, sz, vp]
    L.adafactor_workspace_bytes.restype = sz
    L.adafactor_workspace_bytes.argtypes = [i64, i64, i32]
    L.adafactor_step.restype = i32
    L.adafactor_step.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, C.POINTER(_AfCfg), vp, vp, sz, vp]
    L.adafactor_step_static.restype = i32
    L.adafactor_step_static.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, C.POINTER(_AfCfg), vp, vp]
    L.adafactor_multi_workspace_bytes.restype = sz
    L.adafactor_multi_workspace_bytes.argtypes = [C.POINTER(_AfTensor), i32]
    L.adafactor_step_multi.restype = i32
    L.adafactor_step_multi.argtypes = [C.POINTER(_AfTensor), i32, C.POINTER(_AfCfg), vp, sz, vp]
    L.t5_embed_fwd.restype = i32
    L.t5_embed_fwd.argtypes = [C.POINTER(_EmbedCfg), vp, vp, vp, vp]
    L.t5_embed_bwd_workspace_bytes.restype = sz
    L.t5_embed_bwd_workspace_bytes.argtypes = [C.POINTER(_EmbedCfg)]
    L.t5_embed_bwd.restype = i32
    L.t5_embed_bwd.argtypes = [C.POINTER(_EmbedCfg), vp, vp, vp, i32, vp, sz, vp]
    L.t5_top_logits.restype = i32
    L.t5_top_logits.argtypes = [C.POINTER(_TopCfg), vp, vp, vp, vp]
    L.t5_distill_workspace_bytes.restype = sz
    L.t5_distill_workspace_bytes.argtypes = [C.POINTER(_DistillCfg)]
    L.t5_distill_loss_and_grad.restype = i32
    L.t5_distill_loss_and_grad.argtypes = [C.POINTER(_DistillCfg), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.t5_gemm_bf16.restype = i32
    L.t5_gemm_bf16.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, vp]
    L.t5_fp8_ld.restype = i64
    L.t5_fp8_ld.argtypes = [i64]
    L.t5_fp8_scale_ld.restype = i64
    L.t5_fp8_scale_ld.argtypes = [i64]
    L.t5_quantize_fp8.restype = i32
    L.t5_quantize_fp8.argtypes = [C.POINTER(_QuantizeCfg), vp, vp, vp, vp, vp, vp]
    L.t5_gemm_fp8_workspace_bytes.restype = sz
    L.t5_gemm_fp8_workspace_bytes.argtypes = [C.POINTER(_GemmFp8Cfg)]
    L.t5_gemm_fp8_kernel_path.restype = i32
    L.t5_gemm_fp8_kernel_path.argtypes = [C.POINTER(_GemmFp8Cfg)]
    L.t5_gemm_fp8.restype = i32
    L.t5_gemm_fp8.argtypes = [C.POINTER(_GemmFp8Cfg), vp, vp, vp, vp, vp, vp, sz, vp]
    L.adamw_step_multi.restype = i32
    L.adamw_step_multi.argtypes = [C.POINTER(_AdamTensor), i32, C.POINTER(_AdamCfg), vp]
    L.t5_wgrad_overlap_enable.restype = i32
    L.t5_wgrad_overlap_enable.argtypes = [i32]
    L.t5_step_timing_enable.restype = None
    L.t5_step_timing_enable.argtypes = [i32]
    L.t5_mfma_peak_probe.restype = i32
    L.t5_mfma_peak_probe.argtypes = [i32, i32, i32, vp, vp]
    L.t5_step_timing_read.restype = i32
    L.t5_step_timing_read.argtypes = [C.POINTER(C.c_char_p), C.POINTER(C.c_float), C.POINTER(i32), i32]
    _LIB = L
    return L


def t5_status_string(status: int) -> str:
    return lib().t5_status_string(int(status)).decode()


def _cfg_struct(cfg) -> _Cfg:
    dt = cfg.dtype
    if isinstance(dt, str):
        dt = {"f32": T5_F32, "bf16": T5_BF16}[dt]
    return _Cfg(cfg.batch, cfg.seq, cfg.d_model, cfg.n_heads, cfg.d_kv, cfg.d_ff, cfg.num_buckets,
                cfg.max_distance, int(bool(cfg.causal)), int(dt), float(cfg.rms_eps), float(cfg.attn_scale),
                MLP_KINDS[getattr(cfg, "mlp", "geglu_tanh")], float(getattr(cfg, "dropout_rate", 0.0)),
                int(getattr(cfg, "dropout_seed", 0)) & 0xFFFFFFFF, (int(getattr(cfg, "dropout_seed", 0)) >> 32) & 0xFFFFFFFF,
                int(bool(getattr(cfg, "deterministic", False))))


def _torch_dtype(cfg):
    dt = cfg.dtype
    return torch.bfloat16 if dt in ("bf16", T5_BF16) else torch.float32


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _strided(t):
    """Whether a tensor has strides (sparse and nested ones raise errors of torch's own when asked for theirs)."""
    return t.layout is torch.strided and not t.is_nested


def _check_tensor(t, dtype, numel, name):
    if not _strided(t):
        raise ValueError(f"{name}: need a strided tensor, got layout {t.layout}{', nested' if t.is_nested else ''}")
    if not t.is_cuda or not t.is_contiguous() or t.dtype != dtype or t.numel() != numel:
        raise ValueError(f"{name}: need a contiguous cuda tensor of {dtype} with {numel} elements, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def t5_relpos_bucket(rel_pos: torch.Tensor, bidirectional: bool, num_buckets: int = 32,
                     max_distance: int = 128, out: torch.Tensor | None = None) -> torch.Tensor:
    _check_tensor(rel_pos, torch.int32, rel_pos.numel(), "rel_pos")
    if out is None:
        out = torch.empty_like(rel_pos)
    rc = lib().t5_relpos_bucket(_ptr(rel_pos), _ptr(out), rel_pos.numel(), int(bool(bidirectional)),
                                int(num_buckets), int(max_distance), _stream())
    if rc:
        raise T5Error(rc, "t5_relpos_bucket")
    return out


def t5_dropout_keep(seed: int, site: int, rate: float, rows: int, cols: int) -> torch.Tensor:
    """uint8 [rows, cols] keep mask (1 = kept) of a dropout site, as the block's kernels regenerate it."""
    out = torch.empty(rows, cols, dtype=torch.uint8, device="cuda")
    rc = lib().t5_dropout_keep(C.c_uint64(int(seed) & (2 ** 64 - 1)), int(site), float(rate), int(rows), int(cols),
                               _ptr(out), _stream())
    if rc:
        raise T5Error(rc, "t5_dropout_keep")
    return out


PATH_MFMA_GEMM, PATH_MFMA_ATTN_FWD, PATH_MFMA_ATTN_BWD, PATH_MFMA_CROSS_ATTN = 1, 2, 4, 8


def t5_block_kernel_path(cfg) -> int:
    """Bit mask of the kernel families the configuration runs on (host-side query; -1: invalid configuration)."""
    return int(lib().t5_block_kernel_path(C.byref(_cfg_struct(cfg)), int(getattr(cfg, "enc_seq", 0))))


def t5_block_stash_bytes(cfg) -> int:
    return int(lib().t5_block_stash_bytes(C.byref(_cfg_struct(cfg))))


def t5_block_workspace_bytes(cfg) -> int:
    return int(lib().t5_block_workspace_bytes(C.byref(_cfg_struct(cfg))))


def _block_names(cfg, names=WEIGHT_NAMES):
    """Tensor names of a block: the ungated ReLU feed-forward has no wi1."""
    return tuple(n for n in names if not (n == "wi1" and getattr(cfg, "mlp", "geglu_tanh") == "relu"))


def _addr(d, n):
    t = d.get(n)
    return None if t is None else t.data_ptr()


def _weights_struct(cfg, weights) -> _Weights:
    dt = _torch_dtype(cfg)
    inner = cfg.n_heads * cfg.d_kv
    shapes = {"ln1_scale": cfg.d_model, "ln2_scale": cfg.d_model, "wq": cfg.d_model * inner,
              "wk": cfg.d_model * inner, "wv": cfg.d_model * inner, "wo": inner * cfg.d_model,
              "rel_table": cfg.num_buckets * cfg.n_heads, "wi0": cfg.d_model * cfg.d_ff,
              "wi1": cfg.d_model * cfg.d_ff, "wo_ff": cfg.d_ff * cfg.d_model}
    names = _block_names(cfg)
    for n in names:
        _check_tensor(weights[n], dt, shapes[n], n)
    return _Weights(*[(_addr(weights, n) if n in names else None) for n in WEIGHT_NAMES])


def _byte_buffer(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def t5_block_fwd(cfg, x, weights, y=None, stash=None, workspace=None):
    """Returns (y, stash).  stash/workspace are uint8 cuda tensors (allocated here if None)."""
    cs = _cfg_struct(cfg)
    dt = _torch_dtype(cfg)
    n = cfg.batch * cfg.seq * cfg.d_model
    _check_tensor(x, dt, n, "x")
    ws = _weights_struct(cfg, weights)
    if y is None:
        y = torch.empty_like(x)
    _check_tensor(y, dt, n, "y")
    if stash is None:
        stash = _byte_buffer(lib().t5_block_stash_bytes(C.byref(cs)), x.device)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_block_workspace_bytes(C.byref(cs)), x.device)
    rc = lib().t5_block_fwd(C.byref(cs), _ptr(x), C.byref(ws), _ptr(y), _ptr(stash), _ptr(workspace),
                            workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "t5_block_fwd")
    return y, stash


def alloc_grads(cfg, weights) -> dict:
    return {n: torch.zeros(weights[n].shape, dtype=torch.float32, device=weights[n].device)
            for n in _block_names(cfg)}


def t5_block_bwd(cfg, dy, x, weights, stash, dx=None, grads=None, accumulate=False, workspace=None):
    """Returns (dx, grads); grads is a dict of float32 tensors shaped like the weights."""
    cs = _cfg_struct(cfg)
    dt = _torch_dtype(cfg)
    n = cfg.batch * cfg.seq * cfg.d_model
    _check_tensor(dy, dt, n, "dy")
    _check_tensor(x, dt, n, "x")
    ws = _weights_struct(cfg, weights)
    if dx is None:
        dx = torch.empty_like(dy)
    _check_tensor(dx, dt, n, "dx")
    if grads is None:
        grads = alloc_grads(cfg, weights)
    for nme in _block_names(cfg):
        _check_tensor(grads[nme], torch.float32, weights[nme].numel(), "grad " + nme)
    gs = _Grads(*[_addr(grads, nme) for nme in WEIGHT_NAMES])
    if workspace is None:
        workspace = _byte_buffer(lib().t5_block_workspace_bytes(C.byref(cs)), x.device)
    rc = lib().t5_block_bwd(C.byref(cs), _ptr(dy), _ptr(x), C.byref(ws), _ptr(stash), _ptr(dx), C.byref(gs),
                            int(bool(accumulate)), _ptr(workspace), workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "t5_block_bwd")
    return dx, grads


def t5_decoder_block_stash_bytes(cfg) -> int:
    return int(lib().t5_decoder_block_stash_bytes(C.byref(_cfg_struct(cfg)), int(cfg.enc_seq)))


def t5_decoder_block_workspace_bytes(cfg) -> int:
    return int(lib().t5_decoder_block_workspace_bytes(C.byref(_cfg_struct(cfg)), int(cfg.enc_seq)))


def _cross_weights_struct(cfg, weights) -> _CrossWeights:
    dt = _torch_dtype(cfg)
    inner = cfg.n_heads * cfg.d_kv
    shapes = {"lnx_scale": cfg.d_model, "xq": cfg.d_model * inner, "xk": cfg.d_model * inner,
              "xv": cfg.d_model * inner, "xo": inner * cfg.d_model}
    for n in CROSS_WEIGHT_NAMES:
        _check_tensor(weights[n], dt, shapes[n], n)
    return _CrossWeights(*[weights[n].data_ptr() for n in CROSS_WEIGHT_NAMES])


def t5_decoder_block_fwd(cfg, x, enc, weights, y=None, stash=None, workspace=None):
    """Decoder layer with cross-attention over enc [batch, cfg.enc_seq, d_model].  weights holds the
    block's ten tensors and the five cross-attention tensors.  Returns (y, stash)."""
    cs = _cfg_struct(cfg)
    dt = _torch_dtype(cfg)
    n = cfg.batch * cfg.seq * cfg.d_model
    _check_tensor(x, dt, n, "x")
    _check_tensor(enc, dt, cfg.batch * cfg.enc_seq * cfg.d_model, "enc")
    ws = _weights_struct(cfg, weights)
    xs = _cross_weights_struct(cfg, weights)
    if y is None:
        y = torch.empty_like(x)
    _check_tensor(y, dt, n, "y")
    es = int(cfg.enc_seq)
    if stash is None:
        stash = _byte_buffer(lib().t5_decoder_block_stash_bytes(C.byref(cs), es), x.device)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_decoder_block_workspace_bytes(C.byref(cs), es), x.device)
    rc = lib().t5_decoder_block_fwd(C.byref(cs), es, _ptr(x), _ptr(enc), C.byref(ws), C.byref(xs), _ptr(y),
                                    _ptr(stash), _ptr(workspace), workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "t5_decoder_block_fwd")
    return y, stash


def alloc_decoder_grads(cfg, weights) -> dict:
    return {n: torch.zeros(weights[n].shape, dtype=torch.float32, device=weights[n].device)
            for n in _block_names(cfg) + CROSS_WEIGHT_NAMES}


def t5_decoder_block_bwd(cfg, dy, x, enc, weights, stash, dx=None, denc=None, grads=None, accumulate=False,
                         workspace=None):
    """Returns (dx, denc, grads); grads is a dict of float32 tensors shaped like the fifteen weights."""
    cs = _cfg_struct(cfg)
    dt = _torch_dtype(cfg)
    n = cfg.batch * cfg.seq * cfg.d_model
    ne = cfg.batch * cfg.enc_seq * cfg.d_model
    _check_tensor(dy, dt, n, "dy")
    _check_tensor(x, dt, n, "x")
    _check_tensor(enc, dt, ne, "enc")
    ws = _weights_struct(cfg, weights)
    xs = _cross_weights_struct(cfg, weights)
    if dx is None:
        dx = torch.empty_like(dy)
    if denc is None:
        denc = torch.empty_like(enc)
    _check_tensor(dx, dt, n, "dx")
    _check_tensor(denc, dt, ne, "denc")
    if grads is None:
        grads = alloc_decoder_grads(cfg, weights)
    for nme in _block_names(cfg) + CROSS_WEIGHT_NAMES:
        _check_tensor(grads[nme], torch.float32, weights[nme].numel(), "grad " + nme)
    gs = _Grads(*[_addr(grads, nme) for nme in WEIGHT_NAMES])
    gx = _CrossGrads(*[grads[nme].data_ptr() for nme in CROSS_WEIGHT_NAMES])
    es = int(cfg.enc_seq)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_decoder_block_workspace_bytes(C.byref(cs), es), x.device)
    rc = lib().t5_decoder_block_bwd(C.byref(cs), es, _ptr(dy), _ptr(x), _ptr(enc), C.byref(ws), C.byref(xs),
                                    _ptr(stash), _ptr(dx), _ptr(denc), C.byref(gs), C.byref(gx),
                                    int(bool(accumulate)), _ptr(workspace), workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "t5_decoder_block_bwd")
    return dx, denc, grads


LAYER_WEIGHT_NAMES = tuple(n for n in WEIGHT_NAMES if n != "rel_table")


def _stack_cfg_struct(sc) -> _StackCfg:
    return _StackCfg(_cfg_struct(sc.block), int(sc.n_layers), int(sc.vocab), int(bool(sc.tied_logits)),
                     int(bool(sc.remat)), float(sc.z_loss))


def t5_stack_workspace_bytes(sc) -> int:
    return int(lib().t5_stack_workspace_bytes(C.byref(_stack_cfg_struct(sc))))


def alloc_stack_grads(sc, weights) -> dict:
    """float32 zero tensors shaped like the stack's weights: {"embedding", "rel_table", "final_scale",
    "logits_w" (untied), "layers": [dict per layer]}."""
    z = lambda t: torch.zeros(t.shape, dtype=torch.float32, device=t.device)
    g = {k: z(weights[k]) for k in ("embedding", "rel_table", "final_scale")}
    if not sc.tied_logits:
        g["logits_w"] = z(weights["logits_w"])
    g["layers"] = [{n: z(lw[n]) for n in _block_names(sc.block, LAYER_WEIGHT_NAMES)} for lw in weights["layers"]]
    return g


def _stack_weights_struct(sc, weights) -> _StackWeights:
    b = sc.block
    dt = _torch_dtype(b)
    _check_tensor(weights["embedding"], dt, sc.vocab * b.d_model, "embedding")
    _check_tensor(weights["rel_table"], dt, b.num_buckets * b.n_heads, "rel_table")
    _check_tensor(weights["final_scale"], dt, b.d_model, "final_scale")
    if not sc.tied_logits:
        _check_tensor(weights["logits_w"], dt, sc.vocab * b.d_model, "logits_w")
    if len(weights["layers"]) != sc.n_layers:
        raise ValueError("weights['layers'] must hold n_layers dicts")
    lw = (_Weights * sc.n_layers)()
    for l, d in enumerate(weights["layers"]):
        lw[l] = _weights_struct(b, dict(d, rel_table=weights["rel_table"]))
    return _StackWeights(weights["embedding"].data_ptr(), weights["rel_table"].data_ptr(), lw,
                         weights["final_scale"].data_ptr(),
                         None if sc.tied_logits else weights["logits_w"].data_ptr())


def _stack_grads_struct(sc, weights, grads) -> _StackGrads:
    b = sc.block
    names = ["embedding", "rel_table", "final_scale"] + ([] if sc.tied_logits else ["logits_w"])
    for nme in names:
        _check_tensor(grads[nme], torch.float32, weights[nme].numel(), "grad " + nme)
    lg = (_Grads * sc.n_layers)()
    for l, d in enumerate(grads["layers"]):
        for nme in _block_names(b, LAYER_WEIGHT_NAMES):
            _check_tensor(d[nme], torch.float32, weights["layers"][l][nme].numel(), f"grad layer {l} {nme}")
        lg[l] = _Grads(*[(_addr(d, nme) if nme != "rel_table" else grads["rel_table"].data_ptr())
                         for nme in WEIGHT_NAMES])
    return _StackGrads(grads["embedding"].data_ptr(), grads["rel_table"].data_ptr(), lg,
                       grads["final_scale"].data_ptr(), None if sc.tied_logits else grads["logits_w"].data_ptr())


def t5_stack_loss_and_grad(sc, tokens, targets, weights, grads=None, want_grads=True, accumulate=False,
                           workspace=None, loss=None):
    """Loss (and gradients) of a stack of blocks with embedding, final norm, logits and cross-entropy with
    z-loss.  weights: {"embedding", "rel_table", "final_scale", "logits_w" (untied), "layers": [dict of the
    block's tensors without rel_table, per layer]}.  Returns (loss tensor of one float32, grads or None)."""
    b = sc.block
    cs = _stack_cfg_struct(sc)
    n_tok = b.batch * b.seq
    _check_tensor(tokens, torch.int32, n_tok, "tokens")
    _check_tensor(targets, torch.int32, n_tok, "targets")
    ws = _stack_weights_struct(sc, weights)
    gs_ref = None
    if want_grads:
        if grads is None:
            grads = alloc_stack_grads(sc, weights)
        gs_ref = C.byref(_stack_grads_struct(sc, weights, grads))
    else:
        grads = None
    if loss is None:
        loss = torch.zeros(1, dtype=torch.float32, device=tokens.device)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_stack_workspace_bytes(C.byref(cs)), tokens.device)
    rc = lib().t5_stack_loss_and_grad(C.byref(cs), _ptr(tokens), _ptr(targets), C.byref(ws), _ptr(loss), gs_ref,
                                      int(bool(accumulate)), _ptr(workspace), workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "t5_stack_loss_and_grad")
    return loss, grads


def _top_outputs(batch, seq, top_k, device, values, ids):
    if values is None:
        values = torch.empty(batch, seq, top_k, dtype=torch.float32, device=device)
    if ids is None:
        ids = torch.empty(batch, seq, top_k, dtype=torch.int32, device=device)
    _check_on(device, values, torch.float32, batch * seq * top_k, "values")
    _check_on(device, ids, torch.int32, batch * seq * top_k, "ids")
    return values, ids


def _model_workspace(workspace, nbytes, device):
    if workspace is None:
        return _byte_buffer(nbytes, device)
    _check_on(device, workspace, torch.uint8, workspace.numel(), "workspace")
    return workspace


def _check_devices(device, tensors, name):
    """No tensor among a model's weights or gradients is on another GPU than its tokens.  (Those that the call reads are on a
    GPU, as their own checks see to; whatever else the caller keeps beside them is of no interest.)"""
    if isinstance(tensors, torch.Tensor):
        if tensors.device.type == device.type and tensors.device != device:
            raise ValueError(f"{name}: on {tensors.device}, other arguments on {device}")
    elif isinstance(tensors, (dict, list, tuple)):
        for key, t in tensors.items() if isinstance(tensors, dict) else enumerate(tensors):
            _check_devices(device, t, f"{name} {key}")


def _loss_buffer(loss, device):
    if loss is None:
        return torch.zeros(1, dtype=torch.float32, device=device)
    _check_on(device, loss, torch.float32, 1, "loss")
    return loss


def _teacher_entries(n_tok, teacher_logits, teacher_ids, device):
    """Entries per position of a teacher's top logits [..., top_k]."""
    k = teacher_ids.shape[-1]
    _check_on(device, teacher_ids, torch.int32, n_tok * k, "teacher_ids")
    _check_on(device, teacher_logits, torch.float32, n_tok * k, "teacher_logits")
    return k


def t5_stack_top_logits(sc, tokens, weights, top_k, values=None, ids=None, workspace=None):
    """Forward pass of a stack; (values float32, ids int32), both [batch, seq, top_k]: the largest logits of every position,
    descending, equal ones by ascending id."""
    b, dev = sc.block, tokens.device
    cs = _stack_cfg_struct(sc)
    _check_tensor(tokens, torch.int32, b.batch * b.seq, "tokens")
    ws = _stack_weights_struct(sc, weights)
    _check_devices(dev, weights, "weights")
    nbytes = lib().t5_stack_top_logits_workspace_bytes(C.byref(cs), _i32(top_k))
    if nbytes:  # (0: the call below says what is wrong)
        values, ids = _top_outputs(b.batch, b.seq, top_k, dev, values, ids)
    workspace = _model_workspace(workspace, nbytes, dev)
    _call(lib().t5_stack_top_logits, "t5_stack_top_logits", dev, C.byref(cs), tokens.data_ptr(), C.byref(ws),
          _i32(top_k), _ptr(values), _ptr(ids), workspace.data_ptr(), workspace.numel())
    return values, ids


def t5_stack_distill_loss_and_grad(sc, tokens, targets, teacher_logits, teacher_ids, weights, temperature=1.0,
                                   soft_weight=1.0, grads=None, want_grads=True, accumulate=False, workspace=None, loss=None):
    """t5_stack_loss_and_grad against a teacher's top logits (float32) and ids (int32), both [batch, seq, top_k], as
    t5_stack_top_logits gives them.  Returns (loss tensor of one float32, grads or None)."""
    b, dev = sc.block, tokens.device
    cs = _stack_cfg_struct(sc)
    n_tok = b.batch * b.seq
    _check_tensor(tokens, torch.int32, n_tok, "tokens")
    _check_on(dev, targets, torch.int32, n_tok, "targets")
    opts = _DistillOpts(_i32(_teacher_entries(n_tok, teacher_logits, teacher_ids, dev)), float(temperature), float(soft_weight))
    ws = _stack_weights_struct(sc, weights)
    gs_ref = None
    if want_grads:
        if grads is None:
            grads = alloc_stack_grads(sc, weights)
        gs_ref = C.byref(_stack_grads_struct(sc, weights, grads))
    else:
        grads = None
    _check_devices(dev, weights, "weights")
    _check_devices(dev, grads, "grads")
    loss = _loss_buffer(loss, dev)
    workspace = _model_workspace(workspace, lib().t5_stack_distill_workspace_bytes(C.byref(cs), C.byref(opts)), dev)
    _call(lib().t5_stack_distill_loss_and_grad, "t5_stack_distill_loss_and_grad", dev, C.byref(cs), C.byref(opts),
          tokens.data_ptr(), targets.data_ptr(), teacher_logits.data_ptr(), teacher_ids.data_ptr(), C.byref(ws),
          loss.data_ptr(), gs_ref, int(bool(accumulate)), workspace.data_ptr(), workspace.numel())
    return loss, grads


def _encdec_cfg_struct(ec) -> _EncDecCfg:
    return _EncDecCfg(_cfg_struct(ec.enc_block), _cfg_struct(ec.dec_block), int(ec.n_enc_layers),
                      int(ec.n_dec_layers), int(ec.vocab), int(bool(ec.tied_logits)), int(bool(ec.remat)),
                      float(ec.z_loss))


def t5_encdec_workspace_bytes(ec) -> int:
    return int(lib().t5_encdec_workspace_bytes(C.byref(_encdec_cfg_struct(ec))))


_ENCDEC_FLAT = ("embedding", "enc_rel_table", "enc_final_scale", "dec_rel_table", "dec_final_scale")


def alloc_encdec_grads(ec, weights) -> dict:
    z = lambda t: torch.zeros(t.shape, dtype=torch.float32, device=t.device)
    g = {k: z(weights[k]) for k in _ENCDEC_FLAT}
    if not ec.tied_logits:
        g["logits_w"] = z(weights["logits_w"])
    names = _block_names(ec.enc_block, LAYER_WEIGHT_NAMES)
    g["enc_layers"] = [{n: z(lw[n]) for n in names} for lw in weights["enc_layers"]]
    g["dec_layers"] = [{n: z(lw[n]) for n in names + CROSS_WEIGHT_NAMES} for lw in weights["dec_layers"]]
    return g


def _encdec_weights_struct(ec, weights) -> _EncDecWeights:
    e, d = ec.enc_block, ec.dec_block
    dt = _torch_dtype(d)
    _check_tensor(weights["embedding"], dt, ec.vocab * d.d_model, "embedding")
    for nme, cfgb in (("enc_rel_table", e), ("dec_rel_table", d)):
        _check_tensor(weights[nme], dt, cfgb.num_buckets * cfgb.n_heads, nme)
    for nme in ("enc_final_scale", "dec_final_scale"):
        _check_tensor(weights[nme], dt, d.d_model, nme)
    if not ec.tied_logits:
        _check_tensor(weights["logits_w"], dt, ec.vocab * d.d_model, "logits_w")
    if len(weights["enc_layers"]) != ec.n_enc_layers or len(weights["dec_layers"]) != ec.n_dec_layers:
        raise ValueError("layer lists must hold n_enc_layers / n_dec_layers dicts")
    elw = (_Weights * ec.n_enc_layers)()
    for l, lw in enumerate(weights["enc_layers"]):
        elw[l] = _weights_struct(e, dict(lw, rel_table=weights["enc_rel_table"]))
    dlw = (_Weights * ec.n_dec_layers)()
    dxw = (_CrossWeights * ec.n_dec_layers)()
    for l, lw in enumerate(weights["dec_layers"]):
        dlw[l] = _weights_struct(d, dict(lw, rel_table=weights["dec_rel_table"]))
        dxw[l] = _cross_weights_struct(d, lw)
    p = lambda t: t.data_ptr()
    return _EncDecWeights(p(weights["embedding"]), p(weights["enc_rel_table"]), elw, p(weights["enc_final_scale"]),
                          p(weights["dec_rel_table"]), dlw, dxw, p(weights["dec_final_scale"]),
                          None if ec.tied_logits else p(weights["logits_w"]))


def _encdec_grads_struct(ec, weights, grads) -> _EncDecGrads:
    e, d = ec.enc_block, ec.dec_block
    p = lambda t: t.data_ptr()
    for nme in _ENCDEC_FLAT + (() if ec.tied_logits else ("logits_w",)):
        _check_tensor(grads[nme], torch.float32, weights[nme].numel(), "grad " + nme)
    elg = (_Grads * ec.n_enc_layers)()
    for l, gd in enumerate(grads["enc_layers"]):
        for nme in _block_names(e, LAYER_WEIGHT_NAMES):
            _check_tensor(gd[nme], torch.float32, weights["enc_layers"][l][nme].numel(), f"grad enc {l} {nme}")
        elg[l] = _Grads(*[(_addr(gd, nme) if nme != "rel_table" else p(grads["enc_rel_table"])) for nme in WEIGHT_NAMES])
    dlg = (_Grads * ec.n_dec_layers)()
    dxg = (_CrossGrads * ec.n_dec_layers)()
    for l, gd in enumerate(grads["dec_layers"]):
        for nme in _block_names(d, LAYER_WEIGHT_NAMES) + CROSS_WEIGHT_NAMES:
            _check_tensor(gd[nme], torch.float32, weights["dec_layers"][l][nme].numel(), f"grad dec {l} {nme}")
        dlg[l] = _Grads(*[(_addr(gd, nme) if nme != "rel_table" else p(grads["dec_rel_table"])) for nme in WEIGHT_NAMES])
        dxg[l] = _CrossGrads(*[p(gd[nme]) for nme in CROSS_WEIGHT_NAMES])
    return _EncDecGrads(p(grads["embedding"]), p(grads["enc_rel_table"]), elg, p(grads["enc_final_scale"]),
                        p(grads["dec_rel_table"]), dlg, dxg, p(grads["dec_final_scale"]),
                        None if ec.tied_logits else p(grads["logits_w"]))


def t5_encdec_loss_and_grad(ec, enc_tokens, dec_tokens, targets, weights, grads=None, want_grads=True,
                            accumulate=False, workspace=None, loss=None):
    """Loss (and gradients) of the encoder-decoder model.  weights: {"embedding", "enc_rel_table",
    "enc_layers": [block dicts without rel_table], "enc_final_scale", "dec_rel_table", "dec_layers": [block +
    cross-attention dicts without rel_table], "dec_final_scale", "logits_w" (untied)}.
    Returns (loss tensor of one float32, grads or None)."""
    e, d = ec.enc_block, ec.dec_block
    cs = _encdec_cfg_struct(ec)
    _check_tensor(enc_tokens, torch.int32, e.batch * e.seq, "enc_tokens")
    _check_tensor(dec_tokens, torch.int32, d.batch * d.seq, "dec_tokens")
    _check_tensor(targets, torch.int32, d.batch * d.seq, "targets")
    ws = _encdec_weights_struct(ec, weights)
    gs_ref = None
    if want_grads:
        if grads is None:
            grads = alloc_encdec_grads(ec, weights)
        gs_ref = C.byref(_encdec_grads_struct(ec, weights, grads))
    else:
        grads = None
    if loss is None:
        loss = torch.zeros(1, dtype=torch.float32, device=enc_tokens.device)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_encdec_workspace_bytes(C.byref(cs)), enc_tokens.device)
    rc = lib().t5_encdec_loss_and_grad(C.byref(cs), _ptr(enc_tokens), _ptr(dec_tokens), _ptr(targets), C.byref(ws),
                                       _ptr(loss), gs_ref, int(bool(accumulate)), _ptr(workspace), workspace.numel(),
                                       _stream())
    if rc:
        raise T5Error(rc, "t5_encdec_loss_and_grad")
    return loss, grads


def t5_encdec_top_logits(ec, enc_tokens, dec_tokens, weights, top_k, values=None, ids=None, workspace=None):
    """t5_stack_top_logits for the encoder-decoder model: the largest logits of every decoder position."""
    e, d, dev = ec.enc_block, ec.dec_block, dec_tokens.device
    cs = _encdec_cfg_struct(ec)
    _check_tensor(dec_tokens, torch.int32, d.batch * d.seq, "dec_tokens")
    _check_on(dev, enc_tokens, torch.int32, e.batch * e.seq, "enc_tokens")
    ws = _encdec_weights_struct(ec, weights)
    _check_devices(dev, weights, "weights")
    nbytes = lib().t5_encdec_top_logits_workspace_bytes(C.byref(cs), _i32(top_k))
    if nbytes:  # (0: the call below says what is wrong)
        values, ids = _top_outputs(d.batch, d.seq, top_k, dev, values, ids)
    workspace = _model_workspace(workspace, nbytes, dev)
    _call(lib().t5_encdec_top_logits, "t5_encdec_top_logits", dev, C.byref(cs), enc_tokens.data_ptr(),
          dec_tokens.data_ptr(), C.byref(ws), _i32(top_k), _ptr(values), _ptr(ids), workspace.data_ptr(), workspace.numel())
    return values, ids


def t5_encdec_distill_loss_and_grad(ec, enc_tokens, dec_tokens, targets, teacher_logits, teacher_ids, weights,
                                    temperature=1.0, soft_weight=1.0, grads=None, want_grads=True, accumulate=False,
                                    workspace=None, loss=None):
    """t5_encdec_loss_and_grad against a teacher's top logits and ids of the decoder positions, [batch, seq, top_k]."""
    e, d, dev = ec.enc_block, ec.dec_block, dec_tokens.device
    cs = _encdec_cfg_struct(ec)
    n_tok = d.batch * d.seq
    _check_tensor(dec_tokens, torch.int32, n_tok, "dec_tokens")
    _check_on(dev, enc_tokens, torch.int32, e.batch * e.seq, "enc_tokens")
    _check_on(dev, targets, torch.int32, n_tok, "targets")
    opts = _DistillOpts(_i32(_teacher_entries(n_tok, teacher_logits, teacher_ids, dev)), float(temperature), float(soft_weight))
    ws = _encdec_weights_struct(ec, weights)
    gs_ref = None
    if want_grads:
        if grads is None:
            grads = alloc_encdec_grads(ec, weights)
        gs_ref = C.byref(_encdec_grads_struct(ec, weights, grads))
    else:
        grads = None
    _check_devices(dev, weights, "weights")
    _check_devices(dev, grads, "grads")
    loss = _loss_buffer(loss, dev)
    workspace = _model_workspace(workspace, lib().t5_encdec_distill_workspace_bytes(C.byref(cs), C.byref(opts)), dev)
    _call(lib().t5_encdec_distill_loss_and_grad, "t5_encdec_distill_loss_and_grad", dev, C.byref(cs), C.byref(opts),
          enc_tokens.data_ptr(), dec_tokens.data_ptr(), targets.data_ptr(), teacher_logits.data_ptr(),
          teacher_ids.data_ptr(), C.byref(ws), loss.data_ptr(), gs_ref, int(bool(accumulate)), workspace.data_ptr(),
          workspace.numel())
    return loss, grads


def adafactor_workspace_bytes(rows: int, cols: int, factored: bool) -> int:
    return int(lib().adafactor_workspace_bytes(int(rows), int(cols), int(bool(factored))))


def adafactor_step(param, grad, *, step, lr, factored, v_row=None, v_col=None, v_full=None, decay_pow=0.8,
                   eps1=1e-30, eps2=1e-3, clip=1.0, scale_by_param=True, bf16_copy_out=None, workspace=None,
                   weight_decay=0.0):
    """In-place Adafactor update of a float32 tensor viewed as [rows, cols] (1-D tensors: rows = 1)."""
    rows, cols = (param.shape[0], param.numel() // param.shape[0]) if param.dim() >= 2 else (1, param.numel())
    _check_tensor(param, torch.float32, rows * cols, "param")
    _check_tensor(grad, torch.float32, rows * cols, "grad")
    if factored:
        _check_tensor(v_row, torch.float32, rows, "v_row")
        _check_tensor(v_col, torch.float32, cols, "v_col")
    else:
        _check_tensor(v_full, torch.float32, rows * cols, "v_full")
    if bf16_copy_out is not None:
        _check_tensor(bf16_copy_out, torch.bfloat16, rows * cols, "bf16_copy_out")
    if workspace is None:
        workspace = _byte_buffer(adafactor_workspace_bytes(rows, cols, factored), param.device)
    cfg = _AfCfg(lr, decay_pow, eps1, eps2, clip, int(bool(scale_by_param)), int(step), 0.0, float(weight_decay))
    rc = lib().adafactor_step(_ptr(param), _ptr(grad), _ptr(v_row), _ptr(v_col), _ptr(v_full), rows, cols,
                              int(bool(factored)), C.byref(cfg), _ptr(bf16_copy_out), _ptr(workspace),
                              workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "adafactor_step")
    return param


def adafactor_step_static(param, grad, *, step, lr, factored, v_row=None, v_col=None, v_full=None, decay_pow=0.8,
                          eps1=1e-30, eps2=1e-3, clip=1.0, scale_by_param=True, bf16_copy_out=None,
                          weight_decay=0.0):
    """adafactor_step through the entry point that allocates nothing: no workspace argument, the scratch is a
    fixed device array inside the library (tensors beyond its size are refused)."""
    rows, cols = (param.shape[0], param.numel() // param.shape[0]) if param.dim() >= 2 else (1, param.numel())
    _check_tensor(param, torch.float32, rows * cols, "param")
    _check_tensor(grad, torch.float32, rows * cols, "grad")
    if factored:
        _check_tensor(v_row, torch.float32, rows, "v_row")
        _check_tensor(v_col, torch.float32, cols, "v_col")
    else:
        _check_tensor(v_full, torch.float32, rows * cols, "v_full")
    if bf16_copy_out is not None:
        _check_tensor(bf16_copy_out, torch.bfloat16, rows * cols, "bf16_copy_out")
    cfg = _AfCfg(lr, decay_pow, eps1, eps2, clip, int(bool(scale_by_param)), int(step), 0.0, float(weight_decay))
    rc = lib().adafactor_step_static(_ptr(param), _ptr(grad), _ptr(v_row), _ptr(v_col), _ptr(v_full), rows, cols,
                                     int(bool(factored)), C.byref(cfg), _ptr(bf16_copy_out), _stream())
    if rc:
        raise T5Error(rc, "adafactor_step_static")
    return param


def _af_tensor_array(tensors):
    """tensors: list of dicts with param, grad, factored and v_row/v_col or v_full (+ bf16_copy_out)."""
    arr = (_AfTensor * len(tensors))()
    for i, t in enumerate(tensors):
        p = t["param"]
        rows, cols = (p.shape[0], p.numel() // p.shape[0]) if p.dim() >= 2 else (1, p.numel())
        fact = bool(t["factored"])
        _check_tensor(p, torch.float32, rows * cols, "param")
        _check_tensor(t["grad"], torch.float32, rows * cols, "grad")
        if fact:
            _check_tensor(t["v_row"], torch.float32, rows, "v_row")
            _check_tensor(t["v_col"], torch.float32, cols, "v_col")
        else:
            _check_tensor(t["v_full"], torch.float32, rows * cols, "v_full")
        lp = t.get("bf16_copy_out")
        if lp is not None:
            _check_tensor(lp, torch.bfloat16, rows * cols, "bf16_copy_out")
        mom = t.get("m")
        if mom is not None:
            _check_tensor(mom, torch.float32, rows * cols, "m")
        addr = lambda x: None if x is None else x.data_ptr()
        arr[i] = _AfTensor(addr(p), addr(t["grad"]), addr(t.get("v_row")) if fact else None,
                           addr(t.get("v_col")) if fact else None, None if fact else addr(t.get("v_full")),
                           rows, cols, int(fact), addr(lp), addr(mom))
    return arr


def adafactor_multi_workspace_bytes(tensors) -> int:
    arr = _af_tensor_array(tensors)
    return int(lib().adafactor_multi_workspace_bytes(arr, len(tensors)))


def adafactor_step_multi(tensors, *, step, lr, decay_pow=0.8, eps1=1e-30, eps2=1e-3, clip=1.0,
                         scale_by_param=True, workspace=None, beta1=0.0, weight_decay=0.0):
    """In-place Adafactor update of several float32 tensors in one sequence of launches.  beta1 > 0 adds
    momentum (each tensor dict then holds its float32 buffer "m"); weight_decay is decoupled."""
    arr = _af_tensor_array(tensors)
    if workspace is None:
        workspace = _byte_buffer(max(int(lib().adafactor_multi_workspace_bytes(arr, len(tensors))), 256),
                                 tensors[0]["param"].device)
    cfg = _AfCfg(lr, decay_pow, eps1, eps2, clip, int(bool(scale_by_param)), int(step), float(beta1),
                 float(weight_decay))
    rc = lib().adafactor_step_multi(arr, len(tensors), C.byref(cfg), _ptr(workspace), workspace.numel(), _stream())
    if rc:
        raise T5Error(rc, "adafactor_step_multi")


def _elem_type(t, name):
    """T5_F32 or T5_BF16 of a tensor that may have either type."""
    if t.dtype == torch.bfloat16:
        return T5_BF16
    if t.dtype != torch.float32:
        raise ValueError(f"{name}: need float32 or bfloat16, got {t.dtype}")
    return T5_F32


def _i32(v):
    """A whole number for an int32 field: what does not fit is passed as the largest, which every call refuses."""
    v = operator.index(v)
    return v if -2 ** 31 <= v < 2 ** 31 else 2 ** 31 - 1


def _check_on(device, t, dtype, numel, name):
    _check_tensor(t, dtype, numel, name)
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, other arguments on {device}")


def _check_rows(t, name):
    """Rows of a matrix whose elements are contiguous; (rows, columns, row stride)."""
    if not _strided(t):
        raise ValueError(f"{name}: need a strided tensor, got layout {t.layout}{', nested' if t.is_nested else ''}")
    if t.is_cuda and t.dim() == 2 and t.is_contiguous():
        return t.shape[0], t.shape[1], t.shape[1]
    if not t.is_cuda or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name}: need a 2-D cuda tensor with contiguous rows that do not overlap, got {tuple(t.shape)} "
                         f"with strides {t.stride()} on {t.device}")
    return t.shape[0], t.shape[1], t.stride(0) if t.shape[0] > 1 else t.shape[1]


# (torch.cuda.current_stream() builds an object: 2.8 of the 10 us that a small call takes)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)  # (the tensors are there: CUDA is set up)


def _call(fn, what, device, *args):
    """One library call on the current stream of the tensors' device."""
    if device.index != _current_device():
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(device.index))
    else:
        rc = fn(*args, _raw_stream(device.index))
    if rc:
        raise T5Error(rc, what)


def t5_embed_fwd(tokens, table, scale=1.0, x=None):
    """x[..., :] = scale * table[tokens[...], :]; tokens int32 of any shape, table [vocab, d_model].  Returns x."""
    ty = _elem_type(table, "table")
    vocab, d = table.shape
    _check_tensor(table, table.dtype, vocab * d, "table")
    n = tokens.numel()
    _check_on(table.device, tokens, torch.int32, n, "tokens")
    if x is None:
        x = torch.empty(*tokens.shape, d, dtype=table.dtype, device=table.device)
    else:
        _check_on(table.device, x, table.dtype, n * d, "x")
    cfg = _EmbedCfg(n, _i32(vocab), _i32(d), ty, float(scale))
    _call(lib().t5_embed_fwd, "t5_embed_fwd", table.device, C.byref(cfg), tokens.data_ptr(), table.data_ptr(), x.data_ptr())
    return x


def t5_embed_bwd(tokens, dx, vocab, scale=1.0, dtable=None, accumulate=False, workspace=None):
    """dtable[v, :] (+)= scale * sum of dx[t, :] over tokens[t] == v, float32 [vocab, d_model].  Returns dtable."""
    ty = _elem_type(dx, "dx")
    n, d = tokens.numel(), dx.shape[-1]
    _check_tensor(dx, dx.dtype, n * d, "dx")
    _check_on(dx.device, tokens, torch.int32, n, "tokens")
    if dtable is None:  # (a size that the call refuses is not worth an allocation)
        rows = vocab if 0 < vocab <= 1 << 22 else 0
        dtable = (torch.zeros if accumulate else torch.empty)(rows, d, dtype=torch.float32, device=dx.device)
    else:
        _check_on(dx.device, dtable, torch.float32, vocab * d, "dtable")
    cfg = _EmbedCfg(n, _i32(vocab), _i32(d), ty, float(scale))
    if workspace is None:
        workspace = _byte_buffer(lib().t5_embed_bwd_workspace_bytes(C.byref(cfg)), dx.device)
    else:
        _check_on(dx.device, workspace, torch.uint8, workspace.numel(), "workspace")
    _call(lib().t5_embed_bwd, "t5_embed_bwd", dx.device, C.byref(cfg), tokens.data_ptr(), dx.data_ptr(), dtable.data_ptr(),
          int(bool(accumulate)), workspace.data_ptr(), workspace.numel())
    return dtable


def t5_top_logits(logits, top_k, values=None, ids=None):
    """(values float32, ids int32), both [rows, top_k]: the largest logits of each row, descending, equal ones by ascending
    id.  logits [rows, vocab] may be a view of rows with a longer stride."""
    ty = _elem_type(logits, "logits")
    rows, vocab, ld = _check_rows(logits, "logits")
    dev = logits.device
    k = top_k if 0 < top_k <= 256 else 0  # (a number that the call refuses is not worth an allocation)
    if values is None:
        values = torch.empty(rows, k, dtype=torch.float32, device=dev)
    else:
        _check_on(dev, values, torch.float32, rows * top_k, "values")
    if ids is None:
        ids = torch.empty(rows, k, dtype=torch.int32, device=dev)
    else:
        _check_on(dev, ids, torch.int32, rows * top_k, "ids")
    cfg = _TopCfg(rows, ld, _i32(vocab), _i32(top_k), ty)
    _call(lib().t5_top_logits, "t5_top_logits", dev, C.byref(cfg), logits.data_ptr(), values.data_ptr(), ids.data_ptr())
    return values, ids


def t5_distill_loss_and_grad(logits, targets, teacher_logits, teacher_ids, temperature=1.0, soft_weight=1.0, z_loss=0.0,
                             want_grads=True, loss=None, row_loss=None, dlogits=None, workspace=None):
    """Loss of logits [rows, vocab] (rows may have a longer stride) against a teacher's top logits and ids [rows, top_k] and
    int32 targets [rows] (None: every row counts, soft targets alone).  dlogits may be the logits themselves, or have a row
    stride of its own; by default it is a new tensor whose rows follow each other, or are less than 16 bytes apart where those
    of the logits are no multiple of 16 bytes apart.  Returns (loss of one float32, row losses float32, dlogits or None)."""
    ty = _elem_type(logits, "logits")
    rows, vocab, ld = _check_rows(logits, "logits")
    dev = logits.device
    if teacher_ids.dim() != 2:
        raise ValueError(f"teacher_ids: need [rows, top_k], got {tuple(teacher_ids.shape)}")
    k = teacher_ids.shape[1]
    _check_on(dev, teacher_ids, torch.int32, rows * k, "teacher_ids")
    _check_on(dev, teacher_logits, torch.float32, rows * k, "teacher_logits")
    if targets is not None:
        _check_on(dev, targets, torch.int32, rows, "targets")
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=dev)
    else:
        _check_on(dev, loss, torch.float32, 1, "loss")
    if row_loss is None:
        row_loss = torch.empty(rows, dtype=torch.float32, device=dev)
    else:
        _check_on(dev, row_loss, torch.float32, rows, "row_loss")
    out_ld = ld
    if not want_grads:
        dlogits = None
    elif dlogits is None:
        # (not the logits' stride, which may be a sequence of rows long; pieces of 16 bytes lie in both rows alike)
        out_ld = vocab + (ld - vocab) % (16 // logits.element_size())
        dlogits = torch.empty(rows, out_ld, dtype=logits.dtype, device=dev)
        if out_ld != vocab:
            dlogits = dlogits[:, :vocab]
    else:
        *shape, out_ld = _check_rows(dlogits, "dlogits")
        if dlogits.device != dev or dlogits.dtype != logits.dtype or shape != [rows, vocab]:
            raise ValueError(f"dlogits: need type and shape of logits, got {dlogits.dtype} {tuple(dlogits.shape)} on {dlogits.device}")
    cfg = _DistillCfg(rows, ld, _i32(vocab), _i32(k), ty, float(temperature), float(soft_weight), float(z_loss), out_ld)
    if workspace is None:
        workspace = _byte_buffer(lib().t5_distill_workspace_bytes(C.byref(cfg)), dev)
    else:
        _check_on(dev, workspace, torch.uint8, workspace.numel(), "workspace")
    addr = lambda t: None if t is None else t.data_ptr()
    _call(lib().t5_distill_loss_and_grad, "t5_distill_loss_and_grad", dev, C.byref(cfg), logits.data_ptr(), addr(targets),
          teacher_logits.data_ptr(), teacher_ids.data_ptr(), loss.data_ptr(), row_loss.data_ptr(), addr(dlogits),
          workspace.data_ptr(), workspace.numel())
    return loss, row_loss, dlogits


_LISTS = None


def _lists():
    """The native readers of tensors (csrc/torch_lists.cpp; built with the library) and the entry points that they call.  Raises if they are not there."""
    global _LISTS
    if _LISTS is None:
        try:
            from . import _torch_lists
        except ImportError:
            from . import build as _build
            _build.build_lists()
            from . import _torch_lists
        L = lib()
        addr = lambda fn: C.cast(fn, C.c_void_p).value
        _LISTS = (_torch_lists.quantize_fp8, addr(L.t5_quantize_fp8), _torch_lists.gemm_fp8, addr(L.t5_gemm_fp8),
                  addr(L.t5_gemm_fp8_workspace_bytes), _torch_lists.adamw_entries)
    return _LISTS


_FP8 = {torch.float8_e4m3fn: T5_E4M3, torch.float8_e5m2: T5_E5M2}
_FP8_NAMES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_E8M0 = torch.float8_e8m0fnu


def _fp8_pair(rows, cols, block_rows, q_dtype, device):
    """Codes [rows, cols] and scales of a new quantised matrix, rows as far apart as t5_quantize_fp8 writes them."""
    blocks = -(-cols // 128)
    q = torch.empty(rows, -(-cols // 16) * 16, dtype=q_dtype, device=device)
    s = torch.empty(-(-rows // block_rows), -(-blocks // 4) * 4, dtype=_E8M0, device=device)
    return q if q.shape[1] == cols else q[:, :cols], s if s.shape[1] == blocks else s[:, :blocks]


def _check_fp8_pair(q, scale, rows, cols, block_rows, q_dtype, device, name):
    blocks = -(-cols // 128)
    for t, dt, shape, ld, what in ((q, q_dtype, (rows, cols), -(-cols // 16) * 16, name),
                                   (scale, _E8M0, (-(-rows // block_rows), blocks), -(-blocks // 4) * 4, name + "'s scale")):
        if t is None or t.device != device or t.dtype != dt or tuple(t.shape) != shape or \
                (shape[1] > 1 and t.stride(1) != 1) or (shape[0] > 1 and t.stride(0) != ld):
            raise ValueError(f"{what}: need {dt} {shape} on {device} with rows {ld} apart, got " +
                             ("nothing" if t is None else f"{t.dtype} {tuple(t.shape)}, strides {t.stride()} on {t.device}"))
        room = t.untyped_storage().nbytes() - t.storage_offset()  # (rows are written in whole pieces, the last one too)
        if shape[0] > 0 and room < shape[0] * ld:
            raise ValueError(f"{what}: its last row has no room for the end of its last piece")


def t5_quantize_fp8(x, q_dtype="e4m3", block_rows=1, rows=True, transposed=False, q=None, scale=None, qt=None, scale_t=None):
    """Quantised matrix of x [rows, cols] (float32 or bfloat16; rows may have a longer stride), and with transposed=True the
    transposed one: (q, scale, qt, scale_t), the pairs that are not asked for None.  q_dtype: "e4m3" or "e5m2" (or torch's
    type).  A scale (float8_e8m0fnu) serves 128 columns of one row, or of 128 rows with block_rows=128; with block_rows=1 the
    transposed matrix has scales of its own, for 128 rows of one column of x.  Outputs of the caller's own have rows as far
    apart as the ones made here: codes a multiple of 16, scales a multiple of 4."""
    dt = _FP8_NAMES.get(q_dtype, q_dtype)
    dev = x.device
    if q is None and scale is None and qt is None and scale_t is None and dev.type == "cuda" and dev.index == _current_device() and dt in _FP8:
        lists = _LISTS or _lists()  # (the ordinary call; what it does not take is checked below)
        out = lists[0](lists[1], x, 1 if _FP8[dt] == T5_E5M2 else 0, block_rows, rows, transposed, _raw_stream(dev.index), dev.index)
        if type(out) is tuple:
            return out
        if out:
            raise T5Error(out, "t5_quantize_fp8")
    ty = _elem_type(x, "x")
    n, cols, ld = _check_rows(x, "x")
    if dt not in _FP8:
        raise ValueError(f"q_dtype: need e4m3 or e5m2, got {q_dtype}")
    block_rows = operator.index(block_rows)
    br = block_rows if block_rows in (1, 128) else 1
    if not rows:
        q = scale = None
    elif q is None and scale is None:
        q, scale = _fp8_pair(n, cols, br, dt, dev)
    else:
        _check_fp8_pair(q, scale, n, cols, br, dt, dev, "q")
    if not transposed:
        qt = scale_t = None
    elif qt is None and scale_t is None:
        qt, scale_t = _fp8_pair(cols, n, br, dt, dev)
    else:
        _check_fp8_pair(qt, scale_t, cols, n, br, dt, dev, "qt")
    addr = lambda t: None if t is None else t.data_ptr()
    _call(lib().t5_quantize_fp8, "t5_quantize_fp8", dev, C.byref(_QuantizeCfg(n, cols, ld, ty, _FP8[dt], _i32(block_rows))),
          x.data_ptr(), addr(q), addr(scale), addr(qt), addr(scale_t))
    return q, scale, qt, scale_t


def _fp8_operand(q, scale, name):
    """(rows, K, bytes between rows, type, rows of a block, bytes between rows of scales) of a quantised matrix."""
    ty = _FP8.get(q.dtype)
    if ty is None or scale.dtype != _E8M0:
        raise ValueError(f"{name}: need float8_e4m3fn or float8_e5m2 codes with float8_e8m0fnu scales, got {q.dtype}, {scale.dtype}")
    n, k, ld = _check_rows(q, name)
    sn, sk, sld = _check_rows(scale, name)
    if sk != (k + 127) // 128 or sn != n and sn != (n + 127) // 128:
        raise ValueError(f"{name}: codes {tuple(q.shape)} have scales [{n} or {-(-n // 128)}, {-(-k // 128)}], got {tuple(scale.shape)}")
    # rows are read in whole pieces: the end of the last one has to be there; one row may be of any length
    if k % 16:
        ld = _last_piece(q, n, k, ld, 16, name)
    if sk % 4:
        sld = _last_piece(scale, sn, sk, sld, 4, name + "'s scale")
    return n, k, ld, ty, 1 if sn == n else 128, sld


def _last_piece(t, rows, cols, ld, step, name):
    whole = -(-cols // step) * step
    if rows > 0 and t.untyped_storage().nbytes() - t.storage_offset() < (rows - 1) * ld + whole:
        raise ValueError(f"{name}: its last row ends inside a piece of {step} bytes, and its memory with it")
    return whole if rows <= 1 else ld


def t5_gemm_fp8(a, a_scale, b, b_scale, out=None, out_dtype=torch.bfloat16, accumulate=False, workspace=None):
    """C[m, n] = sum over k of A[m, k] B[n, k] of two quantised matrices as t5_quantize_fp8 makes them (one scale for each
    128 columns of a row, or of 128 rows: by the scales' shape).  out: [M, N] float32 or bfloat16, rows may have a longer
    stride; accumulate adds to it (float32).  Returns out."""
    dev = a.device
    if workspace is None and dev.type == "cuda" and dev.index == _current_device() and out_dtype in (torch.bfloat16, torch.float32):
        lists = _LISTS or _lists()  # (the ordinary call; what it does not take is checked below)
        made = lists[2](lists[3], lists[4], a, a_scale, b, b_scale, out, out_dtype is torch.float32, accumulate, _raw_stream(dev.index), dev.index)
        if isinstance(made, torch.Tensor):
            return made
        if made:
            raise T5Error(made, "t5_gemm_fp8")
    m, k, lda, ta, bra, lsa = _fp8_operand(a, a_scale, "a")
    n, kb, ldb, tb, brb, lsb = _fp8_operand(b, b_scale, "b")
    if k != kb:
        raise ValueError(f"a has {k} columns, b {kb}")
    if b.device != dev or a_scale.device != dev or b_scale.device != dev:
        raise ValueError(f"a on {dev}, its scale on {a_scale.device}, b on {b.device}, its scale on {b_scale.device}")
    if out is None:
        if accumulate:
            raise ValueError("accumulate: there is no out to add to")
        out = torch.empty(m, n, dtype=out_dtype, device=dev)
        ldc = n
    else:
        rows, cols, ldc = _check_rows(out, "out")
        if (rows, cols) != (m, n) or out.device != dev:
            raise ValueError(f"out: need [{m}, {n}] on {dev}, got {tuple(out.shape)} on {out.device}")
    cfg = C.byref(_GemmFp8Cfg(_i32(m), _i32(n), _i32(k), lda, ldb, ldc, lsa, lsb, ta, tb, bra, brb, _elem_type(out, "out"),
                              1 if accumulate else 0))
    L = lib()
    ws, nbytes = None, L.t5_gemm_fp8_workspace_bytes(cfg)
    if workspace is not None:
        _check_on(dev, workspace, torch.uint8, workspace.numel(), "workspace")
        ws, nbytes = workspace.data_ptr(), workspace.numel()
    elif nbytes:
        workspace = _byte_buffer(nbytes, dev)
        ws = workspace.data_ptr()
    _call(L.t5_gemm_fp8, "t5_gemm_fp8", dev, cfg, a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(),
          out.data_ptr(), ws, nbytes)
    return out


FP8_PATH_TILE64, FP8_PATH_TILE128, FP8_PATH_TILE256, FP8_PATH_SHARED, FP8_PATH_ROWS = 1, 2, 4, 8, 16
FP8_PATH_ROWS_A32, FP8_PATH_ROWS_A64, FP8_PATH_ROWS_B32 = 32, 64, 128


def t5_gemm_fp8_kernel_path(m, n, k, out_dtype=torch.bfloat16) -> int:
    """Bit mask of the kernel that a product of [m, k] and [n, k] runs on (host-side query; -1: invalid sizes or type)."""
    ld, lds, ty = -(-k // 16) * 16, -(-k // 512) * 4, {torch.bfloat16: T5_BF16, torch.float32: T5_F32}.get(out_dtype, -1)
    return int(lib().t5_gemm_fp8_kernel_path(C.byref(_GemmFp8Cfg(_i32(m), _i32(n), _i32(k), ld, ld, n, lds, lds, T5_E4M3, T5_E4M3, 1, 1, ty, 0))))


def _adam_check(t, index):
    """Says what is wrong with an entry of adamw_step_multi's list."""
    device = torch.device("cuda", index)
    n = t["param"].numel()
    state = t["m"].dtype if t["m"].dtype == torch.float32 else torch.float8_e4m3fn
    _elem_type(t["grad"], "grad")
    for name, dt, size in (("param", torch.float32, n), ("grad", t["grad"].dtype, n), ("m", state, n), ("v", state, n)):
        _check_on(device, t[name], dt, size, name)
    if state != torch.float32:
        _check_on(device, t["m_scale"], _E8M0, -(-n // 128), "m_scale")
        _check_on(device, t["v_scale"], _E8M0, -(-n // 128), "v_scale")
    if t.get("bf16_copy_out") is not None:
        _check_on(device, t["bf16_copy_out"], torch.bfloat16, n, "bf16_copy_out")
    float(t.get("weight_decay", 0.0))


def adamw_step_multi(tensors, *, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, grad_scale=None):
    """In-place AdamW update of several float32 tensors in one launch (of 40 tensors).  tensors: list of dicts with param,
    grad (float32 or bfloat16), m, v and optionally weight_decay and bf16_copy_out.  States in 32 bits: m and v float32.  In
    8 bits: m and v float8_e4m3fn, codes of m and of sqrt(v), with m_scale and v_scale float8_e8m0fnu, one for each 128
    consecutive elements; zeros throughout before the first step (t.zero_() of a uint8 view).  seed: of their random rounding;
    grad_scale: a float32 tensor of one element that multiplies every gradient, or None."""
    tensors = list(tensors)
    if not tensors or not 0 < operator.index(step) < 2 ** 31:
        raise T5Error(2, "adamw_step_multi")
    dev = tensors[0]["param"].device
    if dev.type != "cuda":
        raise ValueError(f"param: on {dev}")
    arr = bytearray(C.sizeof(_AdamTensor) * len(tensors))
    good = (_LISTS or _lists())[5](tensors, dev.index, arr)
    if good != len(tensors):
        _adam_check(tensors[good], dev.index)
        raise ValueError(f"adamw_step_multi: entry {good} is no dict of tensors")
    if grad_scale is not None:
        _check_on(dev, grad_scale, torch.float32, 1, "grad_scale")
        grad_scale = grad_scale.data_ptr()
    seed = operator.index(seed)
    cfg = _AdamCfg(float(lr), float(beta1), float(beta2), float(eps), operator.index(step), seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF,
                   grad_scale)
    _call(lib().adamw_step_multi, "adamw_step_multi", dev, (_AdamTensor * len(tensors)).from_buffer(arr), len(tensors), C.byref(cfg))


def t5_gemm_bf16(a: torch.Tensor, b: torch.Tensor, a_kc: bool, b_kc: bool, out: torch.Tensor | None = None):
    """C[m,n] = sum_k A(m,k) B(n,k) in float32.  a: [M,K] if a_kc else [K,M]; b: [N,K] if b_kc else [K,N]."""
    for t, nme in ((a, "a"), (b, "b")):
        _check_tensor(t, torch.bfloat16, t.numel(), nme)
    M, K = (a.shape[0], a.shape[1]) if a_kc else (a.shape[1], a.shape[0])
    N = b.shape[0] if b_kc else b.shape[1]
    if out is None:
        out = torch.empty(M, N, dtype=torch.float32, device=a.device)
    rc = lib().t5_gemm_bf16(_ptr(a), _ptr(b), _ptr(out), M, N, K, a.shape[1], b.shape[1], N, int(a_kc), int(b_kc),
                            _stream())
    if rc:
        raise T5Error(rc, "t5_gemm_bf16")
    return out


def t5_wgrad_overlap_enable(enable: bool) -> None:
    """Run the weight-gradient GEMMs of every backward pass on a second stream owned by the library."""
    rc = lib().t5_wgrad_overlap_enable(int(bool(enable)))
    if rc:
        raise T5Error(rc, "t5_wgrad_overlap_enable")


def t5_step_timing_enable(enable: bool) -> None:
    lib().t5_step_timing_enable(int(bool(enable)))


def t5_mfma_peak_probe(workgroups: int, iters: int, random_operands: bool, sink: torch.Tensor) -> float:
    """Launches the register-only MFMA loop; returns the FLOPs it performs (the caller times it)."""
    _check_tensor(sink, torch.float32, 256, "sink")
    rc = lib().t5_mfma_peak_probe(int(workgroups), int(iters), int(bool(random_operands)), _ptr(sink), _stream())
    if rc:
        raise T5Error(rc, "t5_mfma_peak_probe")
    return float(workgroups) * 4 * iters * 32 * 2.0 * 32 * 32 * 16


def t5_step_timing_read(cap: int = 64) -> dict:
    """{step name: (total ms, launches)} since timing was enabled."""
    names = (C.c_char_p * cap)()
    ms = (C.c_float * cap)()
    calls = (C.c_int * cap)()
    n = lib().t5_step_timing_read(names, ms, calls, cap)
    return {names[i].decode(): (float(ms[i]), int(calls[i])) for i in range(n)}
