"""MI355X (gfx950) RoI differentiable N:M mask sampler.

Thin ctypes binding of ``libroi.so`` (declared in ``include/roi.h``): argument
marshalling only.  Every step of the sampler runs in the HIP kernels; torch is
used for device memory and the current stream.  If the library has not been
built, every call raises -- there is no other implementation behind it.
"""
from __future__ import annotations

import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libroi.so")

ROI_OK = 0
ROI_E_INVAL = -1
ROI_E_UNSUPPORTED = -2
ROI_E_HIP = -3

SUPPORTED_M = (4, 8, 16, 32)


class RoiError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{detail} (status {status})")
        self.status = status


_lib = None


class FwdTensor(ctypes.Structure):
    """roi_fwd_tensor (include/roi.h)."""
    _fields_ = [("W", ctypes.c_void_p), ("logits", ctypes.c_void_p),
                ("W_masked", ctypes.c_void_p), ("soft_mask", ctypes.c_void_p),
                ("sel_idx", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("elem_offset", ctypes.c_uint64)]


class AdamWParams(ctypes.Structure):
    """roi_adamw_params (include/roi.h)."""
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("t", ctypes.c_int64)]


class StepParams(ctypes.Structure):
    """roi_step_params (include/roi.h)."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("t", ctypes.c_int64)]


class AdamWTensor(ctypes.Structure):
    """roi_adamw_tensor (include/roi.h)."""
    _fields_ = [("grad_W_masked", ctypes.c_void_p), ("W", ctypes.c_void_p),
                ("logits", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("grad_logits", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("elem_offset", ctypes.c_uint64)]


class BwdTensor(ctypes.Structure):
    """roi_bwd_tensor (include/roi.h)."""
    _fields_ = [("grad_W_masked", ctypes.c_void_p), ("W", ctypes.c_void_p),
                ("logits", ctypes.c_void_p), ("grad_logits", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("elem_offset", ctypes.c_uint64)]

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_u64 = ctypes.c_uint64
_int = ctypes.c_int
_f32 = ctypes.c_float


def lib() -> ctypes.CDLL:
    """The loaded libroi.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2608_23048_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.roi_mask_fwd.argtypes = [_vp, _vp, _i64, _i64, _int, _int, _f32, _f32, _u64, _u64, _u64,
                                   _vp, _vp, _vp, _vp]
        L.roi_mask_fwd.restype = _int
        L.roi_mask_fwd_soft.argtypes = L.roi_mask_fwd.argtypes
        L.roi_mask_fwd_soft.restype = _int
        L.roi_mask_bwd.argtypes = [_vp, _vp, _vp, _i64, _i64, _int, _int, _f32, _f32, _u64, _u64,
                                   _u64, _vp, _vp]
        L.roi_mask_bwd.restype = _int
        grouped = [_vp, _int, _int, _int, _f32, _f32, _u64, _u64, _vp]
        for name in ("roi_mask_fwd_grouped", "roi_mask_fwd_soft_grouped", "roi_mask_bwd_grouped"):
            getattr(L, name).argtypes = grouped
            getattr(L, name).restype = _int
        L.roi_mask_bwd_adamw.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _int, _int,
                                         _f32, _f32, _u64, _u64, _u64, _vp, _vp]
        L.roi_mask_bwd_adamw.restype = _int
        L.roi_mask_bwd_adamw_grouped.argtypes = [_vp, _int, _int, _int, _f32, _f32, _u64, _u64,
                                                 _vp, _vp]
        L.roi_mask_bwd_adamw_grouped.restype = _int
        L.roi_mask_export.argtypes = [_vp, _vp, _i64, _i64, _int, _int, _vp, _vp, _vp, _vp, _vp]
        L.roi_mask_export.restype = _int
        L.roi_cat_num_candidates.argtypes = [_int, _int]
        L.roi_cat_num_candidates.restype = _int
        L.roi_cat_mask_fwd.argtypes = [_vp, _vp, _i64, _i64, _int, _int, _f32, _f32, _u64, _u64,
                                       _u64, _vp, _vp, _vp, _vp]
        L.roi_cat_mask_fwd.restype = _int
        L.roi_cat_mask_bwd.argtypes = [_vp, _vp, _vp, _i64, _i64, _int, _int, _f32, _f32, _u64,
                                       _u64, _u64, _vp, _vp]
        L.roi_cat_mask_bwd.restype = _int
        L.roi_gumbel_noise.argtypes = [_u64, _u64, _u64, _i64, _vp, _vp, _vp]
        L.roi_gumbel_noise.restype = _int
        L.roi_gumbel_from_words.argtypes = [_vp, _i64, _vp, _vp]
        L.roi_gumbel_from_words.restype = _int
        L.roi_fast_noise_from_words.argtypes = [_vp, _i64, _vp, _vp]
        L.roi_fast_noise_from_words.restype = _int
        L.roi_stream_copy.argtypes = [_vp, _vp, _i64, _vp]
        L.roi_stream_copy.restype = _int
        L.roi_quantize_rows.argtypes = [_vp, _int, _i64, _i64, _vp, _vp, _vp]
        L.roi_quantize_rows.restype = _int
        L.roi_dequantize_rows.argtypes = [_vp, _vp, _i64, _i64, _vp, _int, _vp]
        L.roi_dequantize_rows.restype = _int
        L.roi_linear_i8_workspace.argtypes = [_i64, _i64, _i64, _int]
        L.roi_linear_i8_workspace.restype = _i64
        L.roi_linear_i8.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _int,
                                    _vp, _i64, _vp]
        L.roi_linear_i8.restype = _int
        for name in ("roi_linear_i8_grad_weight", "roi_linear_i8_grad_input"):
            getattr(L, name + "_workspace").argtypes = [_i64, _i64, _i64]
            getattr(L, name + "_workspace").restype = _i64
            getattr(L, name).argtypes = [_vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp]
            getattr(L, name).restype = _int
        L.roi_block_scales.argtypes = [_i64]
        L.roi_block_scales.restype = _i64
        L.roi_quantize_blocks.argtypes = [_vp, _int, _i64, _i64, _int, _int, _vp, _i64, _vp, _vp,
                                          _i64, _vp, _vp]
        L.roi_quantize_blocks.restype = _int
        L.roi_dequantize_blocks.argtypes = [_vp, _i64, _vp, _i64, _i64, _int, _int, _vp, _int, _vp]
        L.roi_dequantize_blocks.restype = _int
        L.roi_linear_f8_workspace.argtypes = [_i64, _i64, _i64]
        L.roi_linear_f8_workspace.restype = _i64
        L.roi_linear_f8.argtypes = [_vp, _i64, _vp, _int, _vp, _i64, _vp, _int, _vp, _i64, _i64,
                                    _i64, _vp, _vp, _i64, _vp]
        L.roi_linear_f8.restype = _int
        L.roi_adamw_grouped.argtypes = [_vp, _int, _int, _int, _u64, _u64, _vp, _vp]
        L.roi_adamw_grouped.restype = _int
        L.roi_anneal.argtypes = [_f32, _f32, _i64, _i64]
        L.roi_anneal.restype = _f32
        L.roi_status_string.argtypes = [_int]
        L.roi_status_string.restype = ctypes.c_char_p
        L.roi_last_error.argtypes = []
        L.roi_last_error.restype = ctypes.c_char_p
        L.roi_abi_version.argtypes = []
        L.roi_abi_version.restype = _int
        _lib = L
    return _lib


def _raise_on(status: int):
    if status != ROI_OK:
        raise RoiError(status, lib().roi_last_error().decode() or
                       lib().roi_status_string(status).decode())


# torch, once a call has needed it (the import statement in every call, and
# torch.cuda.current_stream's Stream object, cost more than the arguments'
# marshalling: a call on a small tensor took 7.6 us of host time with them, of
# which 4.4 us are the library's launch, and takes 5.6 us without).
_torch = None
_raw_stream = None


def _load_torch():
    global _torch, _raw_stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _raw_stream = raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch
    return torch


def _stream(t) -> int:
    """The handle of the current stream of t's device."""
    if _torch is None:
        _load_torch()
    index = t.get_device()
    if index < 0:
        raise ValueError(f"expected a device tensor, got one on {t.device}")
    return _raw_stream(index)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _shape2d(t) -> tuple[int, int]:
    shape = t.shape
    if len(shape) == 2:
        return shape[0], shape[1]
    return 1, t.numel()


def _check_tensor(t, dtype, name, like=None):
    torch = _torch
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous()
            and (like is None or t.shape == like.shape)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(like.shape)}")


# --------------------------------------------------------------------------- tensor API
def mask_fwd(W, logits, n: int, m: int, tau: float = 1.0, lam: float = 1.0, seed: int = 0,
             step: int = 0, elem_offset: int = 0, want_soft: bool = False, want_idx: bool = True,
             out: dict | None = None, soft_forward: bool = False):
    """Forward sample.  W: bf16 [rows, cols] (or 1-D), logits: fp32 same shape.

    Returns (W_masked bf16, soft_mask fp32 or None, sel_idx uint8 [groups, n] or
    None).  ``out`` may hold preallocated "W_masked", "soft_mask", "sel_idx".
    soft_forward=False: straight-through forward, W_masked = W (.) hard mask;
    soft_forward=True: pure soft forward, W_masked = bf16(W (.) S).
    """
    torch = _torch or _load_torch()
    _check_tensor(W, torch.bfloat16, "W")
    _check_tensor(logits, torch.float32, "logits", like=W)
    rows, cols = _shape2d(W)
    out = out or {}
    Wm = out.get("W_masked")
    if Wm is None:
        Wm = torch.empty_like(W)
    S = out.get("soft_mask") if want_soft else None
    if want_soft and S is None:
        S = torch.empty_like(logits)
    idx = out.get("sel_idx") if want_idx else None
    if want_idx and idx is None:
        idx = torch.empty((W.numel() // m if m > 0 else 0, n), dtype=torch.uint8, device=W.device)
    fn = lib().roi_mask_fwd_soft if soft_forward else lib().roi_mask_fwd
    st = fn(_ptr(W), _ptr(logits), rows, cols, n, m, tau, lam, seed, step, elem_offset, _ptr(Wm),
            _ptr(S), _ptr(idx), _stream(W))
    _raise_on(st)
    return Wm, S, idx


def mask_bwd(grad_W_masked, W, logits, n: int, m: int, tau: float = 1.0, lam: float = 1.0,
             seed: int = 0, step: int = 0, elem_offset: int = 0, out=None):
    """dL/dlogits (fp32, same shape as logits) from dL/dW_masked (bf16)."""
    torch = _torch or _load_torch()
    _check_tensor(grad_W_masked, torch.bfloat16, "grad_W_masked")
    _check_tensor(W, torch.bfloat16, "W", like=grad_W_masked)
    _check_tensor(logits, torch.float32, "logits", like=grad_W_masked)
    rows, cols = _shape2d(W)
    d = out if out is not None else torch.empty_like(logits)
    st = lib().roi_mask_bwd(_ptr(grad_W_masked), _ptr(W), _ptr(logits), rows, cols, n, m, tau, lam,
                            seed, step, elem_offset, _ptr(d), _stream(W))
    _raise_on(st)
    return d


def adamw_params(lr: float, betas=(0.9, 0.95), eps: float = 1e-8, weight_decay: float = 0.05,
                 t: int = 1) -> AdamWParams:
    """AdamW settings of one step (defaults: the appendix's betas and weight decay)."""
    opt = AdamWParams(lr, betas[0], betas[1], eps, weight_decay, t)
    opt.betas = (float(betas[0]), float(betas[1]))  # the struct holds them in fp32
    return opt


def _step_params(opt):
    """opt's fields as they are now, the betas in 64 bits where adamw_params was given
    them so."""
    b1, b2 = opt.beta1, opt.beta2
    g1, g2 = getattr(opt, "betas", (b1, b2))
    if ctypes.c_float(g1).value == b1:
        b1 = g1
    if ctypes.c_float(g2).value == b2:
        b2 = g2
    return StepParams(opt.lr, b1, b2, opt.eps, opt.weight_decay, opt.t)


def mask_bwd_adamw(grad_W_masked, W, logits, exp_avg, exp_avg_sq, n: int, m: int,
                   tau: float = 1.0, lam: float = 1.0, seed: int = 0, step: int = 0,
                   elem_offset: int = 0, opt: AdamWParams | None = None, grad_out=None):
    """Backward with the AdamW step on the logits fused in: logits, exp_avg and
    exp_avg_sq (fp32, shaped like W) are updated in place; grad_out (fp32,
    optional) also receives dL/dlogits.  Returns grad_out."""
    torch = _torch or _load_torch()
    _check_tensor(grad_W_masked, torch.bfloat16, "grad_W_masked")
    _check_tensor(W, torch.bfloat16, "W", like=grad_W_masked)
    for t, name in ((logits, "logits"), (exp_avg, "exp_avg"), (exp_avg_sq, "exp_avg_sq")):
        _check_tensor(t, torch.float32, name, like=grad_W_masked)
    if grad_out is not None:
        _check_tensor(grad_out, torch.float32, "grad_out", like=grad_W_masked)
    if opt is None:
        raise ValueError("opt (AdamWParams) is required")
    rows, cols = _shape2d(W)
    st = lib().roi_mask_bwd_adamw(_ptr(grad_W_masked), _ptr(W), _ptr(logits), _ptr(exp_avg),
                                  _ptr(exp_avg_sq), _ptr(grad_out), rows, cols, n, m, tau, lam,
                                  seed, step, elem_offset, ctypes.addressof(opt), _stream(W))
    _raise_on(st)
    return grad_out


def mask_bwd_adamw_grouped(tensors, n: int, m: int, tau: float = 1.0, lam: float = 1.0,
                           seed: int = 0, step: int = 0, offsets=None,
                           opt: AdamWParams | None = None, grad_outs=None):
    """mask_bwd_adamw over a list of (grad_W_masked, W, logits, exp_avg,
    exp_avg_sq) in one call (in place); grad_outs: optional list of fp32
    tensors receiving dL/dlogits."""
    torch = _torch or _load_torch()
    if opt is None:
        raise ValueError("opt (AdamWParams) is required")
    fields = []
    offs = _offsets([W.numel() for _, W, *_ in tensors], offsets)
    for i, ((G, W, logits, ea, eas), off) in enumerate(zip(tensors, offs)):
        _check_tensor(G, torch.bfloat16, "grad_W_masked")
        _check_tensor(W, torch.bfloat16, "W", like=G)
        for t, name in ((logits, "logits"), (ea, "exp_avg"), (eas, "exp_avg_sq")):
            _check_tensor(t, torch.float32, name, like=G)
        d = grad_outs[i] if grad_outs is not None else None
        rows, cols = _shape2d(W)
        fields += (_ptr(G), _ptr(W), _ptr(logits), _ptr(ea), _ptr(eas), _ptr(d), rows, cols, off)
    arr = _descriptors(fields)  # roi_adamw_tensor
    stream = _stream(tensors[0][1]) if tensors else 0
    _raise_on(lib().roi_mask_bwd_adamw_grouped(ctypes.addressof(arr), len(tensors), n, m, tau,
                                               lam, seed, step, ctypes.addressof(opt), stream))


def mask_export(logits, W, n: int, m: int, want_dense: bool = True, want_values: bool = True,
                want_idx: bool = True, want_meta: bool = False):
    """Final mask (top-n of the logits per group): returns (W_masked, values
    [G, n], idx [G, n] increasing, meta uint32 [ceil(G/8)] for 2:4), each
    None unless requested."""
    torch = _torch or _load_torch()
    _check_tensor(logits, torch.float32, "logits")
    if W is not None:
        _check_tensor(W, torch.bfloat16, "W", like=logits)
    rows, cols = _shape2d(logits)
    G = logits.numel() // m if m > 0 else 0
    dev = logits.device
    Wm = torch.empty_like(W) if want_dense else None
    vals = torch.empty((G, n), dtype=torch.bfloat16, device=dev) if want_values else None
    idx = torch.empty((G, n), dtype=torch.uint8, device=dev) if want_idx else None
    meta = torch.empty(((G + 7) // 8,), dtype=torch.int32, device=dev) if want_meta else None
    _raise_on(lib().roi_mask_export(_ptr(logits), _ptr(W), rows, cols, n, m, _ptr(Wm), _ptr(vals),
                                    _ptr(idx), _ptr(meta), _stream(logits)))
    return Wm, vals, idx, meta


def cat_num_candidates(n: int, m: int) -> int:
    """binom(m, n): logits per group of the categorical sampler (-1 if not built)."""
    return int(lib().roi_cat_num_candidates(n, m))


def _check_cat(W, cat_logits, n, m):
    torch = _torch or _load_torch()
    _check_tensor(W, torch.bfloat16, "W")
    _check_tensor(cat_logits, torch.float32, "cat_logits")
    C = cat_num_candidates(n, m)
    if C < 1:
        raise RoiError(ROI_E_UNSUPPORTED, f"no categorical sampler for {n}:{m}")
    if cat_logits.numel() != (W.numel() // m) * C:
        raise ValueError(f"cat_logits must hold {C} logits per group of {m} weights")
    return C


def cat_mask_fwd(W, cat_logits, n: int, m: int, tau: float = 1.0, lam: float = 1.0,
                 seed: int = 0, step: int = 0, group_offset: int = 0, want_soft: bool = False,
                 want_choice: bool = True, out: dict | None = None):
    """Categorical sampler forward (one logit per candidate mask, [G, C] fp32):
    returns (W_masked bf16, soft mask fp32 or None, chosen candidate uint8 [G]
    or None)."""
    torch = _torch or _load_torch()
    _check_cat(W, cat_logits, n, m)
    rows, cols = _shape2d(W)
    out = out or {}
    Wm = out.get("W_masked")
    if Wm is None:
        Wm = torch.empty_like(W)
    S = out.get("soft_mask") if want_soft else None
    if want_soft and S is None:
        S = torch.empty(W.shape, dtype=torch.float32, device=W.device)
    ch = out.get("choice") if want_choice else None
    if want_choice and ch is None:
        ch = torch.empty(W.numel() // m, dtype=torch.uint8, device=W.device)
    _raise_on(lib().roi_cat_mask_fwd(_ptr(W), _ptr(cat_logits), rows, cols, n, m, tau, lam, seed,
                                     step, group_offset, _ptr(Wm), _ptr(S), _ptr(ch),
                                     _stream(W)))
    return Wm, S, ch


def cat_mask_bwd(grad_W_masked, W, cat_logits, n: int, m: int, tau: float = 1.0,
                 lam: float = 1.0, seed: int = 0, step: int = 0, group_offset: int = 0, out=None):
    """Categorical sampler backward: dL/dcat_logits (fp32, shaped like cat_logits)."""
    torch = _torch or _load_torch()
    _check_cat(W, cat_logits, n, m)
    _check_tensor(grad_W_masked, torch.bfloat16, "grad_W_masked", like=W)
    rows, cols = _shape2d(W)
    d = out if out is not None else torch.empty_like(cat_logits)
    _raise_on(lib().roi_cat_mask_bwd(_ptr(grad_W_masked), _ptr(W), _ptr(cat_logits), rows, cols,
                                     n, m, tau, lam, seed, step, group_offset, _ptr(d),
                                     _stream(W)))
    return d


def _descriptors(fields):
    """The descriptors of a grouped call, every field of which is 8 bytes wide:
    the fields of all of them in order, None for a NULL pointer."""
    return (_u64 * max(1, len(fields)))(*[0 if f is None else f for f in fields])


def _offsets(sizes, offsets):
    if offsets is not None:
        if len(offsets) != len(sizes):
            raise ValueError("one elem_offset per tensor")
        return [int(o) for o in offsets]
    out, acc = [], 0
    for k in sizes:
        out.append(acc)
        acc += k
    return out


def mask_fwd_grouped(tensors, n: int, m: int, tau: float = 1.0, lam: float = 1.0, seed: int = 0,
                     step: int = 0, offsets=None, want_soft: bool = False, want_idx: bool = True,
                     soft_forward: bool = False, outs=None):
    """mask_fwd over a list of (W, logits) pairs in one call.  The element
    offsets default to the running sum of the sizes (a stack in list order).
    Returns a list of (W_masked, soft_mask or None, sel_idx or None); `outs`
    may hold such a list, preallocated."""
    torch = _torch or _load_torch()
    given, outs, fields = outs, [], []
    offs = _offsets([W.numel() for W, _ in tensors], offsets)
    for i, ((W, logits), off) in enumerate(zip(tensors, offs)):
        _check_tensor(W, torch.bfloat16, "W")
        _check_tensor(logits, torch.float32, "logits", like=W)
        rows, cols = _shape2d(W)
        if given is not None:
            Wm, S, idx = given[i]
            S = S if want_soft else None
            idx = idx if want_idx else None
        else:
            Wm = torch.empty_like(W)
            S = torch.empty_like(logits) if want_soft else None
            idx = (torch.empty((W.numel() // m if m > 0 else 0, n), dtype=torch.uint8,
                               device=W.device) if want_idx else None)
        outs.append((Wm, S, idx))
        fields += (_ptr(W), _ptr(logits), _ptr(Wm), _ptr(S), _ptr(idx), rows, cols, off)
    arr = _descriptors(fields)  # roi_fwd_tensor
    fn = lib().roi_mask_fwd_soft_grouped if soft_forward else lib().roi_mask_fwd_grouped
    stream = _stream(tensors[0][0]) if tensors else 0
    _raise_on(fn(ctypes.addressof(arr), len(outs), n, m, tau, lam, seed, step, stream))
    return outs


def mask_bwd_grouped(tensors, n: int, m: int, tau: float = 1.0, lam: float = 1.0, seed: int = 0,
                     step: int = 0, offsets=None, outs=None):
    """mask_bwd over a list of (grad_W_masked, W, logits) triples in one call;
    returns the list of grad_logits (`outs`: preallocated, optional)."""
    torch = _torch or _load_torch()
    given, outs, fields = outs, [], []
    offs = _offsets([W.numel() for _, W, _ in tensors], offsets)
    for i, ((G, W, logits), off) in enumerate(zip(tensors, offs)):
        _check_tensor(G, torch.bfloat16, "grad_W_masked")
        _check_tensor(W, torch.bfloat16, "W", like=G)
        _check_tensor(logits, torch.float32, "logits", like=G)
        rows, cols = _shape2d(W)
        d = given[i] if given is not None else torch.empty_like(logits)
        _check_tensor(d, torch.float32, "grad_logits", like=logits)
        outs.append(d)
        fields += (_ptr(G), _ptr(W), _ptr(logits), _ptr(d), rows, cols, off)
    arr = _descriptors(fields)  # roi_bwd_tensor
    stream = _stream(tensors[0][1]) if tensors else 0
    _raise_on(lib().roi_mask_bwd_grouped(ctypes.addressof(arr), len(outs), n, m, tau, lam, seed,
                                         step, stream))
    return outs


# ------------------------------------------- the 8-bit linear layer around a mask
ROI_BF16, ROI_FP32 = 0, 1


def _dtype_code(dtype, name="dtype"):
    if dtype is _torch.bfloat16:
        return ROI_BF16
    if dtype is _torch.float32:
        return ROI_FP32
    raise TypeError(f"{name} must be torch.bfloat16 or torch.float32, got {dtype}")


def _check_sized(t, dtype, name, shape, device):
    """_check_tensor, and the shape and the device index that the other arguments
    imply."""
    if (type(t) is _torch.Tensor and t.dtype is dtype and t.shape == shape
            and t.get_device() == device and device >= 0 and t.is_contiguous()):
        return
    _check_tensor(t, dtype, name)
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, expected device {device}")


def _call(device, fn, *args):
    """fn(*args, stream) on a device and its current stream."""
    if device == _torch._C._cuda_getDevice():
        status = fn(*args, _raw_stream(device))
    else:
        with _torch.cuda.device(device):
            status = fn(*args, _raw_stream(device))
    if status:
        _raise_on(status)


def _workspace(given, need, like):
    """The workspace tensor (or None) and its bytes; allocated when none is given."""
    if given is None:
        if need > 0:
            return like.new_empty(need, dtype=_torch.uint8), need
        if need < 0:  # a status: why the call is refused
            _raise_on(need)
        return None, 0
    _check_tensor(given, _torch.uint8, "workspace")
    if given.get_device() != like.get_device():
        raise ValueError(f"workspace is on {given.device}, expected {like.device}")
    return given, given.numel()


def _rows_cols(t, name):
    """Rows and columns of a tensor whose rows have scales: 2-D, or 1-D as one row."""
    shape = t.shape
    if len(shape) == 2:
        return shape
    if len(shape) == 1:
        return 1, shape[0]
    raise ValueError(f"{name} must be 1-D or 2-D, got {len(shape)}-D (flatten the leading "
                     f"dimensions first: every row has its scale)")


def quantize_rows(x, out=None):
    """int8 rows with one fp32 scale each: x bf16 or fp32 [rows, cols] (1-D: one
    row) -> (q int8 like x, scale fp32 [rows]), x ~ q scale[:, None], |q| <= 127.
    Tokens' rows are linear_i8's operand and the checkpoint its weight gradient
    reads; weights' rows (of a masked weight, or the 2:4 export's values viewed
    as [rows, cols / 2]) are its other operand.  A row with a NaN or an infinity
    gets q = 0 and scale NaN.  ``out``: (q, scale), preallocated."""
    torch = _torch or _load_torch()
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    code = _dtype_code(x.dtype, "x")
    if not (x.is_cuda and x.is_contiguous()):
        _check_tensor(x, x.dtype, "x")
    rows, cols = _rows_cols(x, "x")
    device = x.get_device()
    if out is None:
        q = torch.empty_like(x, dtype=torch.int8)
        scale = x.new_empty(rows, dtype=torch.float32)  # 0.4 us less than torch.empty
    else:
        q, scale = out
        _check_sized(q, torch.int8, "q", x.shape, device)
        _check_sized(scale, torch.float32, "scale", (rows,), device)
    _call(device, lib().roi_quantize_rows, x.data_ptr(), code, rows, cols, q.data_ptr(),
          scale.data_ptr())
    return q, scale


def dequantize_rows(q, scale, dtype=None, out=None):
    """x = q scale[:, None] in ``dtype`` (bf16, the default, or fp32): restores
    quantize_rows' rows where the backward of another operation needs them."""
    torch = _torch or _load_torch()
    _check_tensor(q, torch.int8, "q")
    rows, cols = _rows_cols(q, "q")
    device = q.get_device()
    _check_sized(scale, torch.float32, "scale", (rows,), device)
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    code = _dtype_code(dtype)
    if out is None:
        out = torch.empty_like(q, dtype=dtype)
    else:
        _check_sized(out, dtype, "out", q.shape, device)
    _call(device, lib().roi_dequantize_rows, q.data_ptr(), scale.data_ptr(), rows, cols,
          out.data_ptr(), code)
    return out


def linear_i8(xq, xs, wq, ws, meta=None, bias=None, dtype=None, out=None, workspace=None):
    """y[t, r] = xs[t] ws[r] sum_c xq[t, c] wq[r, c] (+ bias[r]), the sum exact.

    xq int8 [tokens, cols], xs fp32 [tokens]; wq int8 [rows, cols], ws fp32
    [rows]; or 2:4-compressed: wq int8 [rows, cols / 2] (quantize_rows of
    mask_export's values as [rows, cols / 2]) with its ``meta``, cols % 32 == 0.
    bias bf16 [rows].  y [tokens, rows] in ``dtype`` (bf16, the default, or
    fp32).  ``workspace``: a uint8 tensor of linear_i8_workspace bytes."""
    torch = _torch or _load_torch()
    _check_tensor(xq, torch.int8, "xq")
    _check_tensor(wq, torch.int8, "wq")
    if xq.dim() != 2 or wq.dim() != 2:
        raise ValueError("xq and wq must be 2-D")
    (tokens, cols), (rows, held), device = xq.shape, wq.shape, xq.get_device()
    _check_sized(xs, torch.float32, "xs", (tokens,), device)
    _check_sized(ws, torch.float32, "ws", (rows,), device)
    if wq.get_device() != device:
        raise ValueError(f"wq is on {wq.device}, expected device {device}")
    if meta is not None:
        if cols % 32:
            raise ValueError(f"2:4 weights need cols % 32 == 0 (got {cols})")
        _check_sized(meta, torch.int32, "meta", (rows * cols // 32,), device)
    if held != (cols if meta is None else cols // 2):
        raise ValueError(f"wq has shape {tuple(wq.shape)}, expected "
                         f"{(rows, cols if meta is None else cols // 2)}")
    if bias is not None:
        _check_sized(bias, torch.bfloat16, "bias", (rows,), device)
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    code = _dtype_code(dtype)
    if out is None:
        out = xq.new_empty(tokens, rows, dtype=dtype)
    else:
        _check_sized(out, dtype, "out", (tokens, rows), device)
    L = lib()
    work, nbytes = _workspace(
        workspace, L.roi_linear_i8_workspace(tokens, rows, cols, meta is not None), xq)
    _call(device, L.roi_linear_i8, xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), _ptr(meta),
          ws.data_ptr(), _ptr(bias), tokens, rows, cols, out.data_ptr(), code, _ptr(work), nbytes)
    return out


def linear_i8_workspace(tokens: int, rows: int, cols: int, packed: bool = False) -> int:
    """Bytes of linear_i8's workspace (packed: 2:4-compressed weights)."""
    return _workspace_bytes(lib().roi_linear_i8_workspace(tokens, rows, cols, packed))


def _workspace_bytes(n):
    if n < 0:  # a status
        _raise_on(n)
    return int(n)


def _grad_i8(name, grad_y, q, scale, by_tokens, out, workspace):
    torch = _torch or _load_torch()
    _check_tensor(grad_y, torch.bfloat16, "grad_y")
    qname, sname = ("xq", "xs") if by_tokens else ("wq", "ws")
    _check_tensor(q, torch.int8, qname)
    if grad_y.dim() != 2 or q.dim() != 2:
        raise ValueError(f"grad_y and {qname} must be 2-D")
    (tokens, rows), cols, device = grad_y.shape, q.shape[1], grad_y.get_device()
    summed, kept = (tokens, rows) if by_tokens else (rows, tokens)
    _check_sized(q, torch.int8, qname, (summed, cols), device)
    _check_sized(scale, torch.float32, sname, (summed,), device)
    if out is None:
        out = grad_y.new_empty(kept, cols)
    else:
        _check_sized(out, torch.bfloat16, "out", (kept, cols), device)
    L = lib()
    work, nbytes = _workspace(workspace, getattr(L, name + "_workspace")(tokens, rows, cols),
                              grad_y)
    _call(device, getattr(L, name), grad_y.data_ptr(), q.data_ptr(), scale.data_ptr(), tokens,
          rows, cols, out.data_ptr(), _ptr(work), nbytes)
    return out


def linear_i8_grad_weight(grad_y, xq, xs, out=None, workspace=None):
    """dL/dW (bf16 [rows, cols], mask_bwd's grad_W_masked) of a linear layer from
    dL/dy (bf16 [tokens, rows]) and the 8-bit checkpoint of its input:
    sum_t grad_y[t, r] xs[t] xq[t, c]."""
    return _grad_i8("roi_linear_i8_grad_weight", grad_y, xq, xs, True, out, workspace)


def linear_i8_grad_input(grad_y, wq, ws, out=None, workspace=None):
    """dL/dx (bf16 [tokens, cols]) of a linear layer with int8 weight rows:
    sum_r grad_y[t, r] ws[r] wq[r, c]."""
    return _grad_i8("roi_linear_i8_grad_input", grad_y, wq, ws, False, out, workspace)


def linear_i8_grad_weight_workspace(tokens: int, rows: int, cols: int) -> int:
    """Bytes of linear_i8_grad_weight's workspace."""
    return _workspace_bytes(lib().roi_linear_i8_grad_weight_workspace(tokens, rows, cols))


def linear_i8_grad_input_workspace(tokens: int, rows: int, cols: int) -> int:
    """Bytes of linear_i8_grad_input's workspace."""
    return _workspace_bytes(lib().roi_linear_i8_grad_input_workspace(tokens, rows, cols))


# ------------------------------------------- the training step in 8-bit floats
ROI_E4M3, ROI_E5M2 = 0, 1


def _format_code(dtype, name):
    if dtype is _torch.float8_e4m3fn:
        return ROI_E4M3
    if dtype is _torch.float8_e5m2:
        return ROI_E5M2
    raise TypeError(f"{name} must be torch.float8_e4m3fn or torch.float8_e5m2, got {dtype}")


def block_scales(cols: int) -> int:
    """Scales kept for a row of ``cols`` values: one byte a block of 128, in whole words."""
    return (cols + 511) // 512 * 4


def _f8_new(like, rows, cols, dtype):
    """[rows, cols] of 8-bit values whose rows start at multiples of 16 bytes."""
    room = (cols + 15) // 16 * 16
    t = like.new_empty(rows, room, dtype=dtype)
    return t if room == cols else t[:, :cols]


def _f8_stride(t, name):
    """Bytes between the rows of a 2-D tensor of 8-bit values."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D, got {t.dim()}-D")
    rows, cols = t.shape
    stride, step = t.stride()
    if rows <= 1 or cols == 0:  # any stride says the same
        stride = (cols + 15) // 16 * 16
    if (step != 1 and cols > 1) or stride % 16 or stride < cols:
        raise ValueError(f"{name} must have consecutive columns and rows that start at multiples "
                         f"of 16 bytes (quantize_blocks lays them out so), got strides "
                         f"{tuple(t.stride())}")
    return stride


def _check_scales(t, name, rows, cols, device):
    """The scales of `rows` rows (of blocks) of `cols` values."""
    _check_sized(t, _torch.float8_e8m0fnu, name, (rows, block_scales(cols)), device)


def quantize_blocks(x, square: bool = False, transposed: bool = False, dtype=None, out=None):
    """8-bit floats with one power-of-two scale for each block of 128 values.

    x bf16 or fp32 [rows, cols] -> (q, scale): q in ``dtype`` (float8_e4m3fn, the
    default, or float8_e5m2) [rows, cols], its rows at multiples of 16 bytes;
    scale float8_e8m0fnu [rows, block_scales(cols)], scale[r, b] that of q[r, 128 b
    : 128 b + 128].  square: blocks are 128 x 128 (a weight's), scale
    [ceil(rows / 128), block_scales(cols)].  transposed: also (qt, scale_t) of the
    transposed x, [cols, rows], with blocks along the rows of x; with square the
    transposed q.  Tokens' rows are linear_f8's left operand, their transposed
    copies (the checkpoint, and dL/dy's) its weight gradient's; a weight's square
    blocks its right operand, and their transposed copy that of the input's
    gradient.  A 1-D x is one row: q and scale are 1-D.  ``out``: what is returned,
    preallocated."""
    torch = _torch or _load_torch()
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    code = _dtype_code(x.dtype, "x")
    if not (x.is_cuda and x.is_contiguous()):
        _check_tensor(x, x.dtype, "x")
    rows, cols = _rows_cols(x, "x")
    flat = x.dim() == 1
    if flat and transposed:
        raise ValueError("a transposed copy is made of a 2-D x")
    device = x.get_device()
    above, below = ((rows + 127) // 128, (cols + 127) // 128) if square else (rows, cols)
    qt = scale_t = None
    if out is None:
        dtype = torch.float8_e4m3fn if dtype is None else dtype
        fmt = _format_code(dtype, "dtype")
        q = x.new_empty(cols, dtype=dtype) if flat else _f8_new(x, rows, cols, dtype)
        shape = (block_scales(cols),) if flat else (above, block_scales(cols))
        scale = x.new_empty(shape, dtype=torch.float8_e8m0fnu)
        if transposed:
            qt = _f8_new(x, cols, rows, dtype)
            scale_t = x.new_empty(below, block_scales(rows), dtype=torch.float8_e8m0fnu)
        out = (q, scale, qt, scale_t) if transposed else (q, scale)
        stride = (cols + 15) // 16 * 16
        stride_t = (rows + 15) // 16 * 16
    else:
        q, scale = out[:2]
        if len(out) != (4 if transposed else 2):
            raise ValueError(f"out must hold {4 if transposed else 2} tensors, got {len(out)}")
        fmt = _format_code(q.dtype, "q")
        if dtype is not None and q.dtype is not dtype:
            raise TypeError(f"q must be {dtype}, got {q.dtype}")

        def check(q, scale, name, rows, cols, blocks):
            if q.dtype is not out[0].dtype:
                raise TypeError(f"{name} must be {out[0].dtype}, got {q.dtype}")
            if q.shape != (rows, cols) or q.get_device() != device:
                raise ValueError(f"{name} must have shape {(rows, cols)} on {x.device}, got "
                                 f"{tuple(q.shape)} on {q.device}")
            _check_scales(scale, "scale" + name[1:].replace("t", "_t"), blocks, cols, device)
            return _f8_stride(q, name)

        if flat:
            _check_sized(q, q.dtype, "q", x.shape, device)
            _check_sized(scale, torch.float8_e8m0fnu, "scale", (block_scales(cols),), device)
            stride = (cols + 15) // 16 * 16
        else:
            stride = check(q, scale, "q", rows, cols, above)
        stride_t = 0
        if transposed:
            qt, scale_t = out[2:]
            stride_t = check(qt, scale_t, "qt", cols, rows, below)
    _call(device, lib().roi_quantize_blocks, x.data_ptr(), code, rows, cols, square, fmt,
          q.data_ptr(), stride, scale.data_ptr(), _ptr(qt), stride_t, _ptr(scale_t))
    return out


def dequantize_blocks(q, scale, dtype=None, out=None):
    """x = q times its blocks' scales in ``dtype`` (bf16, the default, or fp32).
    ``scale`` as quantize_blocks gives it: with a row for each row of q, or for each
    128 (square blocks)."""
    torch = _torch or _load_torch()
    if not isinstance(q, torch.Tensor):
        raise TypeError("q must be a torch.Tensor")
    fmt = _format_code(q.dtype, "q")
    flat = q.dim() == 1
    square = False
    device = q.get_device()
    if flat:
        _check_tensor(q, q.dtype, "q")
        rows, cols = 1, q.shape[0]
        stride = (cols + 15) // 16 * 16
        _check_sized(scale, torch.float8_e8m0fnu, "scale", (block_scales(cols),), device)
    else:
        stride = _f8_stride(q, "q")
        rows, cols = q.shape
        square = _square_scales(scale, rows)
        _check_scales(scale, "scale", (rows + 127) // 128 if square else rows, cols, device)
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    code = _dtype_code(dtype)
    if out is None:
        out = q.new_empty(q.shape, dtype=dtype)
    else:
        _check_sized(out, dtype, "out", q.shape, device)
    _call(device, lib().roi_dequantize_blocks, q.data_ptr(), stride, scale.data_ptr(), rows, cols,
          square, fmt, out.data_ptr(), code)
    return out


def _square_scales(scale, rows):
    """Whether scales are those of square blocks (with one row both are the same)."""
    return (rows > 1 and isinstance(scale, _torch.Tensor) and scale.dim() == 2
            and scale.shape[0] == (rows + 127) // 128)


def linear_f8(xq, xs, wq, ws, bias=None, out=None, workspace=None):
    """y[t, r] = sum_c x[t, c] w[r, c] (+ bias[r]) of operands in blocks, bf16.

    xq [tokens, cols] (e4m3 or e5m2) with xs, quantize_blocks of the tokens' rows;
    wq e4m3 [rows, cols] with ws, the scales of square blocks or of rows.  bias bf16
    [rows].  ``workspace``: a uint8 tensor of linear_f8_workspace bytes."""
    torch = _torch or _load_torch()
    if not (isinstance(xq, torch.Tensor) and isinstance(wq, torch.Tensor)):
        raise TypeError("xq and wq must be torch.Tensors")
    fmt = _format_code(xq.dtype, "xq")
    if wq.dtype is not torch.float8_e4m3fn:
        raise TypeError(f"wq must be torch.float8_e4m3fn, got {wq.dtype}")
    x_stride, w_stride = _f8_stride(xq, "xq"), _f8_stride(wq, "wq")
    (tokens, cols), (rows, held), device = xq.shape, wq.shape, xq.get_device()
    if held != cols:
        raise ValueError(f"wq has {held} columns, expected {cols}")
    if wq.get_device() != device:
        raise ValueError(f"wq is on {wq.device}, expected device {device}")
    square = _square_scales(ws, rows)
    _check_scales(xs, "xs", tokens, cols, device)
    _check_scales(ws, "ws", (rows + 127) // 128 if square else rows, cols, device)
    if bias is not None:
        _check_sized(bias, torch.bfloat16, "bias", (rows,), device)
    if out is None:
        out = xq.new_empty(tokens, rows, dtype=torch.bfloat16)
    else:
        _check_sized(out, torch.bfloat16, "out", (tokens, rows), device)
    L = lib()
    work, nbytes = _workspace(workspace, L.roi_linear_f8_workspace(tokens, rows, cols), xq)
    _call(device, L.roi_linear_f8, xq.data_ptr(), x_stride, xs.data_ptr(), fmt, wq.data_ptr(),
          w_stride, ws.data_ptr(), square, _ptr(bias), tokens, rows, cols, out.data_ptr(),
          _ptr(work), nbytes)
    return out


def linear_f8_grad_input(gq, gs, wqt, wst, out=None, workspace=None):
    """dL/dx (bf16 [tokens, cols]): sum_r dy[t, r] w[r, c], from quantize_blocks of
    dL/dy (gq [tokens, rows], gs) and the weight's transposed copy (wqt [cols, rows],
    wst)."""
    return linear_f8(gq, gs, wqt, wst, None, out, workspace)


def linear_f8_grad_weight(gqt, gst, xqt, xst, out=None, workspace=None):
    """dL/dW (bf16 [rows, cols], mask_bwd's grad_W_masked): sum_t dy[t, r] x[t, c],
    from the transposed copies of dL/dy (gqt [rows, tokens], gst) and of the forward's
    x (xqt e4m3 [cols, tokens], xst)."""
    return linear_f8(gqt, gst, xqt, xst, None, out, workspace)


def linear_f8_workspace(tokens: int, rows: int, cols: int) -> int:
    """Bytes of the workspace of linear_f8 with xq [tokens, cols] and wq [rows, cols]
    (of the gradients: with the shapes of their operands)."""
    return _workspace_bytes(lib().roi_linear_f8_workspace(tokens, rows, cols))


def adamw_moments(param, bits: int = 8):
    """The moments of a tensor before the first step: (exp_avg, exp_avg_sq) for
    adamw_grouped, fp32 zeros like param (bits 32), or each (q float8_e4m3fn like
    param, scale float8_e8m0fnu [block_scales(param.numel())]) (bits 8; exp_avg_sq
    holds the root of the second moment)."""
    torch = _torch or _load_torch()
    if bits == 32:
        return torch.zeros_like(param), torch.zeros_like(param)
    if bits != 8:
        raise ValueError(f"bits must be 8 or 32, got {bits}")

    def zeros():
        scale = torch.zeros(block_scales(param.numel()), dtype=torch.uint8, device=param.device)
        q = torch.zeros(param.shape, dtype=torch.uint8, device=param.device)
        return q.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)

    return zeros(), zeros()


class AdamWPlan:
    """The checked tensors of adamw_grouped, kept for many steps (adamw_plan)."""

    def __init__(self, tensors, offsets=None):
        torch = _torch or _load_torch()
        self.tensors = [tuple(t) for t in tensors]
        self.count = len(self.tensors)
        sizes = [p.numel() for p, *_ in self.tensors]
        self.offsets = _offsets([(n + 3) // 4 * 4 for n in sizes], offsets)
        self.bits, self.grad_code, self.device = 32, ROI_FP32, -1
        fields = []
        for i, ((param, grad, avg, sq), n, off) in enumerate(zip(self.tensors, sizes,
                                                                 self.offsets)):
            eight = isinstance(avg, (tuple, list))
            if eight != isinstance(sq, (tuple, list)):
                raise TypeError(f"tensor {i}: both moments are tensors, or both (q, scale)")
            _check_tensor(param, torch.float32, "param")
            if i == 0:
                self.bits, self.device = 8 if eight else 32, param.get_device()
                self.grad_code = _dtype_code(grad.dtype, "grad")
            if (8 if eight else 32) != self.bits or _dtype_code(grad.dtype, "grad") != self.grad_code:
                raise TypeError(f"tensor {i}: its moments or its gradient are of another type than "
                                f"tensor 0's")
            if param.get_device() != self.device:
                raise ValueError(f"tensor {i} is on {param.device}, expected device {self.device}")
            shape = param.shape
            _check_sized(grad, grad.dtype, "grad", shape, self.device)
            if eight:
                for (q, s), name in ((avg, "exp_avg"), (sq, "exp_avg_sq")):
                    _check_sized(q, torch.float8_e4m3fn, name, shape, self.device)
                    _check_sized(s, torch.float8_e8m0fnu, name + "'s scale", (block_scales(n),),
                                 self.device)
                fields += (param.data_ptr(), grad.data_ptr(), avg[0].data_ptr(), sq[0].data_ptr(),
                           avg[1].data_ptr(), sq[1].data_ptr(), n, off)
            else:
                _check_sized(avg, torch.float32, "exp_avg", shape, self.device)
                _check_sized(sq, torch.float32, "exp_avg_sq", shape, self.device)
                fields += (param.data_ptr(), grad.data_ptr(), avg.data_ptr(), sq.data_ptr(), 0, 0, n,
                           off)
        self.descriptors = _descriptors(fields)  # roi_step_tensor
        self.address = ctypes.addressof(self.descriptors)


def adamw_plan(tensors, offsets=None) -> AdamWPlan:
    """Checks adamw_grouped's list of tensors once and keeps it: what a training loop
    whose gradients stay in place passes to each step instead of the list.  It steps the
    memory that they had then: a tensor given new memory (``p.data = ...``, a gradient
    set to None) needs a new plan."""
    plan = AdamWPlan(tensors, offsets)

    def alias(t):  # keeps the memory that the descriptors point into
        return t.detach() if isinstance(t, _torch.Tensor) else tuple(map(alias, t))

    plan.tensors = [tuple(map(alias, t)) for t in plan.tensors]
    return plan


def adamw_grouped(tensors, opt: AdamWParams, seed: int = 0, step: int = 0, offsets=None):
    """One AdamW step over a list of (param, grad, exp_avg, exp_avg_sq), in place, in
    one call; or over an adamw_plan of it.

    param fp32; grad fp32 or bf16; the moments fp32, or each (q, scale) in 8 bits
    (adamw_moments; about half the memory traffic and a quarter of the memory).  The
    8-bit moments are rounded by the noise of (seed, step, offsets[i] + element):
    use a seed of its own and the step's number; offsets are multiples of 4 and
    default to the running sum of the sizes, each rounded up to one.  A list is checked
    in every call, some 3 us a tensor on the host."""
    if opt is None:
        raise ValueError("opt (AdamWParams) is required")
    plan = tensors
    if type(plan) is not AdamWPlan:
        plan = AdamWPlan(tensors, offsets)
    elif offsets is not None:
        raise ValueError("the plan has its offsets")
    if plan.count:
        params = _step_params(opt)  # alive during the call
        _call(plan.device, lib().roi_adamw_grouped, plan.address, plan.count, plan.grad_code,
              plan.bits, seed, step, ctypes.addressof(params))


def gumbel_noise(count: int, seed: int = 0, step: int = 0, elem_offset: int = 0, device="cuda",
                 want_words: bool = True, want_gumbel: bool = True):
    """Raw Philox words (as int32 bit patterns) and Gumbel noise of `count` elements."""
    torch = _torch or _load_torch()
    words = torch.empty(count, dtype=torch.int32, device=device) if want_words else None
    g = torch.empty(count, dtype=torch.float32, device=device) if want_gumbel else None
    ref = words if words is not None else g
    st = lib().roi_gumbel_noise(seed, step, elem_offset, count, _ptr(words), _ptr(g), _stream(ref))
    _raise_on(st)
    return words, g


def gumbel_from_words(words):
    """g = -L(-L(u(x))) for int32 tensors holding 32-bit words."""
    torch = _torch or _load_torch()
    _check_tensor(words, torch.int32, "words")
    g = torch.empty(words.shape, dtype=torch.float32, device=words.device)
    _raise_on(lib().roi_gumbel_from_words(_ptr(words), words.numel(), _ptr(g), _stream(words)))
    return g


def stream_copy(src, dst):
    """Plain streaming copy of src into dst (device tensors of the same byte
    size, a multiple of 16): the benchmark's data-movement reference."""
    if src.numel() * src.element_size() != dst.numel() * dst.element_size():
        raise ValueError("src and dst differ in size")
    _raise_on(lib().roi_stream_copy(_ptr(src), _ptr(dst), src.numel() * src.element_size(),
                                    _stream(src)))
    return dst


def fast_noise_from_words(words):
    """K = -log2(-log2 u(x)) from the hardware logarithm, for int32 word tensors."""
    torch = _torch or _load_torch()
    _check_tensor(words, torch.int32, "words")
    out = torch.empty(words.shape, dtype=torch.float32, device=words.device)
    _raise_on(lib().roi_fast_noise_from_words(_ptr(words), words.numel(), _ptr(out),
                                              _stream(words)))
    return out


def anneal(v_init: float, v_end: float, t: int, t_anneal: int) -> float:
    """§4.2.3 exponential annealing of a temperature (host-side)."""
    return float(lib().roi_anneal(v_init, v_end, t, t_anneal))
