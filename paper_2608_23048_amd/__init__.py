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
    return AdamWParams(lr, betas[0], betas[1], eps, weight_decay, t)


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
