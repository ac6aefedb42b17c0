"""Thin Python binding of libcmsd.so (ctypes).

Argument marshalling only: torch supplies device memory and the current
stream; every step of the logits pass runs in the library's CUDA kernels.
There is no CPU fallback -- if libcmsd.so is missing or fails to load, every
call raises.
"""
from __future__ import annotations

import ctypes
import os
import threading

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcmsd.so")

F32, BF16 = 0, 1
RULE_PAPER, RULE_SAMPLED = 0, 1
OK, EINVAL, EDTYPE, ECUDA, ENOWS, EALIGN, ESCRATCH = 0, -1, -2, -3, -4, -5, -6

_c_int, _c_u32, _c_u64, _c_sz, _vp = ctypes.c_int, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_void_p


class Params(ctypes.Structure):
    """cmsd_params (include/cmsd.h)."""
    _fields_ = [
        ("k_min", ctypes.c_int32), ("k_max", ctypes.c_int32),
        ("lam", ctypes.c_float * 3),
        ("beta_sig", ctypes.c_float),
        ("beta_rank", ctypes.c_int32),
        ("alpha", ctypes.c_float),
        ("tau_base", ctypes.c_float),
        ("gamma", ctypes.c_float),
        ("tau_sign", ctypes.c_int32),
        ("rule", ctypes.c_int32),
        ("k_fixed", ctypes.c_int32),
        ("bonus", ctypes.c_int32),
    ]

    def as_dict(self):
        return dict(k_min=self.k_min, k_max=self.k_max, lam=tuple(float(x) for x in self.lam),
                    beta_sig=float(self.beta_sig), beta_rank=self.beta_rank, alpha=float(self.alpha),
                    tau_base=float(self.tau_base), gamma=float(self.gamma), tau_sign=self.tau_sign,
                    rule="sampled" if self.rule == RULE_SAMPLED else "paper", k_fixed=self.k_fixed,
                    bonus=bool(self.bonus))


class CmsdError(RuntimeError):
    pass


_lib = None
_lib_lock = threading.Lock()

_SIGS = {
    "cmsd_params_default": (None, [_vp, _c_int, _c_int]),
    "cmsd_params_preset": (_c_int, [_vp, _c_int, _c_int, _c_int]),
    "cmsd_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_workspace_init": (_c_int, [_vp, _c_sz, _vp]),
    "cmsd_workspace_errors": (_c_int, [_vp, _c_sz, _vp, ctypes.POINTER(ctypes.c_uint32)]),
    "cmsd_test_record_wait_timeout": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp, _c_sz, _vp]),
    "cmsd_test_choose": (_c_int, [_c_int] * 9 + [_vp, _vp, _vp]),
    "cmsd_confidence": (_c_int, [_vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp,
                                 _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_sz, _vp]),
    "cmsd_verify": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp,
                             _vp, _vp, _c_u64, _c_u32, _vp, _vp, _vp, _vp, _c_sz, _vp]),
    "cmsd_confidence_verify": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp,
                                        _c_u64, _c_u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _c_sz, _vp]),
    "cmsd_test_draw": (_c_int, [_c_int] * 5 + [_vp, _vp]),
    "cmsd_test_confidence_verify_cluster": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp,
                                                     _c_u64, _c_u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                                     _vp, _c_sz, _vp, _c_int, _c_int]),
    "cmsd_confidence_verify_static": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp,
                                               _c_u64, _c_u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                               _vp, _vp]),
    "cmsd_lmhead_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_lmhead_confidence": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _vp, _c_sz, _vp]),
    "cmsd_lmhead_loss_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_lmhead_loss": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp, _vp, _c_sz, _vp]),
    "cmsd_lmhead_loss_backward_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_lmhead_loss_backward": (_c_int, [_vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp,
                                           _vp, _c_sz, _vp]),
    "cmsd_quantize_rows": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _vp]),
    "cmsd_lmhead_i8_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_lmhead_i8": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _vp, _c_int, _vp, _c_sz, _vp]),
    "cmsd_embedding": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_int, ctypes.c_float, _vp, _vp]),
    "cmsd_embedding_backward_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int]),
    "cmsd_embedding_backward": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_int, ctypes.c_float, _c_int,
                                         _vp, _vp, _c_sz, _vp]),
    "cmsd_embedding_errors": (_c_int, [_vp, ctypes.POINTER(ctypes.c_uint32)]),
    "cmsd_layernorm": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, ctypes.c_float, _vp, _vp, _vp, _vp]),
    "cmsd_layernorm_backward_workspace_bytes": (_c_sz, [_c_int, _c_int]),
    "cmsd_layernorm_backward": (_c_int, [_vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp, _vp, _vp,
                                         _c_sz, _vp]),
    "cmsd_dropout": (_c_int, [_vp, _vp, _c_int, ctypes.c_int64, ctypes.c_double, _c_u64, _c_u32, _c_u32, _vp, _vp,
                              _vp]),
    "cmsd_dropout_backward": (_c_int, [_vp, _c_int, ctypes.c_int64, ctypes.c_double, _c_u64, _c_u32, _c_u32, _vp,
                                       _vp, _vp]),
    "cmsd_test_head_wait": (_c_int, [_c_int, _vp, _c_sz, _vp]),
    "cmsd_lmhead_errors": (_c_int, [_vp, ctypes.POINTER(ctypes.c_uint32)]),
    "cmsd_philox_u32": (_c_u32, [_c_u64, _c_u32, _c_u32, _c_u32, _c_u32, _c_int]),
    "cmsd_philox_fill": (_c_int, [_c_u64, _c_u32, _c_u32, _c_u32, _c_u32, _vp, _c_sz, _vp]),
    "cmsd_profile_start": (_c_int, [_c_int]),
    "cmsd_profile_stop": (_c_int, [_vp, _vp, _c_int, ctypes.POINTER(ctypes.c_int)]),
    "cmsd_launch_plan": (_c_int, [_c_int] * 5 + [_vp, _c_int] + [ctypes.POINTER(ctypes.c_int)] * 3),
    "cmsd_launch_info": (_c_int, [_c_int, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]),
    "cmsd_strerror": (ctypes.c_char_p, [_c_int]),
    "cmsd_last_cuda_error": (_c_int, []),
}


def lib():
    """The loaded libcmsd.so (raises if it is missing)."""
    global _lib
    if _lib is None:
        with _lib_lock:
            if _lib is None:
                if not os.path.exists(LIB_PATH):
                    raise CmsdError(f"{LIB_PATH} is missing: build it with "
                                    "`python -c 'import __graft_entry__ as g; g.build()'`")
                L = ctypes.CDLL(LIB_PATH)
                for name, (res, args) in _SIGS.items():
                    fn = getattr(L, name)
                    fn.restype = res
                    fn.argtypes = args
                _lib = L
    return _lib


def _check(rc, what):
    if rc != OK:
        msg = lib().cmsd_strerror(rc).decode()
        if rc == ECUDA:
            msg += f" (cudaError {lib().cmsd_last_cuda_error()})"
        raise CmsdError(f"{what}: {msg} [{rc}]")


PRESETS = {"full": 0, "fixed_k": 1, "fixed_tau": 2, "fixed_k_tau": 3, "entropy_only": 4,
           "margin_only": 5, "softmax_only": 6}


def params(K, rule="paper", preset="full", **kw):
    """cmsd_params for window K, rule ('paper' or 'sampled') and ablation
    preset (PRESETS: the variants of Table III), then overrides.

    Keyword names: k_min, k_max, lam (3-tuple), beta_sig, beta_rank, alpha,
    tau_base, gamma, tau_sign, k_fixed, bonus.
    """
    r = RULE_SAMPLED if rule in ("sampled", RULE_SAMPLED) else RULE_PAPER
    p = Params()
    _check(lib().cmsd_params_preset(ctypes.byref(p), int(K), r, PRESETS[preset]), "cmsd_params_preset")
    for k, v in kw.items():
        if k == "lam":
            for j in range(3):
                p.lam[j] = float(v[j])
        elif k == "rule":
            p.rule = RULE_SAMPLED if v in ("sampled", RULE_SAMPLED) else RULE_PAPER
        elif k == "bonus":
            p.bonus = 1 if v else 0
        else:
            setattr(p, k, v)
    return p


_torch_mod = None
_raw_stream = None      # (device index) -> cudaStream_t of the current stream, without a Stream object
_get_device = None      # () -> index of the current device, of a runtime that is initialised
_forward_ad = None      # torch.autograd.forward_ad


def _torch():
    global _torch_mod, _raw_stream, _get_device, _forward_ad
    if _torch_mod is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _forward_ad = torch.autograd.forward_ad
        _torch_mod = torch
    return _torch_mod


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise CmsdError(f"logits must be float32 or bfloat16, got {t.dtype}")


def _check_target(draft, target, p):
    B, K, V = draft.shape
    want = (B, K + 1, V) if p.bonus else (B, K, V)
    if draft.dtype != target.dtype or tuple(target.shape) != want:
        raise CmsdError(f"target logits must be {want} of the drafter's dtype, got {tuple(target.shape)}")


def _stream():
    torch = _torch_mod or _torch()
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _need_cuda(*ts):
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise CmsdError("all tensors must be CUDA tensors (the library has no CPU path)")
            if not t.is_contiguous():
                raise CmsdError("tensors must be contiguous")


_ws_cache = {}
_ws_lock = threading.Lock()


def workspace(B, K, V, device=None):
    """A zero-initialised workspace for (B, K, V), cached per device."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device() if device is None else device)
    key = (dev.index, B, K, V)
    with _ws_lock:
        ws = _ws_cache.get(key)
        if ws is None:
            n = int(lib().cmsd_workspace_bytes(B, K, V))
            if n == 0:
                raise CmsdError("cmsd_workspace_bytes failed")
            ws = torch.empty(n, dtype=torch.uint8, device=dev)
            _check(lib().cmsd_workspace_init(_ptr(ws), n, _stream()), "cmsd_workspace_init")
            _ws_cache[key] = ws
    return ws


def workspace_errors(ws):
    f = ctypes.c_uint32(0)
    _check(lib().cmsd_workspace_errors(_ptr(ws), ws.numel(), _stream(), ctypes.byref(f)),
           "cmsd_workspace_errors")
    return int(f.value)


def _out(out, name, shape, dtype, device, want=True):
    if out is not None and name in out:
        return out[name]
    if not want:
        return None
    return _torch().empty(shape, dtype=dtype, device=device)


def confidence(draft, k_row=None, p=None, out=None, ws=None):
    """Confidence pass; returns dict H, margin, argmax, conf, lse, k_next (torch tensors)."""
    torch = _torch()
    _need_cuda(draft, k_row)
    B, K, V = draft.shape
    p = p if p is not None else params(K)
    dev = draft.device
    o = {n: _out(out, n, (B, K), torch.float32, dev) for n in ("H", "margin", "conf", "lse")}
    o["argmax"] = _out(out, "argmax", (B, K), torch.int32, dev)
    o["k_next"] = _out(out, "k_next", (B,), torch.int32, dev)
    ws = ws if ws is not None else workspace(B, K, V)
    rc = lib().cmsd_confidence(_ptr(draft), B, K, V, _dtype_code(draft), _ptr(k_row), ctypes.byref(p),
                               _ptr(o["H"]), _ptr(o["margin"]), _ptr(o["argmax"]), _ptr(o["conf"]),
                               _ptr(o["lse"]), _ptr(o["k_next"]), _ptr(ws), ws.numel(), _stream())
    _check(rc, "cmsd_confidence")
    return o


def lmhead_workspace(R, d, V):
    """A workspace for cmsd_lmhead_confidence(R, d, V) on the current device."""
    torch = _torch()
    n = int(lib().cmsd_lmhead_workspace_bytes(R, d, V))
    if n == 0:
        raise CmsdError("cmsd_lmhead_workspace_bytes failed")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def lmhead_confidence(hidden, weight, p=None, logits=False, out=None, ws=None):
    """The drafter's LM head fused with the confidence signals.

    hidden: bf16 [R, d] (torch.bfloat16 or int16/uint16 bits), weight: bf16
    [V, d].  Returns dict H, margin, argmax, conf, lse ([R]) and, with
    logits=True, the fp32 logits [R, V]."""
    torch = _torch()
    _need_cuda(hidden, weight)
    if hidden.element_size() != 2 or weight.element_size() != 2:
        raise CmsdError("hidden and weight must hold 16-bit (bf16) values")
    R, d = hidden.shape
    V, d2 = weight.shape
    if d2 != d:
        raise CmsdError("hidden [R, d] and weight [V, d] must share d")
    cur = torch.cuda.current_device()
    if hidden.get_device() != cur or weight.get_device() != cur:
        raise CmsdError("hidden and weight must be on the current device")
    p = p if p is not None else params(1)
    dev = hidden.device
    o = {n: _out(out, n, (R,), torch.float32, dev) for n in ("H", "margin", "conf", "lse")}
    o["argmax"] = _out(out, "argmax", (R,), torch.int32, dev)
    if logits:
        o["logits"] = _out(out, "logits", (R, V), torch.float32, dev)
    ws = ws if ws is not None else lmhead_workspace(R, d, V)
    rc = lib().cmsd_lmhead_confidence(_ptr(hidden), _ptr(weight), R, d, V, ctypes.byref(p), _ptr(o["H"]),
                                      _ptr(o["margin"]), _ptr(o["argmax"]), _ptr(o["conf"]), _ptr(o["lse"]),
                                      _ptr(o.get("logits")), _ptr(ws), ws.numel(), _stream())
    _check(rc, "cmsd_lmhead_confidence")
    return o


def _refuse(name, t, shape, dtype, cur):
    """Says what is wrong with a tensor that _need does not take."""
    if t is None or t.dtype is not dtype or t.shape != shape:
        got = "nothing" if t is None else f"{t.dtype} {tuple(t.shape)}"
        raise CmsdError(f"{name} must be {dtype} {tuple(shape)}, got {got}")
    if not t.is_cuda:
        raise CmsdError(f"{name} must be a CUDA tensor (the library has no CPU path)")
    if t.get_device() != cur:
        raise CmsdError(f"{name} must be on the current device")
    raise CmsdError(f"{name} must be contiguous")


def _need(cur, specs):
    """Each (tensor, shape, dtype, name) a contiguous CUDA tensor of that shape and type on device cur."""
    for t, shape, dtype, name in specs:
        if (t is None or t.dtype is not dtype or t.shape != shape or t.get_device() != cur
                or not t.is_contiguous()):
            _refuse(name, t, shape, dtype, cur)
    if cur < 0:
        raise CmsdError("all tensors must be CUDA tensors (the library has no CPU path)")


def _current(t):
    """The current device, where t is a CUDA tensor at all (-1 otherwise: nothing is asked of the runtime)."""
    return _get_device() if t.is_cuda else -1


def _need_ws(ws, cur):
    if ws.get_device() != cur or not ws.is_contiguous():
        raise CmsdError("the workspace must be contiguous on the current device")
    return ws.numel() * ws.element_size()


def _stream_of(cur):
    return _raw_stream(cur) if _raw_stream is not None else _torch_mod.cuda.current_stream().cuda_stream


_INT_MAX = 0x7FFFFFFF      # ctypes takes larger integers modulo 2^32


def _too_large(what):
    raise CmsdError(f"{what}: sizes out of range")


def _ignored(index):
    index = int(index)
    if not -_INT_MAX - 1 <= index <= _INT_MAX:
        raise CmsdError("ignore_index must be a 32-bit integer, as labels and tokens are")
    return index


def _head_sizes(hidden, weight):
    h, w = hidden.shape, weight.shape
    if len(h) != 2 or len(w) != 2 or h[1] != w[1]:
        raise CmsdError("hidden [R, d] and weight [V, d] must share d")
    R, d, V = h[0], h[1], w[0]
    if R > _INT_MAX or d > _INT_MAX or V > _INT_MAX:
        _too_large("hidden [R, d], weight [V, d]")
    return R, d, V


def _given(out, name, shape, dtype, like):
    if out is not None and name in out:
        return out[name]
    return _torch_mod.empty(shape, dtype=dtype, device=like.device)


def _head_workspace(what, R, d, V):
    torch = _torch()
    if max(R, d, V) > _INT_MAX:
        _too_large(what)
    n = int(getattr(lib(), what)(int(R), int(d), int(V)))
    if n == 0:
        raise CmsdError(f"{what}: sizes out of range")
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    _check(lib().cmsd_workspace_init(_ptr(ws), 4, _stream()), "cmsd_workspace_init")   # the error word
    return ws


def lmhead_loss_workspace(R, d, V):
    """A workspace for lmhead_loss(R, d, V) on the current device (workspace_errors reads its error word)."""
    return _head_workspace("cmsd_lmhead_loss_workspace_bytes", R, d, V)


def lmhead_loss_backward_workspace(R, d, V):
    """A workspace for lmhead_loss_backward(R, d, V) on the current device."""
    return _head_workspace("cmsd_lmhead_loss_backward_workspace_bytes", R, d, V)


def lmhead_i8_workspace(R, d, V):
    """A workspace for lmhead_i8(R, d, V) on the current device."""
    return _head_workspace("cmsd_lmhead_i8_workspace_bytes", R, d, V)


def lmhead_errors():
    """The error bits of the calls of lmhead_loss, lmhead_loss_backward and lmhead_i8 on the current device
    since they were last read here, whether or not the caller keeps their workspace (bit 0: a label that is
    neither in the vocabulary nor ignore_index; bit 2: a wait gave up, the results are void).  Clears them and
    waits for the current stream."""
    f = ctypes.c_uint32(0)
    _torch()
    _check(lib().cmsd_lmhead_errors(_stream(), ctypes.byref(f)), "cmsd_lmhead_errors")
    return int(f.value)


def lmhead_loss(hidden, weight, labels, ignore_index=-100, out=None, ws=None):
    """Softmax cross entropy of the head's logits hidden @ weight.T, which are not kept.

    hidden: bf16 [R, d], weight: bf16 [V, d], labels: int32 [R].  Nothing is recorded for autograd: tensors that
    require gradients are refused while it records.  Returns dict
    loss and lse ([R], float32; 0 in rows whose label is ignore_index).  Without ws a workspace is made for the
    call, here and in the calls below; what went wrong is read with lmhead_errors."""
    torch = _torch()
    if (hidden.requires_grad or weight.requires_grad) and torch.is_grad_enabled():
        raise CmsdError("lmhead_loss records nothing for autograd: call it under torch.no_grad() (or from an "
                        "autograd.Function) and take the gradients from lmhead_loss_backward")
    R, d, V = _head_sizes(hidden, weight)
    ignore_index = _ignored(ignore_index)
    f32, bf16 = torch.float32, torch.bfloat16
    loss, lse = _given(out, "loss", (R,), f32, hidden), _given(out, "lse", (R,), f32, hidden)
    cur = _current(hidden)
    _need(cur, ((hidden, (R, d), bf16, "hidden"), (weight, (V, d), bf16, "weight"),
                (labels, (R,), torch.int32, "labels"), (loss, (R,), f32, "loss"), (lse, (R,), f32, "lse")))
    ws = ws if ws is not None else lmhead_loss_workspace(R, d, V)
    rc = lib().cmsd_lmhead_loss(hidden.data_ptr(), weight.data_ptr(), labels.data_ptr(), R, d, V, ignore_index,
                                loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), _need_ws(ws, cur), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_lmhead_loss")
    return {"loss": loss, "lse": lse}


def lmhead_loss_backward(hidden, weight, labels, lse, grad_loss, ignore_index=-100, hidden_grad=True,
                         weight_grad=True, out=None, ws=None):
    """The gradients of lmhead_loss: lse is its output, grad_loss (float32 [R]) is dL/dloss.

    Returns dict d_hidden (bf16 [R, d], with hidden_grad) and d_weight (bf16
    [V, d], with weight_grad), written whole."""
    torch = _torch()
    R, d, V = _head_sizes(hidden, weight)
    ignore_index = _ignored(ignore_index)
    f32, bf16 = torch.float32, torch.bfloat16
    o = {}
    specs = [(hidden, (R, d), bf16, "hidden"), (weight, (V, d), bf16, "weight"),
             (labels, (R,), torch.int32, "labels"), (lse, (R,), f32, "lse"), (grad_loss, (R,), f32, "grad_loss")]
    if hidden_grad:
        o["d_hidden"] = _given(out, "d_hidden", (R, d), bf16, hidden)
        specs.append((o["d_hidden"], (R, d), bf16, "d_hidden"))
    if weight_grad:
        o["d_weight"] = _given(out, "d_weight", (V, d), bf16, hidden)
        specs.append((o["d_weight"], (V, d), bf16, "d_weight"))
    cur = _current(hidden)
    _need(cur, specs)
    ws = ws if ws is not None else lmhead_loss_backward_workspace(R, d, V)
    rc = lib().cmsd_lmhead_loss_backward(hidden.data_ptr(), weight.data_ptr(), labels.data_ptr(), lse.data_ptr(),
                                         grad_loss.data_ptr(), R, d, V, ignore_index, _ptr(o.get("d_hidden")),
                                         _ptr(o.get("d_weight")), ws.data_ptr(), _need_ws(ws, cur), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_lmhead_loss_backward")
    return o


def quantize_rows(x, out=None):
    """Rows of x ([R, d], float32 or bfloat16) as symmetric 8-bit integers: dict q (int8 [R, d]) and
    scale (float32 [R], the row's largest magnitude over 127)."""
    torch = _torch()
    if x.dim() != 2:
        raise CmsdError("x must be [R, d]")
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise CmsdError(f"x must be float32 or bfloat16, got {x.dtype}")
    R, d = x.shape
    if R > _INT_MAX or d > _INT_MAX:
        _too_large("x [R, d]")
    q, scale = _given(out, "q", (R, d), torch.int8, x), _given(out, "scale", (R,), torch.float32, x)
    cur = _current(x)
    _need(cur, ((x, (R, d), x.dtype, "x"), (q, (R, d), torch.int8, "q"), (scale, (R,), torch.float32, "scale")))
    rc = lib().cmsd_quantize_rows(x.data_ptr(), F32 if x.dtype is torch.float32 else BF16, R, d, q.data_ptr(),
                                  scale.data_ptr(), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_quantize_rows")
    return {"q": q, "scale": scale}


def lmhead_i8(hidden_q, hidden_scale, weight_q, weight_scale, dtype=None, out=None, ws=None):
    """The logits of a head in 8-bit integers: hidden_q int8 [R, d] with a scale for each token, weight_q
    int8 [V, d] with one for each vocabulary entry (quantize_rows makes both).  Returns dict logits
    ([R, V], dtype float32 or bfloat16 (the default))."""
    torch = _torch()
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise CmsdError(f"logits are float32 or bfloat16, not {dtype}")
    R, d, V = _head_sizes(hidden_q, weight_q)
    f32, i8 = torch.float32, torch.int8
    logits = _given(out, "logits", (R, V), dtype, hidden_q)
    cur = _current(hidden_q)
    _need(cur, ((hidden_q, (R, d), i8, "hidden_q"), (hidden_scale, (R,), f32, "hidden_scale"),
                (weight_q, (V, d), i8, "weight_q"), (weight_scale, (V,), f32, "weight_scale"),
                (logits, (R, V), dtype, "logits")))
    ws = ws if ws is not None else lmhead_i8_workspace(R, d, V)
    rc = lib().cmsd_lmhead_i8(hidden_q.data_ptr(), hidden_scale.data_ptr(), weight_q.data_ptr(), weight_scale.data_ptr(),
                              R, d, V, logits.data_ptr(), F32 if dtype is f32 else BF16, ws.data_ptr(),
                              _need_ws(ws, cur), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_lmhead_i8")
    return {"logits": logits}


def _code(t, name):
    torch = _torch_mod
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise CmsdError(f"{name} must be float32 or bfloat16, got {t.dtype}")


def _unfollowed(what, *tensors):
    """Refuses a call where autograd would follow one of the tensors: nothing is recorded, and no tangent goes on."""
    if _torch_mod.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                how = (" that is differentiated once)" if what.endswith("_backward")
                       else f") and take the gradients from {what}_backward")
                raise CmsdError(f"{what} records nothing for autograd: call it under torch.no_grad() (or from an "
                                f"autograd.Function{how}")
    if _forward_ad._current_level >= 0 and _torch_mod._C._is_fwd_grad_enabled():
        for t in tensors:
            if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
                raise CmsdError(f"{what} passes no tangent on to autograd: call it on tensors without one (or from an "
                                f"autograd.Function with a jvp of its own)")


def _rows(t, name):
    shape = t.shape
    if len(shape) != 2:
        raise CmsdError(f"{name} must have two dimensions, got {tuple(shape)}")
    n, d = shape
    if n > _INT_MAX or d > _INT_MAX:
        _too_large(name)
    return n, d


def _fits(t, shape, dtype, cur):
    """What _need asks of one tensor."""
    return (t is not None and t.dtype is dtype and t.shape == shape and t.get_device() == cur >= 0
            and t.is_contiguous())


def _here(t, cur):
    """The same of a tensor that shapes and types are taken from."""
    return t.get_device() == cur >= 0 and t.is_contiguous()


def _result(out, name, shape, dtype, like, cur):
    """out's tensor of that name, which must fit, or a new one."""
    if out is not None and name in out:
        t = out[name]
        if not _fits(t, shape, dtype, cur):
            _need(cur, ((t, shape, dtype, name),))
        return t
    return _torch_mod.empty(shape, dtype=dtype, device=like.device)


def embedding(tokens, table, scale=1.0, ignore_index=-100, out=None):
    """Rows of the token table (float32 or bfloat16 [V, d]), scaled: returns dict x ([R, d], table's dtype; 0 in
    rows whose token is ignore_index).

    tokens: int32 [R].  Nothing is recorded for autograd: a table that requires gradients is refused while it
    records, and one with a tangent.  Another token outside the vocabulary gives a row of zeros; embedding_errors tells."""
    torch = _torch()
    _unfollowed("embedding", table)
    V, d = _rows(table, "table")
    code, dtype = _code(table, "table"), table.dtype
    R = tokens.numel()
    if R > _INT_MAX:
        _too_large("tokens [R]")
    ignore_index = _ignored(ignore_index)
    cur = _current(table)
    if not (_fits(tokens, (R,), torch.int32, cur) and _here(table, cur)):
        _need(cur, ((tokens, (R,), torch.int32, "tokens"), (table, (V, d), dtype, "table")))
    x = _result(out, "x", (R, d), dtype, table, cur)
    rc = lib().cmsd_embedding(tokens.data_ptr(), table.data_ptr(), code, R, d, V, ignore_index, float(scale), x.data_ptr(),
                              _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_embedding")
    return {"x": x}


def embedding_backward_workspace(R, d, V):
    """A workspace for embedding_backward of R rows or fewer on the current device (workspace_errors reads its error
    word)."""
    return _head_workspace("cmsd_embedding_backward_workspace_bytes", R, d, V)


def embedding_backward(tokens, d_x, V, scale=1.0, ignore_index=-100, add=False, out=None, ws=None):
    """The table's gradient, scale times the sum of each token's rows of d_x (float32 or bfloat16 [R, d]): returns
    dict d_table ([V, d], d_x's dtype), written whole.

    With add, out["d_table"] is given and the sums are added to it: a head that shares the table passes the d_weight
    of lmhead_loss_backward.  There are no second derivatives, here and in the gradients below: tensors that require
    them are refused while autograd records, and ones with a tangent."""
    torch = _torch()
    _unfollowed("embedding_backward", d_x, out.get("d_table") if add and out is not None else None)
    R, d = _rows(d_x, "d_x")
    V = int(V)
    if not 0 < V <= _INT_MAX:
        _too_large("V")
    code, dtype = _code(d_x, "d_x"), d_x.dtype
    ignore_index = _ignored(ignore_index)
    if add and (out is None or out.get("d_table") is None):
        raise CmsdError("add needs the d_table that is added to, in out")
    cur = _current(d_x)
    if not (_fits(tokens, (R,), torch.int32, cur) and _here(d_x, cur)):
        _need(cur, ((tokens, (R,), torch.int32, "tokens"), (d_x, (R, d), dtype, "d_x")))
    d_table = _result(out, "d_table", (V, d), dtype, d_x, cur)
    ws = ws if ws is not None else embedding_backward_workspace(R, d, V)
    rc = lib().cmsd_embedding_backward(tokens.data_ptr(), d_x.data_ptr(), code, R, d, V, ignore_index, float(scale),
                                       1 if add else 0, d_table.data_ptr(), ws.data_ptr(), _need_ws(ws, cur),
                                       _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_embedding_backward")
    return {"d_table": d_table}


def embedding_errors():
    """The error bits of the calls of embedding and embedding_backward on the current device since they were last
    read here (bit 0: a token that is neither in the vocabulary nor ignore_index).  Clears them and waits for the
    current stream."""
    f = ctypes.c_uint32(0)
    _torch()
    _check(lib().cmsd_embedding_errors(_stream(), ctypes.byref(f)), "cmsd_embedding_errors")
    return int(f.value)


def layernorm(x, weight=None, bias=None, eps=1e-5, stats=True, out=None):
    """Layer norm of the rows of x (float32 or bfloat16 [R, d]); weight and bias: float32 or bfloat16 [d], both of
    one dtype, or None (ones, zeros).

    Returns dict y ([R, d], x's dtype) and, with stats, mean and rstd (float32 [R]) for layernorm_backward.  Nothing
    is recorded for autograd: tensors that require gradients are refused while it records, and ones with
    a tangent."""
    torch = _torch()
    _unfollowed("layernorm", x, weight, bias)
    R, d = _rows(x, "x")
    code, dtype = _code(x, "x"), x.dtype
    wcode, wtype = code, dtype
    if weight is not None:
        wcode, wtype = _code(weight, "weight"), weight.dtype
    elif bias is not None:
        wcode, wtype = _code(bias, "bias"), bias.dtype
    cur = _current(x)
    if not (_here(x, cur) and (weight is None or _fits(weight, (d,), wtype, cur))
            and (bias is None or _fits(bias, (d,), wtype, cur))):
        _need(cur, ((x, (R, d), dtype, "x"),) + (((weight, (d,), wtype, "weight"),) if weight is not None else ())
              + (((bias, (d,), wtype, "bias"),) if bias is not None else ()))
    o = {"y": _result(out, "y", (R, d), dtype, x, cur)}
    mean = rstd = None
    if stats:
        o["mean"] = mean = _result(out, "mean", (R,), torch.float32, x, cur)
        o["rstd"] = rstd = _result(out, "rstd", (R,), torch.float32, x, cur)
    rc = lib().cmsd_layernorm(x.data_ptr(), _ptr(weight), _ptr(bias), code, wcode, R, d, float(eps), o["y"].data_ptr(),
                              _ptr(mean), _ptr(rstd), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_layernorm")
    return o


def layernorm_backward_workspace(R, d):
    """A workspace for layernorm_backward of R rows or fewer on the current device."""
    torch = _torch()
    if max(R, d) > _INT_MAX:
        _too_large("cmsd_layernorm_backward_workspace_bytes")
    n = int(lib().cmsd_layernorm_backward_workspace_bytes(int(R), int(d)))
    if n == 0:
        _too_large("cmsd_layernorm_backward_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def layernorm_backward(x, weight, mean, rstd, d_y, x_grad=True, weight_grad=True, bias_grad=True, out=None, ws=None,
                       dtype=None):
    """The gradients of layernorm: mean and rstd are its outputs, d_y ([R, d], x's dtype) is dL/dy, weight as there
    (None: ones).

    Returns dict d_x ([R, d], x's dtype, with x_grad), d_weight (with weight_grad) and d_bias (with bias_grad), both
    [d] of weight's dtype, written whole.  Without weight dtype says theirs (float32 or bfloat16, a bias's of its own;
    None: x's)."""
    torch = _torch()
    _unfollowed("layernorm_backward", x, weight, mean, rstd, d_y)
    R, d = _rows(x, "x")
    code, xtype = _code(x, "x"), x.dtype
    wcode, wtype = (code, xtype) if weight is None else (_code(weight, "weight"), weight.dtype)
    f32 = torch.float32
    if dtype is not None and dtype is not wtype:
        if weight is not None or dtype not in (f32, torch.bfloat16):
            raise CmsdError(f"dtype must be weight's, or float32 or bfloat16 without one, got {dtype}")
        wcode, wtype = F32 if dtype is f32 else BF16, dtype
    cur = _current(x)
    if not (_here(x, cur) and _fits(mean, (R,), f32, cur) and _fits(rstd, (R,), f32, cur)
            and _fits(d_y, (R, d), xtype, cur) and (weight is None or _fits(weight, (d,), wtype, cur))):
        _need(cur, ((x, (R, d), xtype, "x"), (mean, (R,), f32, "mean"), (rstd, (R,), f32, "rstd"),
                    (d_y, (R, d), xtype, "d_y")) + (((weight, (d,), wtype, "weight"),) if weight is not None else ()))
    o = {}
    if x_grad:
        o["d_x"] = _result(out, "d_x", (R, d), xtype, x, cur)
    if weight_grad:
        o["d_weight"] = _result(out, "d_weight", (d,), wtype, x, cur)
    if bias_grad:
        o["d_bias"] = _result(out, "d_bias", (d,), wtype, x, cur)
    ws = ws if ws is not None else layernorm_backward_workspace(R, d)
    rc = lib().cmsd_layernorm_backward(x.data_ptr(), _ptr(weight), mean.data_ptr(), rstd.data_ptr(), d_y.data_ptr(),
                                       code, wcode, R, d, _ptr(o.get("d_x")), _ptr(o.get("d_weight")),
                                       _ptr(o.get("d_bias")), ws.data_ptr(), _need_ws(ws, cur), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_layernorm_backward")
    return o


def _dropout_args(x, name, yname, iteration, site, step, out):
    code, dtype, shape = _code(x, name), x.dtype, x.shape
    iteration, site = int(iteration), int(site)
    if not (0 <= iteration < 1 << 32 and 0 <= site < 1 << 32):
        raise CmsdError("iteration and site must be 32-bit numbers that are not negative")
    cur = _current(x)
    if not _here(x, cur):
        _need(cur, ((x, shape, dtype, name),))
    if step is not None and not _fits(step, (1,), _torch_mod.int32, cur):
        _need(cur, ((step, (1,), _torch_mod.int32, "step"),))
    return code, cur, iteration, site, _result(out, yname, shape, dtype, x, cur)


def dropout(x, p, seed, iteration=0, site=0, residual=None, step=None, out=None):
    """Dropout with rate p (a multiple of 2^-16, the nearest one) and kept entries scaled up, residual added:
    returns dict y (x's shape and dtype, float32 or bfloat16).

    The mask is a function of seed (any integer, modulo 2^64), iteration (a training step), site (a layer) and an
    entry's place in x, and is not stored.  step: None, or an int32 [1] tensor that is added to iteration when the call runs (a captured call then
    draws another mask at each replay).  Nothing is recorded for autograd: tensors that require gradients are refused
    while it records, and ones with a tangent."""
    _torch()
    _unfollowed("dropout", x, residual)
    code, cur, iteration, site, y = _dropout_args(x, "x", "y", iteration, site, step, out)
    if residual is not None and not _fits(residual, x.shape, x.dtype, cur):
        _need(cur, ((residual, x.shape, x.dtype, "residual"),))
    rc = lib().cmsd_dropout(x.data_ptr(), _ptr(residual), code, x.numel(), float(p), int(seed), iteration, site, _ptr(step),
                            y.data_ptr(), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_dropout")
    return {"y": y}


def dropout_backward(d_y, p, seed, iteration=0, site=0, step=None, out=None):
    """The gradient of dropout by x, given the same p, seed, iteration, site and step: returns dict d_x.  (The
    residual's gradient is d_y itself.)"""
    _torch()
    _unfollowed("dropout_backward", d_y)
    code, cur, iteration, site, d_x = _dropout_args(d_y, "d_y", "d_x", iteration, site, step, out)
    rc = lib().cmsd_dropout_backward(d_y.data_ptr(), code, d_y.numel(), float(p), int(seed), iteration, site, _ptr(step),
                                     d_x.data_ptr(), _stream_of(cur))
    if rc != OK:
        _check(rc, "cmsd_dropout_backward")
    return {"d_x": d_x}


def verify(draft, target, tokens, conf, draft_lse=None, k_row=None, p=None, seed=0, iteration=0,
           out=None, ws=None):
    """Verification given conf (and draft_lse for the sampled rule); returns n_accept, out_tokens, accept."""
    torch = _torch()
    _need_cuda(draft, target, tokens, conf, draft_lse, k_row)
    B, K, V = draft.shape
    p = p if p is not None else params(K)
    _check_target(draft, target, p)
    dev = draft.device
    o = {"n_accept": _out(out, "n_accept", (B,), torch.int32, dev),
         "out_tokens": _out(out, "out_tokens", (B, K + 1 if p.bonus else K), torch.int32, dev),
         "accept": _out(out, "accept", (B, K), torch.uint8, dev)}
    ws = ws if ws is not None else workspace(B, K, V)
    rc = lib().cmsd_verify(_ptr(draft), _ptr(target), _ptr(tokens), _ptr(k_row), B, K, V,
                           _dtype_code(draft), ctypes.byref(p), _ptr(conf), _ptr(draft_lse),
                           int(seed), int(iteration), _ptr(o["n_accept"]), _ptr(o["out_tokens"]),
                           _ptr(o["accept"]), _ptr(ws), ws.numel(), _stream())
    _check(rc, "cmsd_verify")
    return o


def confidence_verify(draft, target, tokens, k_row=None, p=None, seed=0, iteration=0, out=None,
                      ws=None, signals=True):
    """The fused pass.  Returns n_accept, out_tokens, k_next, accept and (signals=True)
    H, margin, argmax, conf, lse."""
    torch = _torch()
    _need_cuda(draft, target, tokens, k_row)
    B, K, V = draft.shape
    p = p if p is not None else params(K)
    _check_target(draft, target, p)
    dev = draft.device
    o = {}
    for n in ("H", "margin", "conf", "lse"):
        o[n] = _out(out, n, (B, K), torch.float32, dev, signals)
    o["argmax"] = _out(out, "argmax", (B, K), torch.int32, dev, signals)
    o["k_next"] = _out(out, "k_next", (B,), torch.int32, dev)
    o["n_accept"] = _out(out, "n_accept", (B,), torch.int32, dev)
    o["out_tokens"] = _out(out, "out_tokens", (B, K + 1 if p.bonus else K), torch.int32, dev)
    o["accept"] = _out(out, "accept", (B, K), torch.uint8, dev, signals)
    ws = ws if ws is not None else workspace(B, K, V)
    rc = lib().cmsd_confidence_verify(
        _ptr(draft), _ptr(target), _ptr(tokens), _ptr(k_row), B, K, V, _dtype_code(draft),
        ctypes.byref(p), int(seed), int(iteration), _ptr(o["H"]), _ptr(o["margin"]), _ptr(o["argmax"]),
        _ptr(o["conf"]), _ptr(o["lse"]), _ptr(o["k_next"]), _ptr(o["n_accept"]), _ptr(o["out_tokens"]),
        _ptr(o["accept"]), _ptr(ws), ws.numel(), _stream())
    _check(rc, "cmsd_confidence_verify")
    return o


def confidence_verify_static(draft, target, tokens, k_row=None, p=None, seed=0, iteration=0, out=None,
                             signals=True):
    """The fused pass through cmsd_confidence_verify_static: the library's own
    fixed device scratch instead of a workspace (nothing is allocated for it).
    Output tensors are allocated here unless passed in `out`; a caller that may
    not allocate passes them all.  Calls on one device must not overlap."""
    torch = _torch()
    _need_cuda(draft, target, tokens, k_row)
    B, K, V = draft.shape
    p = p if p is not None else params(K)
    _check_target(draft, target, p)
    dev = draft.device
    o = {}
    for n in ("H", "margin", "conf", "lse"):
        o[n] = _out(out, n, (B, K), torch.float32, dev, signals)
    o["argmax"] = _out(out, "argmax", (B, K), torch.int32, dev, signals)
    o["k_next"] = _out(out, "k_next", (B,), torch.int32, dev)
    o["n_accept"] = _out(out, "n_accept", (B,), torch.int32, dev)
    o["out_tokens"] = _out(out, "out_tokens", (B, K + 1 if p.bonus else K), torch.int32, dev)
    o["accept"] = _out(out, "accept", (B, K), torch.uint8, dev, signals)
    rc = lib().cmsd_confidence_verify_static(
        _ptr(draft), _ptr(target), _ptr(tokens), _ptr(k_row), B, K, V, _dtype_code(draft),
        ctypes.byref(p), int(seed), int(iteration), _ptr(o["H"]), _ptr(o["margin"]), _ptr(o["argmax"]),
        _ptr(o["conf"]), _ptr(o["lse"]), _ptr(o["k_next"]), _ptr(o["n_accept"]), _ptr(o["out_tokens"]),
        _ptr(o["accept"]), _stream())
    _check(rc, "cmsd_confidence_verify_static")
    return o


def philox_u32(seed, c0, c1, c2, c3, word):
    return int(lib().cmsd_philox_u32(int(seed), c0, c1, c2, c3, int(word)))


def philox_fill(seed, c0, c1, c2, c3, n, device="cuda"):
    torch = _torch()
    out = torch.empty(n, dtype=torch.int32, device=device)
    _check(lib().cmsd_philox_fill(int(seed), c0, c1, c2, c3, _ptr(out), n, _stream()), "cmsd_philox_fill")
    return out


def profile_start(max_calls):
    _check(lib().cmsd_profile_start(int(max_calls)), "cmsd_profile_start")


def profile_stop(max_calls):
    """Per-call (streaming-kernel ms, resample-kernel ms) recorded since profile_start
    (the second is 0 for calls without a resample kernel)."""
    a = (ctypes.c_float * max(1, max_calls))()
    b = (ctypes.c_float * max(1, max_calls))()
    n = ctypes.c_int(0)
    _check(lib().cmsd_profile_stop(a, b, int(max_calls), ctypes.byref(n)), "cmsd_profile_stop")
    return [float(a[j]) for j in range(n.value)], [float(b[j]) for j in range(n.value)]


CONFIDENCE, VERIFY, FUSED = 0, 1, 2


def launch_plan(call, B, K, V, dtype, p, ragged=False):
    """What a call (CONFIDENCE, VERIFY or FUSED) of these sizes launches on the current device:
    (kernels, CTAs per sequence or 0 where the streaming kernel takes it, threads per CTA)."""
    n, c, t = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().cmsd_launch_plan(call, B, K, V, int(dtype), ctypes.byref(p), int(bool(ragged)), ctypes.byref(n),
                                  ctypes.byref(c), ctypes.byref(t)), "cmsd_launch_plan")
    return n.value, c.value, t.value


def launch_info(dtype=BF16):
    w, s = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().cmsd_launch_info(int(dtype), ctypes.byref(w), ctypes.byref(s)), "cmsd_launch_info")
    return w.value, s.value


def to_device_logits(arr, dtype, device="cuda"):
    """numpy logits (float32, or uint16 bfloat16 bit patterns) -> CUDA tensor."""
    torch = _torch()
    if dtype == "bf16":
        t = torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).view(torch.bfloat16)
    else:
        t = torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32))
    return t.to(device)


class FusedCall:
    """cmsd_confidence_verify with its arguments marshalled once.

    For tight loops (benchmarks, decode loops): calling the object re-issues
    the same C call on the current stream, optionally with another iteration
    number.  Holds references to every tensor it points at.
    """

    def __init__(self, draft, target, tokens, p, seed=0, iteration=0, k_row=None, out=None, ws=None,
                 signals=False):
        torch = _torch()
        _need_cuda(draft, target, tokens, k_row)
        B, K, V = draft.shape
        dev = draft.device
        o = dict(out or {})
        for n in ("H", "margin", "conf", "lse"):
            o.setdefault(n, torch.empty((B, K), dtype=torch.float32, device=dev) if signals else None)
        o.setdefault("argmax", torch.empty((B, K), dtype=torch.int32, device=dev) if signals else None)
        o.setdefault("accept", torch.empty((B, K), dtype=torch.uint8, device=dev) if signals else None)
        o.setdefault("k_next", torch.empty((B,), dtype=torch.int32, device=dev))
        o.setdefault("n_accept", torch.empty((B,), dtype=torch.int32, device=dev))
        o.setdefault("out_tokens", torch.empty((B, K + 1 if p.bonus else K), dtype=torch.int32, device=dev))
        self.out = o
        self.ws = ws if ws is not None else workspace(B, K, V)
        self._keep = (draft, target, tokens, k_row, p)
        self.p = p
        self.seed = int(seed)
        self.iteration = int(iteration)
        self._fn = lib().cmsd_confidence_verify
        self._head = (_ptr(draft), _ptr(target), _ptr(tokens), _ptr(k_row), B, K, V, _dtype_code(draft),
                      ctypes.byref(p))
        self._tail = (_ptr(o["H"]), _ptr(o["margin"]), _ptr(o["argmax"]), _ptr(o["conf"]), _ptr(o["lse"]),
                      _ptr(o["k_next"]), _ptr(o["n_accept"]), _ptr(o["out_tokens"]), _ptr(o["accept"]),
                      _ptr(self.ws), self.ws.numel())

    def __call__(self, iteration=None, stream=None):
        it = self.iteration if iteration is None else int(iteration)
        s = _stream() if stream is None else ctypes.c_void_p(stream)
        rc = self._fn(*self._head, self.seed, it, *self._tail, s)
        if rc != OK:
            _check(rc, "cmsd_confidence_verify")
        return self.out
