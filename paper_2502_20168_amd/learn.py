"""Python binding of include/ssm_learn.h: what a learner runs next to the sequence layer.

Like binding.py it marshals arguments and nothing else: every function has the name of the C entry point it calls, tensors live on the
GPU, errors of the library raise SsmError, and there is no fallback.  Activations are float32, bfloat16 or float16 (one type per
call), channels adjacent, sequences and steps at any distance: views of a larger product and time-major arrays are taken as they are.
"""
from __future__ import annotations

import ctypes
from typing import Dict, List, Optional, Sequence, Tuple

from .binding import (SSM_ERR_INVALID_ARG, SSM_ERR_UNSUPPORTED, SSM_ERR_WORKSPACE, SSM_OK, SsmError, _chk, _chk_workspace, _done, _GeneralPathOnly, _handle, _own_workspace,
                      _ptr, _stream, _torch, lib, ssm_workspace_status)

__all__ = ["ssm_gated_carry_rows", "ssm_gated_workspace_bytes", "ssm_gated_scan_fwd", "ssm_gated_scan_bwd", "ssm_gated_step",
           "ssm_policy_loss_workspace_bytes", "ssm_policy_loss_fwd", "ssm_policy_loss_bwd", "ssm_policy_loss_grad",
           "ssm_adamw_state", "ssm_adamw_step", "ssm_adamw_values", "ssm_workspace_status", "SsmError",
           "SSM_OK", "SSM_ERR_INVALID_ARG", "SSM_ERR_WORKSPACE", "SSM_ERR_UNSUPPORTED"]

EXPORTS = ("ssm_gated_carry_rows", "ssm_gated_workspace_bytes", "ssm_gated_scan_fwd", "ssm_gated_scan_bwd", "ssm_gated_step",
           "ssm_policy_loss_workspace_bytes", "ssm_policy_loss_fwd", "ssm_policy_loss_bwd", "ssm_policy_loss_grad",
           "ssm_adamw_step", "ssm_adamw_values")

SSM_GATED_CARRY_STEPS = 128
SSM_ADAMW_BLOCK = 256

_vp, _i64, _sz, _int, _f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int, ctypes.c_float


class _Strides(ctypes.Structure):
    _fields_ = [("seq", _i64), ("step", _i64)]


class _Terms(ctypes.Structure):
    _fields_ = [("clip_low", _f), ("clip_high", _f), ("kl_coef", _f), ("entropy_coef", _f)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(k, _vp) for k in ("param", "grad", "m", "v", "m_scale", "v_scale")] + [("n", _i64)]


class _AdamwStored(ctypes.Structure):
    _fields_ = [(k, _vp) for k in ("m", "v", "m_scale", "v_scale", "m_out", "v_out")] + [("n", _i64)]


class _AdamwRates(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("step", _i64)]


_ready = None
_native = None


def _bind():
    """The native half (csrc/pybind_learn.cpp): it answers None for what it does not take, and the general path below follows."""
    global _native
    if _native is None:
        _lib()
        try:
            from . import _ssmlearn
            _native = _ssmlearn
        except ImportError as e:
            import warnings
            warnings.warn("the native half of the binding does not load (%s): run `python paper_2502_20168_amd/build.py`; calls go "
                          "through ctypes" % e, RuntimeWarning, stacklevel=3)
            _native = _GeneralPathOnly()
    return _native


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        row = [_vp, _i64, _vp, _vp, _vp, _vp, _vp, _Terms, _int, _i64, _i64]
        signatures = {
            "ssm_gated_carry_rows": (_i64, [_i64]),
            "ssm_gated_workspace_bytes": (_sz, [_i64] * 3 + [_int] * 2),
            "ssm_gated_scan_fwd": (_int, [_vp, _Strides, _vp, _Strides, _vp, _vp, _int, _int, _i64, _i64, _i64, _vp, _Strides, _vp, _vp,
                                          _vp, _sz, _vp]),
            "ssm_gated_scan_bwd": (_int, [_vp, _Strides, _vp, _Strides, _vp, _vp, _vp, _vp, _Strides, _vp, _int, _int, _i64, _i64, _i64,
                                          _vp, _Strides, _vp, _Strides, _vp, _vp, _sz, _vp]),
            "ssm_gated_step": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _int, _int, _i64, _i64, _vp, _vp, _vp]),
            "ssm_policy_loss_workspace_bytes": (_sz, [_i64, _i64]),
            "ssm_policy_loss_fwd": (_int, row + [_vp] * 4 + [_vp, _sz, _vp]),
            "ssm_policy_loss_bwd": (_int, row + [_vp] * 5 + [_i64, _vp]),
            "ssm_policy_loss_grad": (_int, row + [_vp] * 6 + [_i64, _vp, _sz, _vp]),
            "ssm_adamw_step": (_int, [_vp, _i64, _AdamwRates, _int, _int, _int, _vp, _vp, _vp]),
            "ssm_adamw_values": (_int, [_vp, _i64, _vp]),
        }
        for name, (res, args) in signatures.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _ready = L
    return _ready


def _dtype(t, name):
    torch = _torch()
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}.get(t.dtype)
    if code is None:
        raise ValueError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    return code


def _chk_rows(t, dtype, shape, name):
    """A cuda tensor of this type and shape whose last dimension is dense."""
    if t is None:
        return
    if not t.is_cuda or t.dtype != dtype or tuple(t.shape) != tuple(shape) or (shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s must be a cuda tensor of dtype %s and shape %s with a dense last dimension, got %s %s strides %s on %s"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape), tuple(t.stride()), t.device))


def _raise(rc, where):
    if rc != SSM_OK:
        raise SsmError(rc, where)



# ------------------------------------------------------------------ gated linear recurrence
def ssm_gated_carry_rows(L: int) -> int:
    return int(_lib().ssm_gated_carry_rows(L))


def ssm_gated_workspace_bytes(Bt: int, L: int, D: int, dtype, want_bwd: bool) -> int:
    """Scratch bytes of a call; 0 where it needs none."""
    torch = _torch()
    return int(_lib().ssm_gated_workspace_bytes(Bt, L, D, {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype], 1 if want_bwd else 0))


def _gated_workspace(given, Bt, L, D, dtype, want_bwd, device, stream):
    if given is not None:
        return _chk_workspace(given)
    n = ssm_gated_workspace_bytes(Bt, L, D, dtype, want_bwd)
    return _own_workspace(_torch().empty(n, dtype=_torch().uint8, device=device), stream) if n else None


def _strides(t):
    return _Strides(t.stride(0), t.stride(1))


def _check_gated(gate, u, is_first, h0):
    torch = _torch()
    if gate.dim() != 3:
        raise ValueError("gate must be [Bt,L,D]")
    Bt, L, D = gate.shape
    code = _dtype(gate, "gate")
    _chk_rows(gate, gate.dtype, (Bt, L, D), "gate")
    _chk_rows(u, gate.dtype, (Bt, L, D), "u")
    _chk(is_first, torch.uint8, (Bt, L), "is_first")
    _chk(h0, torch.float32, (Bt, D), "h0")
    return Bt, L, D, code


def _given(out, name, like=None, shape=None):
    """The caller's tensor of that name, or a new one: as `like` lies in memory (dense where that one overlaps itself), or float32 of `shape`."""
    torch = _torch()
    t = out.get(name) if out else None
    if t is not None:
        return t
    if shape is not None:
        return torch.empty(shape, dtype=torch.float32, device=like.device)
    t = torch.empty_like(like)
    return t if like.shape[-1] <= 1 or t.stride(-1) == 1 else torch.empty(like.shape, dtype=like.dtype, device=like.device)


def ssm_gated_scan_fwd(gate, u, is_first=None, h0=None, *, linear: bool = False, want_carry: bool = True, workspace=None, stream=None,
                       out: Optional[Dict] = None) -> Dict[str, object]:
    """h_t = [not first_t] f_t h_{t-1} + (1 - f_t) u_t with f = sigmoid(gate); linear: [not first_t] gate_t h_{t-1} + u_t.
    gate, u [Bt,L,D].  Returns dict(h [Bt,L,D], h_last [Bt,D] float32, carry for the gradient pass or None).  linear: a state that is not zero
    is lost (infinite, NaN or zero) where the product of the coefficients of consecutive steps leaves the range of float32."""
    r = (_native or _bind()).gated_scan_fwd(gate, u, is_first, h0, linear, want_carry, workspace, _handle(stream), out)
    if r is not None:
        return _done(r, "ssm_gated_scan_fwd")
    torch = _torch()
    Bt, L, D, code = _check_gated(gate, u, is_first, h0)
    rows = ssm_gated_carry_rows(L)
    h, h_last = _given(out, "h", u), _given(out, "h_last", u, (Bt, D))
    carry = _given(out, "carry", u, (Bt, rows, D)) if want_carry and rows else None
    _chk_rows(h, gate.dtype, (Bt, L, D), "h")
    _chk(h_last, torch.float32, (Bt, D), "h_last")
    _chk(carry, torch.float32, (Bt, rows, D), "carry")
    ws = _gated_workspace(workspace, Bt, L, D, gate.dtype, False, gate.device, stream)
    _raise(_lib().ssm_gated_scan_fwd(_ptr(gate), _strides(gate), _ptr(u), _strides(u), _ptr(is_first), _ptr(h0), code, int(bool(linear)),
                                     Bt, L, D, _ptr(h), _strides(h), _ptr(h_last), _ptr(carry), _ptr(ws), ws.numel() if ws is not None else 0,
                                     _stream(stream)), "ssm_gated_scan_fwd")
    return {"h": h, "h_last": h_last, "carry": carry}


def ssm_gated_scan_bwd(gate, u, is_first, h0, carry, dh, dh_last=None, *, linear: bool = False, want_dh0: bool = True, workspace=None,
                       stream=None, out: Optional[Dict] = None) -> Dict[str, object]:
    """Gradient pass of ssm_gated_scan_fwd (carry: its result) for sum(dh h) + sum(dh_last h_last).
    Returns dict(dgate, du [Bt,L,D], dh0 [Bt,D] float32 or None)."""
    r = (_native or _bind()).gated_scan_bwd(gate, u, is_first, h0, carry, dh, dh_last, linear, want_dh0, workspace, _handle(stream), out)
    if r is not None:
        return _done(r, "ssm_gated_scan_bwd")
    torch = _torch()
    Bt, L, D, code = _check_gated(gate, u, is_first, h0)
    rows = ssm_gated_carry_rows(L)
    if carry is None and rows:
        raise ValueError("carry must be that of the forward call (want_carry=True)")
    _chk(carry, torch.float32, (Bt, rows, D), "carry")
    _chk_rows(dh, gate.dtype, (Bt, L, D), "dh")
    _chk(dh_last, torch.float32, (Bt, D), "dh_last")
    dgate, du = _given(out, "dgate", gate), _given(out, "du", u)
    dh0 = _given(out, "dh0", u, (Bt, D)) if want_dh0 else None
    _chk_rows(dgate, gate.dtype, (Bt, L, D), "dgate")
    _chk_rows(du, gate.dtype, (Bt, L, D), "du")
    _chk(dh0, torch.float32, (Bt, D), "dh0")
    ws = _gated_workspace(workspace, Bt, L, D, gate.dtype, True, gate.device, stream)
    _raise(_lib().ssm_gated_scan_bwd(_ptr(gate), _strides(gate), _ptr(u), _strides(u), _ptr(is_first), _ptr(h0), _ptr(carry), _ptr(dh),
                                     _strides(dh), _ptr(dh_last), code, int(bool(linear)), Bt, L, D, _ptr(dgate), _strides(dgate), _ptr(du), _strides(du),
                                     _ptr(dh0), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)), "ssm_gated_scan_bwd")
    return {"dgate": dgate, "du": du, "dh0": dh0}


def ssm_gated_step(gate, u, h_prev=None, is_first=None, *, linear: bool = False, h=None, y=None, stream=None):
    """One step of Bt sequences: gate, u [Bt,D], h_prev [Bt,D] float32 or None.  Returns (y, h): the new state in the type of u and
    in float32 (h may be h_prev, which is then updated in place)."""
    r = (_native or _bind()).gated_step(gate, u, h_prev, is_first, linear, h, y, _handle(stream))
    if r is not None:
        return _done(r, "ssm_gated_step")
    torch = _torch()
    if gate.dim() != 2:
        raise ValueError("gate must be [Bt,D]")
    Bt, D = gate.shape
    code = _dtype(gate, "gate")
    _chk_rows(gate, gate.dtype, (Bt, D), "gate")
    _chk_rows(u, gate.dtype, (Bt, D), "u")
    _chk(h_prev, torch.float32, (Bt, D), "h_prev")
    _chk(is_first, torch.uint8, (Bt,), "is_first")
    _chk(h, torch.float32, (Bt, D), "h")
    _chk(y, gate.dtype, (Bt, D), "y")
    h = h if h is not None else torch.empty((Bt, D), dtype=torch.float32, device=gate.device)
    y = y if y is not None else torch.empty((Bt, D), dtype=gate.dtype, device=gate.device)
    _raise(_lib().ssm_gated_step(_ptr(gate), gate.stride(0), _ptr(u), u.stride(0), _ptr(h_prev), _ptr(is_first), code, int(bool(linear)), Bt, D,
                                 _ptr(h), _ptr(y), _stream(stream)), "ssm_gated_step")
    return y, h


# ------------------------------------------------------------------ clipped policy loss
def ssm_policy_loss_workspace_bytes(N: int, K: int) -> int:
    return int(_lib().ssm_policy_loss_workspace_bytes(N, K))


def _check_policy(logits, action, logp_old, advantage, weight, logp_ref):
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [N,K]")
    N, K = logits.shape
    code = _dtype(logits, "logits")
    _chk_rows(logits, logits.dtype, (N, K), "logits")
    _chk(action, torch.int64, (N,), "action")
    for name, t in (("logp_old", logp_old), ("advantage", advantage), ("weight", weight), ("logp_ref", logp_ref)):
        _chk(t, torch.float32, (N,), name)
    return N, K, code


def _policy_workspace(given, N, K, device, stream):
    if given is not None:
        return _chk_workspace(given)
    n = ssm_policy_loss_workspace_bytes(N, K)
    if n == 0:
        raise SsmError(SSM_ERR_UNSUPPORTED if N > 0 and K > 0 else SSM_ERR_INVALID_ARG, "ssm_policy_loss_workspace_bytes")
    return _own_workspace(_torch().empty(n, dtype=_torch().uint8, device=device), stream)


def _policy_outputs(logits, out):
    torch = _torch()
    N = logits.shape[0]
    res = {"loss": _given(out, "loss", logits, ()), "logp": _given(out, "logp", logits, (N,)),
           "entropy": _given(out, "entropy", logits, (N,)), "lse": _given(out, "lse", logits, (N,))}
    for name in ("logp", "entropy", "lse"):
        _chk(res[name], torch.float32, (N,), name)
    _chk(res["loss"], torch.float32, (), "loss")
    return res


def _check_dlogits(logits, dlogits, out):
    dlogits = _given(out, "dlogits", logits) if dlogits is None else dlogits
    _chk_rows(dlogits, logits.dtype, tuple(logits.shape), "dlogits")
    return dlogits


def ssm_policy_loss_fwd(logits, action, logp_old, advantage, weight=None, logp_ref=None, *, clip_low: float = 0.2, clip_high: float = 0.2,
                        kl_coef: float = 0.0, entropy_coef: float = 0.0, workspace=None, stream=None, out: Optional[Dict] = None) -> Dict[str, object]:
    """Clipped policy loss of N rows of logits [N,K].  Returns dict(loss [], logp, entropy, lse [N]), float32."""
    r = (_native or _bind()).policy_loss_fwd(logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef,
                                             workspace, _handle(stream), out)
    if r is not None:
        return _done(r, "ssm_policy_loss_fwd")
    N, K, code = _check_policy(logits, action, logp_old, advantage, weight, logp_ref)
    r = _policy_outputs(logits, out)
    ws = _policy_workspace(workspace, N, K, logits.device, stream)
    _raise(_lib().ssm_policy_loss_fwd(_ptr(logits), logits.stride(0), _ptr(action), _ptr(logp_old), _ptr(advantage), _ptr(weight), _ptr(logp_ref),
                                      _Terms(clip_low, clip_high, kl_coef, entropy_coef), code, N, K, _ptr(r["loss"]), _ptr(r["logp"]),
                                      _ptr(r["entropy"]), _ptr(r["lse"]), _ptr(ws), ws.numel(), _stream(stream)), "ssm_policy_loss_fwd")
    return r


def ssm_policy_loss_bwd(logits, action, logp_old, advantage, weight, logp_ref, logp, entropy, lse, dloss=None, *, clip_low: float = 0.2,
                        clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, dlogits=None, stream=None):
    """Gradient with respect to the logits, from the forward call's logp, entropy and lse; dloss: float32 scalar tensor or None for 1.
    Returns dlogits [N,K] in the type of the logits (`dlogits=logits` stores it over them)."""
    r = (_native or _bind()).policy_loss_bwd(logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef,
                                             logp, entropy, lse, dloss, dlogits, _handle(stream))
    if r is not None:
        return _done(r, "ssm_policy_loss_bwd")
    torch = _torch()
    N, K, code = _check_policy(logits, action, logp_old, advantage, weight, logp_ref)
    for name, t in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        _chk(t, torch.float32, (N,), name)
    _chk(dloss, torch.float32, () if dloss is None else tuple(dloss.shape) if dloss.numel() == 1 else (), "dloss")
    dlogits = _check_dlogits(logits, dlogits, None)
    _raise(_lib().ssm_policy_loss_bwd(_ptr(logits), logits.stride(0), _ptr(action), _ptr(logp_old), _ptr(advantage), _ptr(weight), _ptr(logp_ref),
                                      _Terms(clip_low, clip_high, kl_coef, entropy_coef), code, N, K, _ptr(logp), _ptr(entropy), _ptr(lse),
                                      _ptr(dloss), _ptr(dlogits), dlogits.stride(0), _stream(stream)), "ssm_policy_loss_bwd")
    return dlogits


def ssm_policy_loss_grad(logits, action, logp_old, advantage, weight=None, logp_ref=None, dloss=None, *, clip_low: float = 0.2,
                         clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, workspace=None, stream=None,
                         out: Optional[Dict] = None) -> Dict[str, object]:
    """Loss and gradient in one call: dict(loss, logp, entropy, lse, dlogits); out={"dlogits": logits} stores it over the logits."""
    r = (_native or _bind()).policy_loss_grad(logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef,
                                              dloss, workspace, _handle(stream), out)
    if r is not None:
        return _done(r, "ssm_policy_loss_grad")
    torch = _torch()
    N, K, code = _check_policy(logits, action, logp_old, advantage, weight, logp_ref)
    _chk(dloss, torch.float32, () if dloss is None else tuple(dloss.shape) if dloss.numel() == 1 else (), "dloss")
    r = _policy_outputs(logits, out)
    r["dlogits"] = _check_dlogits(logits, None, out)
    ws = _policy_workspace(workspace, N, K, logits.device, stream)
    _raise(_lib().ssm_policy_loss_grad(_ptr(logits), logits.stride(0), _ptr(action), _ptr(logp_old), _ptr(advantage), _ptr(weight), _ptr(logp_ref),
                                       _Terms(clip_low, clip_high, kl_coef, entropy_coef), code, N, K, _ptr(dloss), _ptr(r["loss"]), _ptr(r["logp"]),
                                       _ptr(r["entropy"]), _ptr(r["lse"]), _ptr(r["dlogits"]), r["dlogits"].stride(0), _ptr(ws), ws.numel(),
                                       _stream(stream)), "ssm_policy_loss_grad")
    return r


# ------------------------------------------------------------------ AdamW
def _blocks(n):
    return -(-n // SSM_ADAMW_BLOCK)


def ssm_adamw_state(params: Sequence, bits: int = 32) -> Dict[str, Optional[List]]:
    """The state of a new optimizer, all zero: dict(m, v, m_scale, v_scale) of lists, one tensor per parameter; bits 32: float32
    and no scales, bits 8: bytes and a float32 scale per SSM_ADAMW_BLOCK elements."""
    torch = _torch()
    if bits == 32:
        zero = lambda: [torch.zeros_like(p, dtype=torch.float32) for p in params]
        return {"m": zero(), "v": zero(), "m_scale": None, "v_scale": None}
    if bits != 8:
        raise ValueError("bits must be 8 or 32, got %r" % (bits,))
    code = lambda: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device) for p in params]
    scale = lambda: [torch.zeros(_blocks(p.numel()), dtype=torch.float32, device=p.device) for p in params]
    return {"m": code(), "v": code(), "m_scale": scale(), "v_scale": scale()}


def _same_length(params, **lists):
    for name, l in lists.items():
        if l is not None and len(l) != len(params):
            raise ValueError("%s must have one tensor per parameter (%d), got %d" % (name, len(params), len(l)))


def ssm_adamw_step(params: Sequence, grads: Sequence, m: Sequence, v: Sequence, m_scale: Optional[Sequence] = None,
                   v_scale: Optional[Sequence] = None, *, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                   weight_decay: float = 0.0, step: int, grad_scale=None, skip=None, stream=None) -> None:
    """One AdamW step over all tensors at once, in place.  params and grads: lists of contiguous tensors, each list of one type;
    m, v (and, where they are bytes, m_scale, v_scale) as ssm_adamw_state makes them; step counts from 1.  grad_scale and skip:
    float32 tensors of one element, read on the device: gradients are multiplied by the first, and nothing changes where the second is not zero."""
    r = (_native or _bind()).adamw_step(params, grads, m, v, m_scale, v_scale, lr, beta1, beta2, eps, weight_decay, step, grad_scale, skip,
                                        _handle(stream))
    if r is not None:
        _done(r, "ssm_adamw_step")
        return
    torch = _torch()
    if len(params) == 0:
        raise ValueError("params must hold at least one tensor")
    _same_length(params, grads=grads, m=m, v=v, m_scale=m_scale, v_scale=v_scale)
    eight = m[0].dtype == torch.uint8
    if eight and (m_scale is None or v_scale is None):
        raise ValueError("m_scale and v_scale must be given where m and v are bytes")
    pdt, gdt = params[0].dtype, grads[0].dtype
    codes = _dtype(params[0], "params[0]"), _dtype(grads[0], "grads[0]")
    state = torch.uint8 if eight else torch.float32
    rows = (_AdamwTensor * len(params))()
    for i, p in enumerate(params):
        shape = tuple(p.shape)
        _chk(p, pdt, shape, "params[%d]" % i)
        _chk(grads[i], gdt, shape, "grads[%d]" % i)
        _chk(m[i], state, shape, "m[%d]" % i)
        _chk(v[i], state, shape, "v[%d]" % i)
        if eight:
            _chk(m_scale[i], torch.float32, (_blocks(p.numel()),), "m_scale[%d]" % i)
            _chk(v_scale[i], torch.float32, (_blocks(p.numel()),), "v_scale[%d]" % i)
        rows[i] = _AdamwTensor(p.data_ptr(), grads[i].data_ptr(), m[i].data_ptr(), v[i].data_ptr(), m_scale[i].data_ptr() if eight else None,
                               v_scale[i].data_ptr() if eight else None, p.numel())
    for name, t in (("grad_scale", grad_scale), ("skip", skip)):
        _chk(t, torch.float32, () if t is None else tuple(t.shape) if t.numel() == 1 else (), name)
    _raise(_lib().ssm_adamw_step(rows, len(params), _AdamwRates(lr, beta1, beta2, eps, weight_decay, step), codes[0], codes[1], 8 if eight else 32,
                                 _ptr(grad_scale), _ptr(skip), _stream(stream)), "ssm_adamw_step")


def ssm_adamw_values(m: Sequence, v: Sequence, m_scale: Sequence, v_scale: Sequence, m_out: Optional[Sequence] = None,
                     v_out: Optional[Sequence] = None, *, stream=None) -> Tuple[Sequence, Sequence]:
    """What 8-bit states stand for, in float32: (list of m, list of v), into the given tensors or new ones."""
    torch = _torch()
    if len(m) == 0:
        raise ValueError("m must hold at least one tensor")
    m_out = [torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in m] if m_out is None else m_out
    v_out = [torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in m] if v_out is None else v_out
    r = (_native or _bind()).adamw_values(m, v, m_scale, v_scale, m_out, v_out, _handle(stream))
    if r is not None:
        _done(r, "ssm_adamw_values")
        return m_out, v_out
    _same_length(m, v=v, m_scale=m_scale, v_scale=v_scale, m_out=m_out, v_out=v_out)
    rows = (_AdamwStored * len(m))()
    for i, t in enumerate(m):
        shape = tuple(t.shape)
        _chk(t, torch.uint8, shape, "m[%d]" % i)
        _chk(v[i], torch.uint8, shape, "v[%d]" % i)
        for name, s in (("m_scale", m_scale), ("v_scale", v_scale)):
            _chk(s[i], torch.float32, (_blocks(t.numel()),), "%s[%d]" % (name, i))
        for name, s in (("m_out", m_out), ("v_out", v_out)):
            _chk(s[i], torch.float32, shape, "%s[%d]" % (name, i))
        rows[i] = _AdamwStored(t.data_ptr(), v[i].data_ptr(), m_scale[i].data_ptr(), v_scale[i].data_ptr(), m_out[i].data_ptr(),
                               v_out[i].data_ptr(), t.numel())
    _raise(_lib().ssm_adamw_values(rows, len(m), _stream(stream)), "ssm_adamw_values")
    return m_out, v_out
