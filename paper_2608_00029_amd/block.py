"""Thin ctypes binding over the decoder-block operators of include/cattn.h:
RMSNorm with the residual added, rotary positions, sliding-window attention
with sinks.

As in binding.py this is argument marshalling only: tensors are checked, outputs
allocated with torch where the caller passes none, and device pointers, strides
and torch's current stream of the tensors' device handed to the library.  Tensors
of heads may be strided views (a row's columns consecutive); outputs that are
allocated here are contiguous.
"""

from __future__ import annotations

import ctypes
import functools
from typing import Optional

import torch

from .binding import (CATTN_BF16, CATTN_ERR_UNSUPPORTED, CATTN_F32, CATTN_OK, CattnError, _check_workspace, _dtype_code,
                      _LAYOUTS, _rows_cols, _stream, last_error_string, lib)

_F32, _F64, _I32 = torch.float32, torch.float64, torch.int32
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "ramp": 3}


# One expression decides; only then is it looked for what is wrong (binding.py).
def _plain(name, t, shape, dtype, device):
    """A contiguous tensor of this shape, type and device."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.device == device \
            and t.is_contiguous():
        return
    _refuse(name, t, shape, dtype, device)
    raise ValueError(f"{name} must be contiguous")


def _view(name, t, shape, dtype, device):
    """A tensor of this shape, type and device whose last dimension is consecutive."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.device == device \
            and (t.is_contiguous() or t.stride()[-1] == 1 or t.shape[-1] == 1):  # (stride(-1) takes three times that)
        return
    _refuse(name, t, shape, dtype, device)
    raise ValueError(f"the last dimension of {name} must be consecutive")


def _rows_consecutive(name, t):
    if not t.is_contiguous() and t.stride()[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"the last dimension of {name} must be consecutive")


def _refuse(name, t, shape, dtype, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")


def _on_hip(name, t):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a HIP device")


_get_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _run(where: str, device, *args):
    """Calls the library's `where` on torch's current stream of the tensors' device, which is made
    the current one for the call if it is not."""
    was = _get_device()
    if was == device.index:
        st = getattr(lib(), where)(*args, _stream(device))
    else:
        torch.cuda.set_device(device)
        try:
            st = getattr(lib(), where)(*args, _stream(device))
        finally:
            torch.cuda.set_device(was)
    if st != CATTN_OK:
        raise CattnError(st, where, last_error_string())


def _at(t) -> int:
    return 0 if t is None else t.data_ptr()


def _int(n) -> int:
    """n as a C int: what does not fit becomes the largest (or -1), which the library clamps or refuses.
    (ctypes would hand over its low 32 bits.)"""
    return n if -1 <= n <= 2147483647 else 2147483647 if n > 0 else -1


# Sizes (not negative) are all C ints iff none has a bit from 31 on: `(B | S | ...) >> 31` asks once for all.
def _too_large(where):
    raise CattnError(CATTN_ERR_UNSUPPORTED, where, "a size exceeds 2^31 - 1")


def _heads(name, t, layout):
    """(B, H, S, D) of a 4-d tensor of heads in `layout`."""
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be 'bhsd' or 'bshd', not {layout!r}")
    _on_hip(name, t)
    if t.dim() != 4:
        raise ValueError(f"{name} must be 4-d ({layout.upper()})")
    B, x, y, D = t.shape
    return (B, x, y, D) if layout == "bhsd" else (B, y, x, D)


def _shape(B, H, S, D, layout):
    return (B, H, S, D) if layout == "bhsd" else (B, S, H, D)


def _strides(tensors, layout) -> Optional[ctypes.Array]:
    """The strides argument: None where every tensor is contiguous, else three per tensor
    (batch, head, row).  A 3-d tensor is one row per head."""
    for t in tensors:
        if not t.is_contiguous():
            break
    else:
        return None
    out = []
    for t in tensors:
        s = t.stride()
        if len(s) == 3:
            out += (s[0], s[1], 0)
        elif layout == "bhsd":
            out += s[:3]
        else:
            out += (s[0], s[2], s[1])
    return (ctypes.c_longlong * len(out))(*out)


def _like(t):
    """A contiguous tensor of t's shape and type."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _batch(name, t, B, device):
    if t is not None:
        _plain(name, t, (B,), _I32, device)


# ---------------------------------------------------------------------------
# RMSNorm
# ---------------------------------------------------------------------------
# (empty_like costs less host time than new_empty, and that less than torch.empty with its keywords)
def _norm_inputs(where, x, gamma, residual):
    _on_hip("x", x)
    R, C = _rows_cols(x)
    if (R | C) >> 31:
        _too_large(where)
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    _plain("gamma", gamma, (C,), _F32, x.device)
    if residual is None:
        return R, C, None, gamma.new_empty(R), _dtype_code(x)
    _plain("residual", residual, x.shape, x.dtype, x.device)
    return R, C, torch.empty_like(x), gamma.new_empty(R), _dtype_code(x)


def rmsnorm_fwd(x, gamma, residual=None, eps: float = 1e-5):
    """(y, h, rstd): root-mean-square norm of h = x + residual over the last axis.

    x (and residual): float32 or bfloat16, contiguous; gamma: float32 [C].  h is
    x itself without a residual; rstd is float32 [rows].
    """
    R, C, h, rstd, code = _norm_inputs("cattn_rmsnorm_fwd", x, gamma, residual)
    y = torch.empty_like(x)
    _run("cattn_rmsnorm_fwd", x.device, _at(x), _at(residual), _at(gamma), _at(y), _at(h), _at(rstd), R, C, eps, code)
    return y, x if h is None else h, rstd


def rmsnorm_fwd_q8(x, gamma, residual=None, eps: float = 1e-5, group: int = 0):
    """(q, scale, h, rstd): rmsnorm_fwd with y in 8 bits, y ~ q * scale.

    q is float8_e4m3fn of x's shape; scale float32 [rows, ceil(C / group)], one per
    `group` consecutive columns (a power of two from 8 to 512), or one per row for 0.
    """
    R, C, h, rstd, code = _norm_inputs("cattn_rmsnorm_fwd_q8", x, gamma, residual)
    if not isinstance(group, int) or (group and (group < 8 or group > 512 or group & (group - 1))):
        raise ValueError("group must be 0 or a power of two from 8 to 512")
    q = torch.empty_like(x, dtype=torch.float8_e4m3fn)
    scale = gamma.new_empty((R, -(-C // group) if group else 1))
    _run("cattn_rmsnorm_fwd_q8", x.device, _at(x), _at(residual), _at(gamma), _at(q), _at(scale), _at(h), _at(rstd),
         R, C, group, eps, code)
    return q, scale, x if h is None else h, rstd


@functools.lru_cache(maxsize=256)  # (a call into the library each time costs 1 us)
def rmsnorm_bwd_workspace_bytes(rows: int, C: int) -> int:
    return int(lib().cattn_rmsnorm_bwd_workspace_bytes(_int(rows), _int(C)))


def rmsnorm_bwd(h, gamma, rstd, dy, dh=None, workspace=None):
    """(dx, dgamma) of rmsnorm_fwd for upstream dy, given its h and rstd.

    dh: the gradient that reaches h beside the norm (the residual stream's), added
    to dx; dx is the gradient of x and of the residual.  dgamma is float32.
    """
    _on_hip("h", h)
    R, C = _rows_cols(h)
    if (R | C) >> 31:
        _too_large("cattn_rmsnorm_bwd")
    code = _dtype_code(h)
    if not h.is_contiguous():
        raise ValueError("h must be contiguous")
    _plain("gamma", gamma, (C,), _F32, h.device)
    _plain("rstd", rstd, (R,), _F32, h.device)
    _plain("dy", dy, h.shape, h.dtype, h.device)
    if dh is not None:
        _plain("dh", dh, h.shape, h.dtype, h.device)
    dx = torch.empty_like(h)
    dgamma = torch.empty_like(gamma) if R else torch.zeros_like(gamma)  # (no rows: a sum over nothing)
    n = rmsnorm_bwd_workspace_bytes(R, C) // 4
    if workspace is None:
        workspace = gamma.new_empty(n)
    else:
        _check_workspace(workspace, n, h.device)
    _run("cattn_rmsnorm_bwd", h.device, _at(h), _at(gamma), _at(rstd), _at(dy), _at(dh), _at(dx), _at(dgamma),
         _at(workspace), R, C, code)
    return dx, dgamma


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
def rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     context: float = 0.0, low: float = 1.0, high: float = 32.0, device=None):
    """float64 [rot / 2]: radians per position of each rotated pair, the `freqs` of rope_fwd.

    scaling: "none"; "linear" (divided by factor); "ntk" (a larger base); "ramp" (by the
    turns a pair makes in `context` positions: kept from `high` on, divided by factor
    up to `low`, between them linearly).
    """
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_SCALINGS)}, not {scaling!r}")
    rot = int(rot)
    if rot > 2147483647:
        _too_large("cattn_rope_frequencies")
    out = (ctypes.c_double * max(1, rot // 2))()
    st = lib().cattn_rope_frequencies(out, rot, base, _SCALINGS[scaling], factor, context, low, high)
    if st != CATTN_OK:
        raise CattnError(st, "cattn_rope_frequencies", last_error_string())
    return torch.tensor(list(out), dtype=_F64, device=device)


def _rope(q, k, freqs, positions, layout, interleaved, amplitude, q_out, k_out, inverse):
    B, Hq, S, D = _heads("q", q, layout)
    code = _dtype_code(q)
    dev = q.device
    _rows_consecutive("q", q)
    Hkv = 0
    if k is not None:
        Hkv = _heads("k", k, layout)[1]
        _view("k", k, _shape(B, Hkv, S, D, layout), q.dtype, dev)
    elif k_out is not None:
        raise ValueError("k_out without k")
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1:
        raise TypeError("freqs must be a 1-d float64 tensor (rope_frequencies)")
    _plain("freqs", freqs, freqs.shape, _F64, dev)
    rot = 2 * freqs.shape[0]
    if (B | Hq | Hkv | S | D | rot) >> 31:
        _too_large("cattn_rope")
    batched = 0
    if positions is not None:
        batched = int(isinstance(positions, torch.Tensor) and positions.dim() == 2)
        _plain("positions", positions, (B, S) if batched else (S,), _I32, dev)
    if q_out is None:
        q_out = _like(q)
    else:
        _view("q_out", q_out, q.shape, q.dtype, dev)
    if k is not None:
        if k_out is None:
            k_out = _like(k)
        else:
            _view("k_out", k_out, k.shape, q.dtype, dev)
    strides = _strides((q, k, q_out, k_out) if k is not None else (q, q, q_out, q_out), layout)
    _run("cattn_rope", dev, _at(q), _at(k), _at(q_out), _at(k_out), _at(positions), _at(freqs), B, S, Hq, Hkv, D, rot,
         batched, strides, _LAYOUTS[layout], bool(interleaved), inverse, amplitude, code)
    return q_out, k_out


def rope_fwd(q, k, freqs, positions=None, layout: str = "bhsd", interleaved: bool = False, amplitude: float = 1.0,
             q_out=None, k_out=None):
    """(q', k'): queries and keys turned by their positions' angles.

    q [B, Hq, S, D] and k [B, Hkv, S, D] (or [B, S, H, D] for "bshd"; k may be None),
    float32 or bfloat16, possibly strided.  The first 2 * len(freqs) columns of a
    head are rotated, the others copied.  positions: int32 [B, S] or [S], or None for
    0 .. S - 1.  q_out / k_out may be q / k themselves: in place.
    """
    return _rope(q, k, freqs, positions, layout, interleaved, amplitude, q_out, k_out, 0)


def rope_bwd(dq, dk, freqs, positions=None, layout: str = "bhsd", interleaved: bool = False, amplitude: float = 1.0,
             dq_out=None, dk_out=None):
    """The gradients of rope_fwd's q and k for those of its results: turned back."""
    return _rope(dq, dk, freqs, positions, layout, interleaved, amplitude, dq_out, dk_out, 1)


def rope_append(q, k, v, k_cache, v_cache, lens, freqs, counts=None, window: int = 0, sinks: int = 0,
                rolling: bool = False, layout: str = "bhsd", interleaved: bool = False, amplitude: float = 1.0,
                q_out=None, k_out=None):
    """(q', k') as rope_fwd, with k' and v stored into the caches [B, Hkv, cap, D] in the same pass.

    lens: int32 [B], each sequence's tokens after the call; counts: int32 [B], how many
    of the S rows are its new tokens (None: all).  Row i is at position lens - counts +
    i; a row past counts, or at a negative position, gives 0 and is not stored.
    rolling: the cache holds the sinks and the last `window` positions.
    """
    B, Hq, S, D = _heads("q", q, layout)
    code = _dtype_code(q)
    dev, dt = q.device, q.dtype
    Hkv = _heads("k", k, layout)[1]
    cap = _heads("k_cache", k_cache, layout)[2]
    _rows_consecutive("q", q)
    _view("k", k, _shape(B, Hkv, S, D, layout), dt, dev)
    _view("v", v, k.shape, dt, dev)
    _view("k_cache", k_cache, _shape(B, Hkv, cap, D, layout), dt, dev)
    _view("v_cache", v_cache, k_cache.shape, dt, dev)
    _plain("lens", lens, (B,), _I32, dev)
    _batch("counts", counts, B, dev)
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1:
        raise TypeError("freqs must be a 1-d float64 tensor (rope_frequencies)")
    _plain("freqs", freqs, freqs.shape, _F64, dev)
    rot = 2 * freqs.shape[0]
    if (B | Hq | Hkv | S | D | rot | cap) >> 31:
        _too_large("cattn_rope_append")
    if q_out is None:
        q_out = _like(q)
    else:
        _view("q_out", q_out, q.shape, dt, dev)
    if k_out is None:
        k_out = _like(k)
    else:
        _view("k_out", k_out, k.shape, dt, dev)
    strides = _strides((q, k, v, q_out, k_out, k_cache, v_cache), layout)
    _run("cattn_rope_append", dev, _at(q), _at(k), _at(v), _at(q_out), _at(k_out), _at(k_cache), _at(v_cache),
         _at(lens), _at(counts), _at(freqs), B, S, Hq, Hkv, D, rot, cap, _int(window), _int(sinks),
         bool(rolling), strides, _LAYOUTS[layout], bool(interleaved), amplitude, code)
    return q_out, k_out


# ---------------------------------------------------------------------------
# Sliding-window attention with sinks
# ---------------------------------------------------------------------------
def swa_fwd(q, k, v, scale: float, window: int, sinks: int = 0, lens=None, layout: str = "bhsd", o=None, lse=None):
    """O, LSE of causal attention in which query i sees key j iff i - j < window or j < sinks.

    q [B, Hq, S, D]; k, v [B, Hkv, S, D] (or [B, S, H, D] for "bshd"), Hq a multiple of
    Hkv, float32 or bfloat16, possibly strided.  LSE: float32 [B, Hq, S].  lens: int32
    [B] or None, the tokens of each sequence; rows from there on are padding: not
    read, O 0, LSE -inf.
    """
    B, Hq, S, D = _heads("q", q, layout)
    code = _dtype_code(q)
    dev, dt = q.device, q.dtype
    Hkv = _heads("k", k, layout)[1]
    _rows_consecutive("q", q)
    _view("k", k, _shape(B, Hkv, S, D, layout), dt, dev)
    _view("v", v, k.shape, dt, dev)
    _batch("lens", lens, B, dev)
    if (B | Hq | Hkv | S | D) >> 31:
        _too_large("cattn_swa_fwd")
    if o is None:
        o = _like(q)
    else:
        _view("o", o, q.shape, dt, dev)
    if lse is None:
        lse = q.new_empty((B, Hq, S), dtype=_F32)
    else:
        _plain("lse", lse, (B, Hq, S), _F32, dev)
    _run("cattn_swa_fwd", dev, _at(q), _at(k), _at(v), _at(o), _at(lse), _at(lens), B, Hq, Hkv, S, D, _int(window),
         _int(sinks), scale, _strides((q, k, v, o), layout), _LAYOUTS[layout], code)
    return o, lse


@functools.lru_cache(maxsize=256)
def swa_bwd_workspace_bytes(B: int, Hq: int, Hkv: int, S: int, D: int, window: int, sinks: int = 0) -> int:
    return int(lib().cattn_swa_bwd_workspace_bytes(*map(_int, (B, Hq, Hkv, S, D, window, sinks))))


def swa_bwd(q, k, v, o, do, lse, scale: float, window: int, sinks: int = 0, lens=None, layout: str = "bhsd",
            dq=None, dk=None, dv=None, workspace=None):
    """dQ, dK, dV of swa_fwd for upstream gradient `do`, given its O and LSE (and the same lens)."""
    B, Hq, S, D = _heads("q", q, layout)
    code = _dtype_code(q)
    dev, dt = q.device, q.dtype
    Hkv = _heads("k", k, layout)[1]
    kv = _shape(B, Hkv, S, D, layout)
    _rows_consecutive("q", q)
    for n, t, shape in (("k", k, kv), ("v", v, kv), ("o", o, q.shape), ("do", do, q.shape)):
        _view(n, t, shape, dt, dev)
    _plain("lse", lse, (B, Hq, S), _F32, dev)
    _batch("lens", lens, B, dev)
    if (B | Hq | Hkv | S | D) >> 31:
        _too_large("cattn_swa_bwd")
    for n, t, shape in (("dq", dq, q.shape), ("dk", dk, kv), ("dv", dv, kv)):
        if t is not None:
            _view(n, t, shape, dt, dev)
    dq = _like(q) if dq is None else dq
    dk = _like(k) if dk is None else dk
    dv = _like(v) if dv is None else dv
    n = swa_bwd_workspace_bytes(B, Hq, Hkv, S, D, window, sinks) // 4
    if workspace is None:
        workspace = lse.new_empty(n)
    else:
        _check_workspace(workspace, n, dev)
    _run("cattn_swa_bwd", dev, _at(q), _at(k), _at(v), _at(o), _at(do), _at(lse), _at(lens), _at(dq), _at(dk), _at(dv),
         _at(workspace), B, Hq, Hkv, S, D, _int(window), _int(sinks), scale,
         _strides((q, k, v, o, do, dq, dk, dv), layout), _LAYOUTS[layout], code)
    return dq, dk, dv


@functools.lru_cache(maxsize=256)
def swa_decode_workspace_bytes(B: int, Hq: int, Hkv: int, cap: int, D: int, window: int, sinks: int = 0,
                               dtype: Optional[torch.dtype] = None) -> int:
    """Bytes of swa_decode's workspace; without a dtype what either takes."""
    sizes = tuple(map(_int, (B, Hq, Hkv, cap, D, window, sinks)))
    codes = {torch.float32: (CATTN_F32,), torch.bfloat16: (CATTN_BF16,)}.get(dtype, (CATTN_F32, CATTN_BF16))
    return max(int(lib().cattn_swa_decode_workspace_bytes(*sizes, code)) for code in codes)


def swa_decode(q, k_cache, v_cache, lens, scale: float, window: int, sinks: int = 0, rolling: bool = False,
               layout: str = "bhsd", o=None, lse=None, workspace=None):
    """O [B, Hq, D], LSE [B, Hq] of one query per sequence, its newest token, over its cache.

    q [B, Hq, D], possibly strided; k_cache, v_cache [B, Hkv, cap, D] (or [B, cap, Hkv,
    D] for "bshd") hold the sequence's lens[b] tokens, the newest included, as
    rope_append leaves them with the same window, sinks and rolling.  A sequence
    without tokens gives 0 and -inf.
    """
    _on_hip("q", q)
    if q.dim() != 3:
        raise ValueError("q must be 3-d [B, Hq, D]")
    B, Hq, D = q.shape
    code = _dtype_code(q)
    dev, dt = q.device, q.dtype
    _, Hkv, cap, _ = _heads("k_cache", k_cache, layout)
    _rows_consecutive("q", q)
    _view("k_cache", k_cache, _shape(B, Hkv, cap, D, layout), dt, dev)
    _view("v_cache", v_cache, k_cache.shape, dt, dev)
    _plain("lens", lens, (B,), _I32, dev)
    if (B | Hq | Hkv | cap | D) >> 31:
        _too_large("cattn_swa_decode")
    if o is None:
        o = _like(q)
    else:
        _view("o", o, q.shape, dt, dev)
    if lse is None:
        lse = q.new_empty((B, Hq), dtype=_F32)
    else:
        _plain("lse", lse, (B, Hq), _F32, dev)
    n = swa_decode_workspace_bytes(B, Hq, Hkv, cap, D, window, sinks, dt) // 4
    if workspace is None:
        workspace = lse.new_empty(n) if n else None
    else:
        _check_workspace(workspace, n, dev)
    _run("cattn_swa_decode", dev, _at(q), _at(k_cache), _at(v_cache), _at(o), _at(lse), _at(lens), _at(workspace), B,
         Hq, Hkv, cap, D, _int(window), _int(sinks), bool(rolling), scale,
         _strides((q, k_cache, v_cache, o), layout), _LAYOUTS[layout], code)
    return o, lse
