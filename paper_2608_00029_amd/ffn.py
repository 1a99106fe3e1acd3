"""Thin ctypes binding over the feed-forward operators of include/cattn.h: the
gated projections and dropout with the residual added.

As in block.py this is argument marshalling only: tensors are checked, outputs
allocated with torch, and device pointers and torch's current stream of the
tensors' device handed to the library.
"""

from __future__ import annotations

import functools

import torch

from .binding import CATTN_BF16, CATTN_F32, _check_workspace, _dtype_code, _rows_cols, lib
from .block import _at, _int, _like, _on_hip, _plain, _run, _too_large

_ACTIVATIONS = {"silu": 0, "gelu": 1}
_CODES = {torch.float32: CATTN_F32, torch.bfloat16: CATTN_BF16}


# ---------------------------------------------------------------------------
# Gated projections
# ---------------------------------------------------------------------------
def _gated_inputs(where, x, w_gate, w_up, activation):
    """(T, C, F, activation's code, type's code)."""
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be 'silu' or 'gelu', not {activation!r}")
    _on_hip("x", x)
    T, C = _rows_cols(x)
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    code = _dtype_code(x)
    if not isinstance(w_gate, torch.Tensor) or w_gate.dim() != 2:
        raise TypeError("w_gate must be a 2-d tensor [F, C]")
    F = w_gate.shape[0]
    _plain("w_gate", w_gate, (F, C), x.dtype, x.device)
    _plain("w_up", w_up, (F, C), x.dtype, x.device)
    if (T | C | F) >> 31:
        _too_large(where)
    return T, C, F, _ACTIVATIONS[activation], code


def gated_fwd(x, w_gate, w_up, activation: str = "silu", save: bool = False):
    """(h, gate, up): h = act(x w_gate^T) * (x w_up^T) over the last axis of x.

    x [..., C]; w_gate, w_up [F, C]; h [..., F]; float32 or bfloat16, contiguous, from
    a 16-byte boundary on; C and F multiples of 8.
    activation: "silu", or "gelu" (the tanh form).  save: the two products are kept
    for gated_bwd; without it gate and up are None.
    """
    T, C, F, act, code = _gated_inputs("cattn_gated_fwd", x, w_gate, w_up, activation)
    shape = x.shape[:-1] + (F,)
    h = x.new_empty(shape) if C else x.new_zeros(shape)  # (no columns: a sum over nothing)
    gate, up = (_like(h), _like(h)) if save else (None, None)
    if save and not C:
        gate.zero_()
        up.zero_()
    _run("cattn_gated_fwd", x.device, _at(x), _at(w_gate), _at(w_up), _at(h), _at(gate), _at(up), T, C, F, act, code)
    return h, gate, up


class _UnsupportedType(TypeError, KeyError):  # (a KeyError too: callers may catch it as one)
    __str__ = Exception.__str__


@functools.lru_cache(maxsize=256)
def gated_bwd_workspace_bytes(T: int, C: int, F: int, dtype: torch.dtype = torch.float32) -> int:
    """Bytes of gated_bwd's workspace; 0 for sizes that it refuses."""
    if dtype not in _CODES:
        raise _UnsupportedType(f"unsupported dtype {dtype}: use float32 or bfloat16")
    return int(lib().cattn_gated_bwd_workspace_bytes(_int(T), _int(C), _int(F), _CODES[dtype]))


def gated_bwd(x, w_gate, w_up, gate, up, dh, activation: str = "silu", workspace=None):
    """(dx, dw_gate, dw_up) of gated_fwd for upstream dh, given its gate and up; tensors as there."""
    T, C, F, act, code = _gated_inputs("cattn_gated_bwd", x, w_gate, w_up, activation)
    shape = x.shape[:-1] + (F,)
    for name, t in (("gate", gate), ("up", up), ("dh", dh)):
        _plain(name, t, shape, x.dtype, x.device)
    make = torch.empty_like if T and F else torch.zeros_like  # (no rows, or no products: sums over nothing)
    dx, dw_gate, dw_up = make(x), make(w_gate), make(w_up)
    n = gated_bwd_workspace_bytes(T, C, F, x.dtype) // 4
    if workspace is None:
        workspace = x.new_empty(n, dtype=torch.float32)
    else:
        _check_workspace(workspace, n, x.device)
    _run("cattn_gated_bwd", x.device, _at(x), _at(w_gate), _at(w_up), _at(gate), _at(up), _at(dh), _at(dx), _at(dw_gate),
         _at(dw_up), _at(workspace), T, C, F, act, code)
    return dx, dw_gate, dw_up


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
def _dropout_numbers(seed, site, step, device):
    """(seed, site, step, address of the step's tensor)"""
    for name, v, bits in (("seed", seed, 64), ("site", site, 32)):
        if not isinstance(v, int) or v < 0 or v >> bits:
            raise ValueError(f"{name} must be an integer of {bits} bits")
    if isinstance(step, torch.Tensor):
        _plain("step", step, (1,), torch.int64, device)
        return seed, site, 0, step.data_ptr()
    if not isinstance(step, int) or step < 0 or step >> 64:
        raise ValueError("step must be an integer of 64 bits or an int64 tensor of one element")
    return seed, site, step, None


def dropout_fwd(x, p: float, seed: int, site: int = 0, step=0, residual=None, y=None):
    """y = residual + x / (1 - p) where kept, residual (or 0) elsewhere; no mask is stored.

    x (and residual, y): float32 or bfloat16, contiguous, any shape, from a 16-byte
    boundary on (a slice such as x[1:] may begin elsewhere: clone it).  An element's
    fate depends on seed, site, step and its index alone: dropout_bwd with the same
    ones drops the same.  site: which of the model's dropouts this is; step: an
    integer, or an int64 tensor [1] on x's device, which is read when the kernel
    runs (a captured graph whose step is advanced drops anew).  y may be x or
    residual: in place.
    """
    _on_hip("x", x)
    code = _dtype_code(x)
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    numbers = _dropout_numbers(seed, site, step, x.device)
    if residual is not None:
        _plain("residual", residual, x.shape, x.dtype, x.device)
    if y is None:
        y = torch.empty_like(x)
    else:
        _plain("y", y, x.shape, x.dtype, x.device)
    _run("cattn_dropout_fwd", x.device, _at(x), _at(residual), _at(y), x.numel(), p, *numbers, code)
    return y


def dropout_bwd(dy, p: float, seed: int, site: int = 0, step=0, dx=None):
    """dx of dropout_fwd's x for upstream dy, with its p, seed, site and step; dy itself is the residual's."""
    _on_hip("dy", dy)
    code = _dtype_code(dy)
    if not dy.is_contiguous():
        raise ValueError("dy must be contiguous")
    numbers = _dropout_numbers(seed, site, step, dy.device)
    if dx is None:
        dx = torch.empty_like(dy)
    else:
        _plain("dx", dx, dy.shape, dy.dtype, dy.device)
    _run("cattn_dropout_bwd", dy.device, _at(dy), _at(dx), dy.numel(), p, *numbers, code)
    return dx
