"""Float64 definitions of the feed-forward operators: gated projections and
dropout with the residual added, with Philox-4x32-10 in Python integers' width.
Test infrastructure only: plain numpy, nothing shared with the HIP path.

These operators are not in the paper; their formulas are stated here.
"""

from __future__ import annotations

import numpy as np


def _f64(x):
    return np.asarray(x, dtype=np.float64)


# ---------------------------------------------------------------------------
# Gated projections
# ---------------------------------------------------------------------------
def activation(g, kind):
    """act(g): silu g / (1 + exp(-g)), gelu (tanh form) 0.5 g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3)))."""
    g = _f64(g)
    if kind == "silu":
        return g * np.exp(-np.logaddexp(0.0, -g))
    t = np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    return g * np.exp(-np.logaddexp(0.0, -2 * t))  # (1 + tanh t) / 2 = 1 / (1 + exp(-2 t)), without its cancellation


def slope(g, kind):
    """act'(g)"""
    g = _f64(g)
    z, zd = (g, 1.0) if kind == "silu" else (2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3),
                                             2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g * g))
    s, c = np.exp(-np.logaddexp(0.0, -z)), np.exp(-np.logaddexp(0.0, z))  # s(z), 1 - s(z)
    return s + g * s * c * zd


def gated_fwd(x, w_gate, w_up, kind="silu"):
    """(h, gate, up): gate = x w_gate^T, up = x w_up^T, h = act(gate) up."""
    gate, up = _f64(x) @ _f64(w_gate).T, _f64(x) @ _f64(w_up).T
    return activation(gate, kind) * up, gate, up


def gated_bwd(x, w_gate, w_up, gate, up, dh, kind="silu"):
    """(dx, dw_gate, dw_up) for given gate and up."""
    dg = _f64(dh) * _f64(up) * slope(gate, kind)
    du = _f64(dh) * activation(gate, kind)
    return dg @ _f64(w_gate) + du @ _f64(w_up), dg.T @ _f64(x), du.T @ _f64(x)


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
def philox(counter, key, rounds=10):
    """Philox-4x32: counter four, key two arrays (or numbers) of 32-bit values; four uint64 arrays of 32-bit words."""
    mask = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]),
             a & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keep(n, p, seed, site=0, step=0, first=0):
    """Which of the elements first .. first + n - 1 are kept (first a multiple of 4)."""
    i = np.arange(first // 4, (first + n + 3) // 4, dtype=np.uint64)
    like = np.zeros_like(i)
    step %= 1 << 64
    words = philox((i, like + np.uint64(site), like + np.uint64(step & 0xFFFFFFFF), like + np.uint64(step >> 32)),
                   (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack(np.broadcast_arrays(*words), 1).reshape(-1)[:n] >= np.uint64(round(p * 2.0 ** 32))


def dropout(x, p, seed, site=0, step=0, residual=None):
    x = _f64(x)
    keep = dropout_keep(x.size, p, seed, site, step).reshape(x.shape)
    y = np.where(keep, x / (1 - p), 0.0)
    return y if residual is None else y + _f64(residual)
