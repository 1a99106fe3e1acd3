"""Shared by the tests of the decoder-block operators: inputs, and error bounds
derived from the arithmetic.

U is the rounding of an output's type, half a step: 2^-8 relative for bfloat16,
2^-24 for float32; E = 2^-24 one float32 operation.  Bounds count the roundings:

RMSNorm.  A row's sum of squares adds at most 32 terms in a lane, 6 levels across
the wave, 16 waves: under 64 roundings of non-negative terms, so rstd is within
(64 / 2 + 4) E; y takes three products more.  64 E covers each.

Rotary positions.  The turns are exact to 2^-52 p f / 2 pi (double), their
fraction times two, at most 1, rounds by 2^-25, an angle error of pi 2^-25; sine
and cosine add two units of 2^-24 at most, the products and the sum three E more:
(3.2 + 2 + 3) E < 10 E of amplitude (|a| + |b|).

Attention.  As parity_util derives it, tau = 2 U + (n + D + 80) E + 2 eps_s of the
terms' absolute sum, n the keys (queries of the group) summed over; the 80 E are
the exponential (2 units) and its argument, whose size is under 64 for these
inputs, rounded.  (bfloat16 rounds P, or dS, and the result; for float32 U = E.)
"""

import numpy as np
import torch

from parity_util import to64

E = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = 2.0 ** -126


def randn(gen, *shape, dtype="f32", scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(TYPES[dtype])


def gen(seed):
    return torch.Generator().manual_seed(seed)


def within(name, got, ref, bound):
    """Every element within its bound; infinities and their signs equal; no NaN."""
    got, ref = to64(got), to64(ref)
    bound = np.broadcast_to(np.asarray(bound, dtype=np.float64), ref.shape)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert not np.isnan(got).any(), f"{name}: NaN"
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]) and not np.isinf(got[~inf]).any(), f"{name}: infinities differ"
    err = np.abs(np.where(inf, 0.0, got) - np.where(inf, 0.0, ref))
    over = err > np.where(inf, 0.0, bound)
    if over.any():
        at = np.unravel_index(int(np.argmax(np.where(over, err, -1.0))), err.shape)
        raise AssertionError(f"{name}: {over.sum()} elements off, worst at {at}: {got[at]!r} for {ref[at]!r}, "
                             f"error {err[at]:.3e} > {bound[at]:.3e}")


def swa_bounds(ref, q, k, v, do, scale, dtype, lse_err, rows):
    """Bounds of o, lse, dq, dk, dv from the oracle's term sums (`rows`: the most terms a sum adds)."""
    q, k, v = (np.nan_to_num(to64(t)) for t in (q, k, v))
    D = q.shape[-1]
    eps_s = scale * D * E * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    acc = (rows + D + 80) * E
    tau_o = 2 * U[dtype] + acc + 2 * eps_s
    out = {"o": tau_o * ref["m_o"] + (rows * np.abs(v).max() + 1) * TINY,
           "lse": eps_s + acc + 4 * E * np.abs(np.where(np.isinf(ref["lse"]), 0.0, ref["lse"]))}
    if do is not None:
        do = np.nan_to_num(to64(do))
        tau_b, tau_d = 2 * U[dtype] + acc + eps_s + lse_err, tau_o + D * E
        out["dv"] = tau_b * ref["m_dv"] + (rows * np.abs(do).max() + 1) * TINY
        out["dq"] = scale * (tau_b * ref["g_dq"] + tau_d * ref["h_dq"] + (rows * np.abs(k).max() + 1) * TINY)
        out["dk"] = scale * (tau_b * ref["g_dk"] + tau_d * ref["h_dk"] + (rows * np.abs(q).max() + 1) * TINY)
    return out
