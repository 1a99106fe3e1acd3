"""Shared by the tests of the feed-forward operators: error bounds derived from
the arithmetic (U, E, TINY: block_util).

Products.  A sum of n products in float32 is within (n + 8) E of its terms'
absolute sum M, in any order.

Activations, act = g s(z).  z takes at most 4 roundings and the exponent's argument
two more: an error of 6 |z| E of the exponential, which s passes on at most whole;
the exponential, the sum, the reciprocal and the product add 2 + 1 + 2 + 1: act is
within (6 |z| + 6) E of its size.  Far out, |z| > 80, exponentials leave the range
of float32 or are held at exp(80): an absolute 2^-110 (1 + |g|) covers that.  act' =
s + g z' s (1 - s) is within (6 |z| + 12) E of the sum of its terms' sizes, |act'| is
at most 1.13, and its own slope at most 1.6.
"""

import numpy as np

from block_util import E, TINY, U
from parity_util import to64


def _z(g, kind):
    k = 2 * np.sqrt(2 / np.pi)
    return (g, np.ones_like(g)) if kind == "silu" else (k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g))


def _act_error(g, kind):
    """Relative error of act, the size of act' as the sum of its terms, and their relative error."""
    z, zd = _z(g, kind)
    far = np.minimum(np.abs(z), 100)
    s, c = np.exp(-np.logaddexp(0.0, -z)), np.exp(-np.logaddexp(0.0, z))
    return (6 * far + 6) * E, s + np.abs(g) * zd * s * c, (6 * far + 12) * E


def fwd_bounds(x, wg, wu, ref, kind, dtype):
    """Bounds of (h, gate, up) for the oracle's `ref`."""
    h, g, u = ref
    import oracle.ffn_oracle as orc
    acc = (x.shape[-1] + 8) * E
    eg, eu = acc * (np.abs(to64(x)) @ np.abs(to64(wg)).T), acc * (np.abs(to64(x)) @ np.abs(to64(wu)).T)
    act = np.abs(orc.activation(g, kind))
    rel, _, _ = _act_error(g, kind)
    e_act = 1.13 * eg + rel * act + 2.0 ** -110 * (1 + np.abs(g))
    eh = e_act * (np.abs(u) + eu) + act * eu + 2 * E * np.abs(h)
    return tuple(e + U[dtype] * (np.abs(v) + e) + TINY for e, v in ((eh, h), (eg, g), (eu, u)))


def bwd_bounds(x, wg, wu, gate, up, dh, ref, kind, dtype):
    """Bounds of (dx, dw_gate, dw_up) for given gate and up."""
    import oracle.ffn_oracle as orc
    x, wg, wu, g, u, dh = (to64(t) for t in (x, wg, wu, gate, up, dh))
    rel, size, rel_slope = _act_error(g, kind)
    act = np.abs(orc.activation(g, kind))
    floor = 2.0 ** -110 * (1 + np.abs(g))
    dg, du = np.abs(dh * u * orc.slope(g, kind)), np.abs(dh) * act
    eg = np.abs(dh * u) * ((rel_slope + 2 * E) * size + floor)
    eu = np.abs(dh) * ((rel + E) * act + floor)
    eg, eu = eg + U[dtype] * (dg + eg) + TINY, eu + U[dtype] * (du + eu) + TINY  # rounded: operands

    def product(a, ea, b):  # sum over the middle axis of a b, a off by ea
        return ea @ b + (a.shape[1] + 8) * E * ((a + ea) @ b)

    ax, ag, au = np.abs(x), np.abs(wg), np.abs(wu)
    F, T = wg.shape[0], x.shape[0]
    edx = eg @ ag + eu @ au + (2 * F + 8) * E * ((dg + eg) @ ag + (du + eu) @ au)
    out = []
    for e, v in zip((edx, product(dg.T, eg.T, ax), product(du.T, eu.T, ax)), ref):
        out.append(e + U[dtype] * (np.abs(v) + e) + TINY)
    return tuple(out)
