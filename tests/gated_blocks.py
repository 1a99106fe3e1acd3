"""Shared by the tests that have to see a lost piece of a long sum: errors of the gated projections' outputs by blocks of
32 x 32 elements, in the 2-norm, against what independent roundings leave.

For an output v = sum over n terms a_j b_j of independent inputs let S = sqrt(sum a_j^2 b_j^2), the size that such a sum has.
A partial sum of m terms has size S sqrt(m / n), each addition rounds by at most E of it, and norms add at most, so the n
additions leave at most n E S.  16 E more are the sum's other roundings.  The output is rounded by U |v|.

Backward.  The reference's dg and du are rounded to the type as the operands are (a rounding is not left to chance: where the
kernel's float value lies on the other side of a border, it differs by a step, 2 U).  A float value of dg is within (6 |z|
+ 15) E of its terms' sizes (ffn_util), for these inputs under 100 E, so that at most one element in 2^8 (bfloat16: a step
is 2^16 E) is near a border, typically one in 2^11: sqrt(2^-8) 2 U = U / 8 of the size S.  float32: 100 E S.

Forward.  gate and up: n E S and U.  h = act(g) u with |act'| <= 1.13: E_h = 1.13 |u| E_g + |act| E_u, and the activation's
own (6 |z| + 8) E |h|, under 100 E |h|.

A sum without `lost` of its n terms is off by S sqrt(lost / n).  U is at most 2^-8 and n E 1.9e-3 (n = 31200): together
6.3e-3; 64 lost terms of 31200 are 4.5e-2, eight 1.6e-2.
"""

import numpy as np
import torch

import oracle.ffn_oracle as orc
from block_util import E, TINY, TYPES, U, gen, randn
from parity_util import to64

BLOCK = 32


def inputs(T, C, F, dtype):
    g = gen(5 * T + 11 * C + F)
    x, dh = randn(g, T, C, dtype=dtype), randn(g, T, F, dtype=dtype)
    return x, randn(g, F, C, dtype=dtype, scale=C ** -0.5), randn(g, F, C, dtype=dtype, scale=C ** -0.5), dh


def rounded(v, dtype):
    return torch.from_numpy(v).to(TYPES[dtype]).double().numpy()


def _size(a, b):
    return np.sqrt((a * a) @ (b * b))


def forward(x, wg, wu, kind, dtype):
    """{output: (reference, error that its blocks' norms stay below)}"""
    x, wg, wu = to64(x), to64(wg).T, to64(wu).T
    h, g, u = orc.gated_fwd(x, wg.T, wu.T, kind)
    acc = (x.shape[1] + 16) * E
    eg, eu = acc * _size(x, wg), acc * _size(x, wu)
    eh = 1.13 * np.abs(u) * eg + np.abs(orc.activation(g, kind)) * eu + 100 * E * np.abs(h)
    return {n: (v, e + U[dtype] * np.abs(v) + TINY) for n, v, e in (("h", h, eh), ("gate", g, eg), ("up", u, eu))}


def operands(x, wg, wu, gate, up, dh, kind, dtype):
    """{output: the pairs (a, b) whose products a @ b are added up}"""
    dg = rounded(to64(dh) * to64(up) * orc.slope(to64(gate), kind), dtype)
    du = rounded(to64(dh) * orc.activation(to64(gate), kind), dtype)
    return {"dx": [(dg, to64(wg)), (du, to64(wu))], "dw_gate": [(dg.T, to64(x))], "dw_up": [(du.T, to64(x))]}


def backward(products, dtype):
    """{output: (reference, error)} of operands()"""
    out = {}
    for name, pairs in products.items():
        n = sum(a.shape[1] for a, _ in pairs)
        ref = sum(a @ b for a, b in pairs)
        size = np.sqrt(sum((a * a) @ (b * b) for a, b in pairs))
        out[name] = (ref, ((n + 116) * E + (U[dtype] / 8 if dtype == "bf16" else 0)) * size + U[dtype] * np.abs(ref) + TINY)
    return out


def _norms(v):
    rows, cols = (np.arange(0, n, BLOCK) for n in v.shape)
    return np.sqrt(np.add.reduceat(np.add.reduceat(v * v, rows, 0), cols, 1))


def off(got, ref, error):
    """The blocks' errors as shares of what they may be."""
    got = to64(got)
    assert got.shape == ref.shape and np.isfinite(got).all()
    return _norms(got - ref) / _norms(error)
