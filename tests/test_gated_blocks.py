"""That the checks of test_gpu_gated_blocks.py can fail: for each of its cases a sum without one chunk of k, without one
16-byte piece of k, or with the piece twice, planted in the reference, is seen in every whole block of 32 x 32, and a sum that
is rounded as the kernels round it is taken."""

import numpy as np
import pytest

import gated_blocks as gb
import oracle.ffn_oracle as orc
from parity_util import to64
from test_gpu_gated_forms import CASES

N = 64  # rows and columns of the outputs that are looked at: the sums are whole


@pytest.mark.parametrize("T,C,F,dtype", CASES)
def test_lost_pieces_are_seen(T, C, F, dtype):
    x, wg, wu, dh = gb.inputs(T, C, F, dtype)
    chunk, piece = (64, 8) if dtype == "bf16" else (32, 4)

    def seen(name, at, ref, error, lost):
        whole = np.ones(tuple(n // gb.BLOCK for n in ref.shape), dtype=bool)
        for what, sign in (("lost", -1), ("twice", 1)):
            share = gb.off(gb.rounded(ref + sign * lost, dtype), ref, error)
            share = share[:whole.shape[0], :whole.shape[1]] if whole.size else share.max(keepdims=True)
            assert (share > 1).all(), (name, what, at, float(share.min()))

    # the forward, by its pre-activations
    a, b = to64(x[:N]), to64(wg[:N]).T
    ref, error = gb.forward(x[:N], wg[:N], wu[:N], "gelu", dtype)["gate"]
    assert (gb.off(gb.rounded(ref, dtype), ref, error) <= 1).all()
    for n in (chunk, piece):
        for at in {0, C // 2 // piece * piece, C - piece}:
            seen("gate", at, ref, error, a[:, at:at + n] @ b[at:at + n])
    for names, xs, fs in (("dx",), slice(N), slice(None)), (("dw_gate", "dw_up"), slice(None), slice(N)):
        part = (x[xs], wg[fs], wu[fs])
        _, gate, up = orc.gated_fwd(*(to64(t) for t in part), "gelu")
        products = gb.operands(*part, gb.rounded(gate, dtype), gb.rounded(up, dtype), dh[xs, fs], "gelu", dtype)
        for name in names:
            pairs = [(a[:N], b[:, :N]) for a, b in products[name]]
            ref, error = gb.backward({name: pairs}, dtype)[name]
            assert (gb.off(gb.rounded(ref, dtype), ref, error) <= 1).all()
            for a, b in pairs:
                K = a.shape[1]
                for n in (chunk, piece):
                    for at in {0, K // 2 // piece * piece, max(0, (K - 1) // chunk * chunk)}:
                        seen(name, at, ref, error, a[:, at:at + n] @ b[at:at + n])
