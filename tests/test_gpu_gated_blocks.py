"""Every form and every cut of k of the gated projections, by blocks of 32 x 32 elements: no piece of a sum is lost or taken
twice, however long the sum (gated_blocks.py; that a lost piece is seen: test_gated_blocks.py)."""

import pytest

import gated_blocks as gb
import paper_2608_00029_amd as cattn
from parity_util import say
from test_gpu_gated_forms import CASES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,C,F,dtype", CASES)
def test_no_piece_is_lost(cuda, T, C, F, dtype):
    say(f"gated T={T} C={C} F={F} {dtype}")
    x, wg, wu, dh = gb.inputs(T, C, F, dtype)
    dev = [t.to(cuda) for t in (x, wg, wu)]
    h, gate, up = cattn.gated_fwd(*dev, "gelu", save=True)
    grads = cattn.gated_bwd(*dev, gate, up, dh.to(cuda), "gelu")
    got = dict(zip(("h", "gate", "up", "dx", "dw_gate", "dw_up"), (h, gate, up, *grads)))
    want = gb.forward(x, wg, wu, "gelu", dtype) | gb.backward(gb.operands(x, wg, wu, gate, up, dh, "gelu", dtype), dtype)
    for name, (ref, error) in want.items():
        share = gb.off(got[name], ref, error)
        print(f"  {name}: {share.max():.2f}")
        assert (share <= 1).all(), (name, float(share.max()), int((share > 1).sum()), share.size)
