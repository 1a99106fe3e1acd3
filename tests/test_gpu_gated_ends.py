"""Gated projections: nothing past the ends of an input reaches a result.  Every input, and what the backward reads of the
forward, lies between NaN in a buffer of its own, so that a piece past the end of k that one operand alone takes as zero, or
a row past the last that is summed over, makes a NaN; the same calls on tensors of their own give the same bits."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from block_util import TYPES, gen, randn
from parity_util import say
from test_gpu_gated_forms import CASES

pytestmark = pytest.mark.gpu

GUARD = 1 << 20  # elements


def guarded(t):
    buf = torch.full((t.numel() + 2 * GUARD,), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[GUARD:GUARD + t.numel()].view(t.shape)
    view.copy_(t)
    assert view.data_ptr() % 16 == 0 and view.is_contiguous()
    return view


# one 16-byte piece of k, one past a chunk, one short of it; every form and cut of k
@pytest.mark.parametrize("T,C,F,dtype", [(T, C, F, d) for T, C, F in ((1, 8, 8), (3, 72, 40), (17, 136, 264), (65, 120, 72), (300, 328, 264))
                                         for d in TYPES] + CASES)
def test_between_nan(cuda, T, C, F, dtype):
    say(f"gated T={T} C={C} F={F} {dtype}")
    g = gen(T + C + F)
    x, dh = randn(g, T, C, dtype=dtype).to(cuda), randn(g, T, F, dtype=dtype).to(cuda)
    wg, wu = (randn(g, F, C, dtype=dtype, scale=C ** -0.5).to(cuda) for _ in range(2))

    def run(wrap):
        a = [wrap(t) for t in (x, wg, wu)]
        out = cattn.gated_fwd(*a, "silu", save=True)
        return out + cattn.gated_bwd(*a, wrap(out[1]), wrap(out[2]), wrap(dh), "silu")

    ws = cattn.gated_bwd_workspace_bytes(T, C, F, TYPES[dtype]) // 4
    out = run(lambda t: t)
    for a, b in zip(run(guarded), out):
        assert a.isfinite().all() and torch.equal(a, b)
    nan = torch.full((ws,), float("nan"), device=cuda)  # (what the workspace held does not matter either)
    for a, b in zip(cattn.gated_bwd(x, wg, wu, out[1], out[2], dh, "silu", workspace=nan), out[3:]):
        assert torch.equal(a, b)
