"""Every form of the gated projections' tile kernel, in every product and with k in parts, and of the few-rows kernel, on
the GPU against the float64 oracle.  The cases' forms are derived on the CPU (test_gated_forms.py)."""

import pytest
import torch

import oracle.ffn_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import gen, randn, within
from ffn_util import bwd_bounds, fwd_bounds
from parity_util import say, to64

pytestmark = pytest.mark.gpu

# T, C, F, dtype: products that take each form, ragged in every direction
CASES = [
    # few rows: 8 or 16 columns a work group, up to 16 tokens and up to 32
    (3, 200, 136, "bf16"), (4, 72, 8200, "bf16"), (13, 200, 72, "bf16"), (29, 136, 456, "bf16"), (3, 200, 136, "f32"),
    (11, 200, 4104, "f32"), (31, 200, 4104, "f32"), (13, 200, 72, "f32"), (29, 136, 456, "f32"),
    # the tiles with as few
    (11, 328, 4104, "bf16"), (30, 328, 2056, "bf16"), (7, 200, 8200, "bf16"),
    # bfloat16 tiles: forward by each form; dx and dW by each, whole and in parts
    (33, 40, 904, "bf16"), (1799, 40, 72, "bf16"), (65, 72, 4112, "bf16"), (258, 40, 8280, "bf16"), (132, 40, 8408, "bf16"), (386, 40, 10936, "bf16"),
    (9781, 136, 136, "bf16"), (16441, 40, 40, "bf16"), (68, 1032, 2312, "bf16"), (33, 9224, 272, "bf16"), (21661, 136, 528, "bf16"),
    (33, 8520, 136, "bf16"), (16239, 32, 1048, "bf16"), (34, 264, 12816, "bf16"), (12871, 4168, 200, "bf16"), (518, 11216, 40, "bf16"),
    (1026, 136, 12216, "bf16"), (16528, 136, 40, "bf16"), (1033, 32, 15288, "bf16"), (16565, 528, 40, "bf16"), (193, 4272, 11400, "bf16"),
    # float32
    (300, 72, 40, "f32"), (494, 40, 264, "f32"), (35, 8312, 40, "f32"), (67, 8224, 32, "f32"), (33, 8480, 72, "f32"), (16640, 72, 32, "f32"),
    (21293, 72, 800, "f32"), (5747, 3232, 32, "f32"), (67, 3136, 5632, "f32"), (33, 3200, 5968, "f32"),
]


@pytest.mark.parametrize("T,C,F,dtype", CASES)
def test_against_the_oracle(cuda, T, C, F, dtype):
    say(f"gated T={T} C={C} F={F} {dtype}")
    g = gen(T + 3 * C + 7 * F)
    x, dh = randn(g, T, C, dtype=dtype), randn(g, T, F, dtype=dtype)
    wg, wu = randn(g, F, C, dtype=dtype, scale=C ** -0.5), randn(g, F, C, dtype=dtype, scale=C ** -0.5)
    dev = [t.to(cuda) for t in (x, wg, wu)]
    out = cattn.gated_fwd(*dev, "silu", save=True)
    ref = orc.gated_fwd(to64(x), to64(wg), to64(wu), "silu")
    for name, got, r, b in zip(("h", "gate", "up"), out, ref, fwd_bounds(x, wg, wu, ref, "silu", dtype)):
        within(name, got, r, b)
    ws = torch.full((cattn.gated_bwd_workspace_bytes(T, C, F, x.dtype) // 4 + 64,), float("nan"), device=cuda)
    grads = cattn.gated_bwd(*dev, out[1], out[2], dh.to(cuda), "silu", workspace=ws)
    ref = orc.gated_bwd(to64(x), to64(wg), to64(wu), to64(out[1]), to64(out[2]), to64(dh), "silu")
    for name, got, r, b in zip(("dx", "dw_gate", "dw_up"), grads, ref,
                               bwd_bounds(x, wg, wu, out[1], out[2], dh, ref, "silu", dtype)):
        within(name, got, r, b)
    assert ws[-64:].isnan().all()
