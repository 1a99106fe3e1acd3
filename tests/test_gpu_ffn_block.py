"""The feed-forward operators together, as a decoder block's second half uses them, beside RMSNorm: a training step and its
gradients, a captured one, and single tokens after a prompt; and offsets past 32 bits."""

import numpy as np
import pytest
import torch

import oracle.ffn_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import gen, randn, within
from ffn_util import bwd_bounds, fwd_bounds
from parity_util import say, to64

pytestmark = pytest.mark.gpu

SEED, P = 77, 0.2


class Block:
    """a = r + drop(y); n = norm(a); h = act(n Wg^T) (n Wu^T); out = a + drop(h Wd^T)"""

    def __init__(self, C=256, F=712, dtype="f32"):
        g = gen(21)
        self.gamma = 1 + 0.1 * randn(g, C)
        self.wg, self.wu = randn(g, F, C, dtype=dtype, scale=C ** -0.5), randn(g, F, C, dtype=dtype, scale=C ** -0.5)
        self.wd = randn(g, C, F, dtype=dtype, scale=F ** -0.5)

    def to(self, device):
        self.gamma, self.wg, self.wu, self.wd = (t.to(device) for t in (self.gamma, self.wg, self.wu, self.wd))
        return self

    def step(self, y, r, dout, step):
        a = cattn.dropout_fwd(y, P, SEED, 0, step, r)
        n, _, rstd = cattn.rmsnorm_fwd(a, self.gamma)
        h, gate, up = cattn.gated_fwd(n, self.wg, self.wu, "gelu", save=True)
        out = cattn.dropout_fwd(h @ self.wd.t(), P, SEED, 1, step, a)
        dz = cattn.dropout_bwd(dout, P, SEED, 1, step)
        dn, dwg, dwu = cattn.gated_bwd(n, self.wg, self.wu, gate, up, dz @ self.wd, "gelu")
        da, dgamma = cattn.rmsnorm_bwd(a, self.gamma, rstd, dn, dout)
        dwd = dz.t() @ h
        return {"out": out, "dy": cattn.dropout_bwd(da, P, SEED, 0, step), "dr": da, "dgamma": dgamma, "dwg": dwg, "dwu": dwu,
                "dwd": dwd}


@pytest.mark.parametrize("T", [5, 70, 300])
def test_a_training_step_and_its_gradients(cuda, T):
    """Against autograd in float64 on the CPU, with the oracle's masks."""
    g = gen(T)
    y, r, dout = (randn(g, T, 256) for _ in range(3))
    got = Block().to(cuda).step(*(t.to(cuda) for t in (y, r, dout)), 9)
    ref = Block()
    leaves = {n: t.double().requires_grad_() for n, t in (("y", y), ("r", r), ("gamma", ref.gamma), ("wg", ref.wg), ("wu", ref.wu), ("wd", ref.wd))}

    def drop(x, site):
        keep = torch.from_numpy(orc.dropout_keep(x.numel(), P, SEED, site, 9)).view(x.shape)
        return torch.where(keep, x / (1 - P), torch.zeros_like(x))

    a = leaves["r"] + drop(leaves["y"], 0)
    n = a * (a.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * leaves["gamma"]
    h = torch.nn.functional.gelu(n @ leaves["wg"].t(), approximate="tanh") * (n @ leaves["wu"].t())
    out = a + drop(h @ leaves["wd"].t(), 1)
    out.backward(dout.double())
    want = {"out": out.detach()} | {"d" + n: t.grad for n, t in leaves.items()}
    # float32 throughout: chains of sums of at most 1424 terms, 2^-24 each; 1e-5 of the norm is ample for one that adds
    # up (1432 * 2^-24 = 8.5e-5 of the terms' absolute sum only where all roundings agree; independent ones stay below
    # 40 * 2^-24) and far below any wrong term
    for name, v in want.items():
        err = (got[name].cpu().double() - v).norm() / v.norm()
        assert err <= 1e-5, (name, float(err))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_training_step(cuda, dtype):
    """One graph for the step, its counter in device memory: every replay equals the eager step of that number."""
    T, blk = 130, Block(dtype=dtype).to(cuda)
    blk.wd = blk.wd.contiguous()
    g = gen(4)
    y, r, dout = (randn(g, T, 256, dtype=dtype).to(cuda) for _ in range(3))
    step = torch.tensor([5], device=cuda)
    blk.step(y, r, dout, step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = blk.step(y, r, dout, step)
        step += 1
    seen = []
    for k in range(5, 9):
        graph.replay()
        eager = blk.step(y, r, dout, k)
        torch.cuda.synchronize()
        for n, t in eager.items():
            assert torch.equal(out[n], t), (k, n)
        seen.append(out["out"].clone())
    assert not any(torch.equal(seen[0], s) for s in seen[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_equal_the_batch(cuda, dtype):
    """Rows one, three, twenty at a time (the few-rows kernel) against the same rows of a prompt (the tiles): each within
    its bound of the exact result, so within two of the other's."""
    T, C, F = 150, 520, 1368
    g = gen(8)
    x = randn(g, T, C, dtype=dtype)
    wg, wu = randn(g, F, C, dtype=dtype, scale=C ** -0.5), randn(g, F, C, dtype=dtype, scale=C ** -0.5)
    dev = [t.to(cuda) for t in (x, wg, wu)]
    whole = cattn.gated_fwd(*dev)[0]
    bound = fwd_bounds(x, wg, wu, orc.gated_fwd(to64(x), to64(wg), to64(wu)), "silu", dtype)[0]
    for n in (1, 3, 20):
        for at in (0, 71, T - n):
            h = cattn.gated_fwd(dev[0][at:at + n].contiguous(), dev[1], dev[2])[0]
            within("rows", h, to64(whole[at:at + n]), 2 * bound[at:at + n])


def test_offsets_past_32_bits(cuda):
    """gate, up, h and dh of 2^31 elements and more: the first and last rows."""
    T, C, F = 262208, 16, 8200
    assert T * F > 1 << 31
    say(f"gated T={T} C={C} F={F}")
    g = gen(1)
    x, wg, wu = randn(g, T, C, dtype="bf16"), randn(g, F, C, dtype="bf16", scale=0.25), randn(g, F, C, dtype="bf16", scale=0.25)
    dev = [t.to(cuda) for t in (x, wg, wu)]
    out = cattn.gated_fwd(*dev, "silu", save=True)
    rows = [0, 1, 261888, 262077, T - 1]
    ref = orc.gated_fwd(to64(x[rows]), to64(wg), to64(wu))
    for name, t, r, b in zip(("h", "gate", "up"), out, ref, fwd_bounds(x[rows], wg, wu, ref, "silu", "bf16")):
        within(name, t[rows], r, b)
    dh = torch.zeros_like(out[0])  # gradients of these rows alone
    up = randn(g, len(rows), F, dtype="bf16")
    dh[rows] = up.to(cuda)
    dx, dwg, dwu = cattn.gated_bwd(*dev, out[1], out[2], dh)
    args = (x[rows], wg, wu, out[1][rows].cpu(), out[2][rows].cpu(), up)
    ref = orc.gated_bwd(*(to64(t) for t in args))
    bounds = bwd_bounds(*args, ref, "silu", "bf16")
    within("dx", dx[rows], ref[0], bounds[0])
    dx[rows] = 0
    assert not dx.any()
    within("dw_gate", dwg, ref[1], bounds[1])  # (zeros add nothing, and no rounding)
    within("dw_up", dwu, ref[2], bounds[2])
