"""Gated projections on the GPU against the float64 oracle (bounds: ffn_util)."""

import numpy as np
import pytest
import torch

import oracle.ffn_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import TYPES, gen, randn, within
from ffn_util import bwd_bounds, fwd_bounds
from parity_util import say, to64

pytestmark = pytest.mark.gpu

# T x C x F: one row, one piece of 8 columns; rows that end inside a tile, columns that end inside a tile, a chunk
# or a 16-byte piece of one; each form that few rows take; whole tiles; more tiles than work groups at once
SHAPES = [(1, 8, 8), (1, 1600, 4288), (2, 24, 40), (3, 64, 8), (7, 520, 136), (8, 4096, 1024), (15, 72, 256), (16, 768, 2048),
          (17, 136, 264), (24, 1000, 504), (31, 32, 32), (32, 2048, 520), (33, 40, 72), (48, 800, 640), (63, 8, 264),
          (64, 256, 384), (65, 264, 1032), (100, 512, 1368), (128, 128, 128), (129, 192, 136), (200, 2048, 776), (255, 96, 2056),
          (256, 1024, 512), (257, 88, 1000), (511, 776, 264), (777, 1000, 728), (1024, 768, 2048), (1300, 320, 648),
          (3000, 64, 200), (40, 64, 9000)]


def data(T, C, F, dtype, seed=0):
    g = gen(T * 131 + C * 17 + F + seed)
    w = C ** -0.5
    return (randn(g, T, C, dtype=dtype), randn(g, F, C, dtype=dtype, scale=w), randn(g, F, C, dtype=dtype, scale=1.5 * w),
            randn(g, T, F, dtype=dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,C,F", SHAPES)
def test_forward_and_backward(cuda, T, C, F, dtype):
    kind = "gelu" if (T + C // 8) % 2 else "silu"
    say(f"gated T={T} C={C} F={F} {dtype} {kind}")
    x, wg, wu, dh = data(T, C, F, dtype)
    xd, wgd, wud, dhd = (t.to(cuda) for t in (x, wg, wu, dh))
    h, gate, up = cattn.gated_fwd(xd, wgd, wud, kind, save=True)
    ref = orc.gated_fwd(to64(x), to64(wg), to64(wu), kind)
    for name, got, r, b in zip(("h", "gate", "up"), (h, gate, up), ref, fwd_bounds(x, wg, wu, ref, kind, dtype)):
        assert got.dtype == TYPES[dtype] and got.shape == (T, F)
        within(name, got, r, b)
    alone = cattn.gated_fwd(xd, wgd, wud, kind)
    assert torch.equal(alone[0], h) and alone[1] is None and alone[2] is None
    grads = cattn.gated_bwd(xd, wgd, wud, gate, up, dhd, kind)
    ref = orc.gated_bwd(to64(x), to64(wg), to64(wu), to64(gate), to64(up), to64(dh), kind)
    for name, got, r, b in zip(("dx", "dw_gate", "dw_up"), grads, ref,
                               bwd_bounds(x, wg, wu, gate, up, dh, ref, kind, dtype)):
        assert got.dtype == TYPES[dtype]
        within(name, got, r, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_far_activations(cuda, kind, dtype):
    """Products from far below to far above: one column, so that gate and up are what x says."""
    v = torch.tensor([0.0, 1e-30, 1e-3, 0.5, 3.0, 8.0, 20.0, 60.0, 87.0, 89.0, 200.0, 1e4, 1e10, 1e15, 1e18])
    x = torch.zeros(2 * v.numel(), 8)
    x[:, 0] = torch.cat([v, -v])
    wg, wu = torch.zeros(8, 8), torch.zeros(8, 8)
    wg[:, 0] = 1
    wu[:, 0] = torch.tensor([1, -1, 0.5, 2, 0, 1e-3, 4, -8.0]) * 2.0 ** -20
    dh = torch.ones(x.shape[0], 8)
    x, wg, wu, dh = (t.to(TYPES[dtype]) for t in (x, wg, wu, dh))
    dev = [t.to(cuda) for t in (x, wg, wu)]
    h, gate, up = cattn.gated_fwd(*dev, kind, save=True)
    ref = orc.gated_fwd(to64(x), to64(wg), to64(wu), kind)
    for name, got, r, b in zip(("h", "gate", "up"), (h, gate, up), ref, fwd_bounds(x, wg, wu, ref, kind, dtype)):
        within(name, got, r, b)
    grads = cattn.gated_bwd(*dev, gate, up, dh.to(cuda), kind)
    ref = orc.gated_bwd(to64(x), to64(wg), to64(wu), to64(gate), to64(up), to64(dh), kind)
    for name, got, r, b in zip(("dx", "dw_gate", "dw_up"), grads, ref, bwd_bounds(x, wg, wu, gate, up, dh, ref, kind, dtype)):
        within(name, got, r, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 40, 300])
def test_non_finite_rows_stay_their_own(cuda, T, dtype):
    """A NaN or an infinity of x reaches its own row of h, gate, up and dx, one of a weight its own column."""
    C, F = 264, 328
    x, wg, wu, dh = data(T, C, F, dtype, 5)
    x[1, 260], x[T - 1, 0], wu[327, 3] = float("nan"), float("inf"), float("nan")
    dev = [t.to(cuda) for t in (x, wg, wu)]
    h, gate, up = cattn.gated_fwd(*dev, save=True)
    rows = [i for i in range(T) if i not in (1, T - 1)]
    for t in (h, gate, up):
        assert t[1].isnan().all() and t[rows, :327].isfinite().all()
    assert not gate[T - 1].isfinite().any() and h[:, 327].isnan().all() and gate[rows].isfinite().all()
    dx, _, dwu = cattn.gated_bwd(dev[0].nan_to_num(0, 0, 0), dev[1], dev[2].nan_to_num(0), gate, up.nan_to_num(0, 0, 0), dh.to(cuda))
    assert dx[1].isnan().all() and dx[rows].isfinite().all() and dwu.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_and_shapes(cuda, dtype):
    dt = TYPES[dtype]
    x, w = torch.empty(0, 64, device=cuda, dtype=dt), torch.ones(24, 64, device=cuda, dtype=dt)
    h, gate, up = cattn.gated_fwd(x, w, w, save=True)
    assert h.shape == gate.shape == up.shape == (0, 24)
    dx, dwg, dwu = cattn.gated_bwd(x, w, w, gate, up, h)
    assert dx.shape == (0, 64) and not dwg.any() and not dwu.any()
    x, w = torch.ones(3, 0, device=cuda, dtype=dt), torch.ones(24, 0, device=cuda, dtype=dt)
    h, gate, up = cattn.gated_fwd(x, w, w, save=True)
    assert h.shape == (3, 24) and not h.any() and not gate.any() and not up.any()
    assert [t.shape for t in cattn.gated_bwd(x, w, w, gate, up, h)] == [(3, 0), (24, 0), (24, 0)]
    x, w = torch.ones(3, 16, device=cuda, dtype=dt), torch.ones(0, 16, device=cuda, dtype=dt)
    h, gate, up = cattn.gated_fwd(x, w, w, save=True)
    dx, dwg, dwu = cattn.gated_bwd(x, w, w, gate, up, h)
    assert h.shape == (3, 0) and dwg.shape == (0, 16) and not dx.any()
    x = randn(gen(1), 2, 5, 64, dtype=dtype).to(cuda)
    w = randn(gen(2), 24, 64, dtype=dtype).to(cuda)
    h, gate, up = cattn.gated_fwd(x, w, w, save=True)
    assert h.shape == (2, 5, 24) and cattn.gated_bwd(x, w, w, gate, up, h)[0].shape == (2, 5, 64)
    one = cattn.gated_fwd(x[1, 2], w, w)[0]
    assert one.shape == (24,)
    b = fwd_bounds(x[1, 2:3].cpu(), w.cpu(), w.cpu(), orc.gated_fwd(to64(x[1, 2:3].cpu()), to64(w.cpu()), to64(w.cpu())), "silu", dtype)[0]
    within("one row", one[None], to64(h[1, 2:3].cpu()), 2 * b)


@pytest.mark.parametrize("T,C,F,dtype", [(1, 768, 512, "bf16"), (20, 512, 1032, "bf16"), (300, 264, 648, "bf16"), (700, 768, 2048, "bf16"),
                                         (1, 768, 512, "f32"), (300, 264, 648, "f32")])
def test_a_replayed_graph_and_two_streams(cuda, T, C, F, dtype):
    x, wg, wu, dh = (t.to(cuda) for t in data(T, C, F, dtype, 9))

    def run():
        out = cattn.gated_fwd(x, wg, wu, "gelu", save=True)
        return out + cattn.gated_bwd(x, wg, wu, out[1], out[2], dh, "gelu")

    first = run()
    torch.cuda.synchronize()
    results = []
    for s in [torch.cuda.Stream(), torch.cuda.Stream()] * 2:
        with torch.cuda.stream(s):
            results.append(run())
    torch.cuda.synchronize()
    for out in results:
        assert all(torch.equal(a, b) for a, b in zip(out, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(3):
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        eager = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(captured, first, eager))
    x.copy_(-x)  # the same addresses, other values
    graph.replay()
    eager = run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, eager)) and not torch.equal(captured[0], first[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,C,F", [(3, 72, 40), (20, 264, 136), (130, 72, 200), (300, 328, 264)])
def test_nothing_is_written_past_the_outputs(cuda, T, C, F, dtype):
    """Outputs and workspace inside one guarded allocation each, through the C entry points; inputs at the very end of theirs."""
    from paper_2608_00029_amd import binding as b
    dt, e = TYPES[dtype], 2 if dtype == "bf16" else 4
    x, wg, wu, dh = (t.to(cuda) for t in data(T, C, F, dtype, 3))
    guard = 4096
    code = b.CATTN_BF16 if dtype == "bf16" else b.CATTN_F32
    ws = b.lib().cattn_gated_bwd_workspace_bytes(T, C, F, code)
    sizes = {"h": T * F * e, "gate": T * F * e, "up": T * F * e, "dx": T * C * e, "dwg": F * C * e, "dwu": F * C * e, "ws": ws}
    buf = {n: torch.full((s + 2 * guard,), 0x5A, dtype=torch.uint8, device=cuda) for n, s in sizes.items()}
    at = {n: t.data_ptr() + guard for n, t in buf.items()}
    st = torch.cuda.current_stream().cuda_stream
    assert b.lib().cattn_gated_fwd(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), at["h"], at["gate"], at["up"], T, C, F, 0, code, st) == 0
    assert b.lib().cattn_gated_bwd(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), at["gate"], at["up"], dh.data_ptr(), at["dx"],
                                   at["dwg"], at["dwu"], at["ws"], T, C, F, 0, code, st) == 0
    torch.cuda.synchronize()
    for n, s in sizes.items():
        assert (buf[n][:guard] == 0x5A).all() and (buf[n][guard + s:] == 0x5A).all(), n
    h, gate, up = cattn.gated_fwd(x, wg, wu, save=True)
    out = dict(zip(("dx", "dwg", "dwu"), cattn.gated_bwd(x, wg, wu, gate, up, dh)), h=h, gate=gate, up=up)
    for n, t in out.items():
        assert torch.equal(buf[n][guard:guard + sizes[n]].view(dt).view(t.shape), t), n
