"""RMSNorm on the GPU against the float64 oracle (bounds: block_util)."""

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import E, TINY, TYPES, U, gen, randn, within
from parity_util import say, to64

pytestmark = pytest.mark.gpu

# rows x C: one row, one 8-column row, a row that ends inside a wave's step, each number of waves and
# steps a row takes, more rows than work groups take at once, the widest row
SHAPES = [(1, 8), (3, 64), (5, 520), (7, 1600), (2, 2048), (9, 2056), (1, 4096), (70, 4104), (3, 8192), (2, 8200),
          (2, 16384), (300, 2056), (1030, 768), (1024, 1024), (1025, 1032), (8200, 128), (2100, 2560), (513, 8192), (600, 8200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_forward_and_backward(cuda, rows, C, dtype):
    say(f"rmsnorm rows={rows} C={C} {dtype}")
    g = gen(rows * 31 + C)
    x, r = randn(g, rows, C, dtype=dtype), randn(g, rows, C, dtype=dtype, scale=3.0)
    gamma, dy, dh = 1 + 0.2 * randn(g, C), randn(g, rows, C, dtype=dtype), randn(g, rows, C, dtype=dtype)
    xd, rd, gd, dyd, dhd = (t.to(cuda) for t in (x, r, gamma, dy, dh))
    for res, resd, up, upd in ((r, rd, dh, dhd), (None, None, None, None)):
        y, h, rstd = cattn.rmsnorm_fwd(xd, gd, resd)
        assert (h is xd) == (res is None) and y.dtype == TYPES[dtype] and rstd.shape == (rows,)
        ry, rh, rr = orc.rmsnorm_fwd(to64(x), to64(gamma), None if res is None else to64(res))
        within("rstd", rstd, rr, 40 * E * rr)
        within("y", y, ry, (64 * E + U[dtype]) * np.abs(ry) + TINY)
        if res is not None:
            within("h", h, rh, (E + U[dtype]) * np.abs(rh) + TINY)
        dx, dgamma = cattn.rmsnorm_bwd(h, gd, rstd, dyd, upd)
        rdx, rdg = orc.rmsnorm_bwd(to64(h), to64(gamma), to64(rstd), to64(dy), None if up is None else to64(up))
        xhat = np.abs(to64(h) * to64(rstd)[:, None])
        gr = np.abs(to64(dy) * to64(gamma))
        size = to64(rstd)[:, None] * (gr + xhat * np.mean(gr * xhat, axis=1, keepdims=True)) \
            + (0 if up is None else np.abs(to64(up)))
        within("dx", dx, rdx, 64 * E * size + U[dtype] * np.abs(rdx) + TINY)
        # a work group adds at most its block of rows, the rest is 128 streams of partial rows
        terms = np.sum(np.abs(to64(dy)) * xhat, axis=0)
        within("dgamma", dgamma, rdg, (rows / 512 + 64) * E * terms + TINY)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C,group", [(1, 8, 8), (3, 1600, 128), (16, 4096, 128), (5, 2056, 0), (70, 520, 512),
                                          (1030, 768, 64), (2, 16384, 0), (2, 16384, 16), (300, 2056, 0), (1025, 1032, 0),
                                          (9, 72, 32)])
def test_eight_bits(cuda, rows, C, group, dtype):
    say(f"rmsnorm q8 rows={rows} C={C} group={group} {dtype}")
    g = gen(rows + C + group)
    x, r, gamma = randn(g, rows, C, dtype=dtype), randn(g, rows, C, dtype=dtype), 1 + 0.2 * randn(g, C)
    x[0, :8] = r[0, :8] = 0  # a group of zeros (in groups of 8)
    q, scale, h, rstd = cattn.rmsnorm_fwd_q8(x.to(cuda), gamma.to(cuda), r.to(cuda), 1e-5, group)
    y, h2, rstd2 = cattn.rmsnorm_fwd(x.to(cuda), gamma.to(cuda), r.to(cuda))
    assert torch.equal(h, h2) and torch.equal(rstd, rstd2) and q.dtype == torch.float8_e4m3fn
    ry, _, _ = orc.rmsnorm_fwd(to64(x), to64(gamma), to64(r))
    rs = orc.q8_scales(ry, group)
    within("scale", scale, rs, 66 * E * rs)
    # half a step of the code: 2^-4 of a normal value, 2^-10 of the scale below 2^-6 of it
    wide = np.repeat(to64(scale), group or C, axis=1)[:, :C]
    got = q.cpu().float().double().numpy() * wide
    assert np.abs(q.cpu().float().numpy()).max() <= 448
    within("y", got, ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * wide) + 70 * E * np.abs(ry))
    if group != 8:
        assert (np.abs(q.cpu().float().numpy()).reshape(rows, -1).max(1) == 448).all()  # the largest takes the last code


def test_non_finite_rows_stay_their_own(cuda):
    """A NaN or an infinity makes its own row's results non-finite and no other's."""
    x = randn(gen(3), 6, 2056)
    x[1, 7], x[4, 2000] = float("nan"), float("inf")
    gamma = torch.ones(2056)
    y, _, rstd = cattn.rmsnorm_fwd(x.to(cuda), gamma.to(cuda))
    q, scale, _, _ = cattn.rmsnorm_fwd_q8(x.to(cuda), gamma.to(cuda), None, 1e-5, 128)
    y, rstd, q = y.cpu(), rstd.cpu(), q.cpu().float()
    assert y[1].isnan().all() and rstd[1].isnan() and q[1].isnan().all()
    assert rstd[4] == 0 and y[4, 2000].isnan() and (y[4, :2000] == 0).all() and q[4, 2000].isnan()
    keep = [0, 2, 3, 5]
    assert y[keep].isfinite().all() and q[keep].isfinite().all() and scale.cpu()[keep].isfinite().all()


def test_empty_and_shapes(cuda):
    x = torch.empty(0, 64, device=cuda, dtype=torch.bfloat16)
    gamma = torch.ones(64, device=cuda)
    y, h, rstd = cattn.rmsnorm_fwd(x, gamma)
    dx, dgamma = cattn.rmsnorm_bwd(h, gamma, rstd, x)
    assert y.shape == dx.shape == (0, 64) and rstd.shape == (0,) and not dgamma.any()
    x = randn(gen(1), 2, 3, 64).to(cuda)
    assert cattn.rmsnorm_fwd(x, gamma)[0].shape == (2, 3, 64) and cattn.rmsnorm_fwd(x, gamma)[2].shape == (6,)


@pytest.mark.parametrize("rows,C", [(700, 768), (90, 4096)])
def test_a_replayed_graph_and_two_streams(cuda, rows, C):
    x, r, dy = (randn(gen(40 + i), rows, C, dtype="bf16").to(cuda) for i in range(3))
    gamma = torch.ones(C, device=cuda)

    def run():
        y, h, rstd = cattn.rmsnorm_fwd(x, gamma, r)
        q, scale, _, _ = cattn.rmsnorm_fwd_q8(x, gamma, r, group=64)
        return (y, h, rstd, q.view(torch.uint8), scale) + cattn.rmsnorm_bwd(h, gamma, rstd, dy, r)

    first = run()
    torch.cuda.synchronize()
    results = []
    for s in [torch.cuda.Stream(), torch.cuda.Stream()] * 2:
        with torch.cuda.stream(s):
            results.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in results for a, b in zip(first, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(3):
        x.copy_(torch.roll(x, 1, 0))
        gamma += 0.25
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_offsets_past_32_bits(cuda):
    """2^31 elements and some: the last rows as a call of their own gives them."""
    rows, C = (1 << 17) + 40, 16384
    x = torch.zeros(rows, C, dtype=torch.bfloat16, device=cuda)
    x[-40:] = randn(gen(60), 40, C, dtype="bf16").to(cuda)
    gamma = torch.ones(C, device=cuda)
    say(f"rmsnorm rows{rows} C{C}")
    y, _, rstd = cattn.rmsnorm_fwd(x, gamma)
    want, _, want_rstd = cattn.rmsnorm_fwd(x[-40:].contiguous(), gamma)
    assert torch.equal(y[-40:], want) and torch.equal(rstd[-40:], want_rstd)
    dx, _ = cattn.rmsnorm_bwd(x, gamma, rstd, x)
    assert torch.equal(dx[-40:], cattn.rmsnorm_bwd(x[-40:].contiguous(), gamma, want_rstd, x[-40:].contiguous())[0])
    q, scale, _, _ = cattn.rmsnorm_fwd_q8(x, gamma)
    q40, scale40, _, _ = cattn.rmsnorm_fwd_q8(x[-40:].contiguous(), gamma)
    assert torch.equal(q[-40:].view(torch.uint8), q40.view(torch.uint8)) and torch.equal(scale[-40:], scale40)


def test_repeats_bit_for_bit_and_refuses(cuda):
    x, dy = randn(gen(5), 3000, 1600).to(cuda), randn(gen(6), 3000, 1600).to(cuda)
    gamma = torch.ones(1600, device=cuda)
    y, h, rstd = cattn.rmsnorm_fwd(x, gamma, dy)
    first = cattn.rmsnorm_bwd(h, gamma, rstd, dy)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, cattn.rmsnorm_bwd(h, gamma, rstd, dy)))
    with pytest.raises(cattn.CattnError):
        cattn.rmsnorm_fwd(x[:, :12].contiguous(), gamma[:12].contiguous())
    with pytest.raises(ValueError):
        cattn.rmsnorm_fwd(x[:, :64], gamma[:64])
    with pytest.raises(TypeError):
        cattn.rmsnorm_fwd(x.half(), gamma)
    with pytest.raises(TypeError):
        cattn.rmsnorm_fwd(x, gamma.bfloat16())
    with pytest.raises(TypeError):
        cattn.rmsnorm_fwd(x, gamma, dy.bfloat16())
    with pytest.raises(ValueError):
        cattn.rmsnorm_fwd_q8(x, gamma, None, 1e-5, 24)
    with pytest.raises(ValueError):
        cattn.rmsnorm_bwd(h, gamma, rstd[:-1].contiguous(), dy)
