"""Dropout on the GPU against the float64 oracle: masks element by element, sums within their roundings."""

import numpy as np
import pytest
import torch

import oracle.ffn_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import E, TINY, TYPES, U, gen, randn, within
from parity_util import say, to64

pytestmark = pytest.mark.gpu

SEED = 0xFEDCBA9876543210


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 15, 31, 2047, 2048, 2049, 2051, 100003])
def test_forward_and_backward(cuda, n, residual, dtype):
    say(f"dropout n={n} residual={residual} {dtype}")
    g = gen(n)
    x, r, dy = randn(g, n, dtype=dtype), randn(g, n, dtype=dtype, scale=3.0) if residual else None, randn(g, n, dtype=dtype)
    p, site, step = 0.1 + 0.2 * residual, n % 7, n * (1 << 33) + 5
    y = cattn.dropout_fwd(x.to(cuda), p, SEED, site, step, None if r is None else r.to(cuda))
    dx = cattn.dropout_bwd(dy.to(cuda), p, SEED, site, step)
    keep = orc.dropout_keep(n, p, SEED, site, step)
    ref = orc.dropout(to64(x), p, SEED, site, step, None if r is None else to64(r))
    # 1 / (1 - p) rounded, the product (or the sum) rounded, then the result
    size = np.abs(to64(x)) / (1 - p) * keep
    within("y", y, ref, E * size + (E + U[dtype]) * (np.abs(ref) + E * size) + TINY)
    rdx = orc.dropout(to64(dy), p, SEED, site, step)
    within("dx", dx, rdx, (2 * E + U[dtype]) * np.abs(rdx) * 1.01 + TINY)
    assert np.array_equal(to64(dx) != 0, keep & (to64(dy) != 0))
    if residual:
        assert np.array_equal(to64(y)[~keep], to64(r)[~keep])
    else:
        assert np.array_equal(to64(y) != 0, keep & (to64(x) != 0))


@pytest.mark.parametrize("p", [0.0, 1e-9, 0.5, 0.999, 1 - 2.0 ** -32])
def test_probabilities(cuda, p):
    n = 1 << 16
    x = torch.ones(n, device=cuda)
    y = cattn.dropout_fwd(x, p, 99)
    keep = orc.dropout_keep(n, p, 99)
    assert np.array_equal((y != 0).cpu().numpy(), keep) and (y[y != 0] == np.float32(1 / (1 - p))).all()
    assert p or torch.equal(y, x)


def test_what_is_dropped_does_not_matter(cuda):
    n, p = 4099, 0.4
    keep = torch.from_numpy(orc.dropout_keep(n, p, 5)).to(cuda)
    for dtype in TYPES.values():
        x, r = torch.randn(n, device=cuda).to(dtype), torch.randn(n, device=cuda).to(dtype)
        bad = torch.where(keep, x, torch.full_like(x, float("nan")))
        bad[torch.nonzero(~keep)[0]] = float("inf")
        for res in (None, r):
            assert torch.equal(cattn.dropout_fwd(bad, p, 5, residual=res), cattn.dropout_fwd(x, p, 5, residual=res))
        assert torch.equal(cattn.dropout_bwd(bad, p, 5), cattn.dropout_bwd(x, p, 5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_shapes(cuda, dtype):
    x, r = randn(gen(1), 3, 5, 72, dtype=dtype).to(cuda), randn(gen(2), 3, 5, 72, dtype=dtype).to(cuda)
    y, alone = cattn.dropout_fwd(x, 0.3, 1, residual=r), cattn.dropout_fwd(x, 0.3, 1)
    assert y.shape == x.shape and torch.equal(cattn.dropout_fwd(x.view(-1), 0.3, 1).view(x.shape), alone)
    a, b, c = x.clone(), r.clone(), x.clone()
    assert cattn.dropout_fwd(a, 0.3, 1, residual=r, y=a) is a and torch.equal(a, y)
    assert cattn.dropout_fwd(x, 0.3, 1, residual=b, y=b) is b and torch.equal(b, y)
    assert cattn.dropout_bwd(c, 0.3, 1, dx=c) is c and torch.equal(c, alone)
    assert cattn.dropout_fwd(x[:0], 0.3, 1).shape == (0, 5, 72) and cattn.dropout_bwd(x[:0], 0.3, 1).shape == (0, 5, 72)


def test_the_step_in_device_memory(cuda):
    """A tensor's step is the number it holds when the kernel runs: a replayed graph drops anew."""
    n = 5000
    x = torch.ones(n, device=cuda, dtype=torch.bfloat16)
    step = torch.tensor([(1 << 32) - 1], device=cuda)
    for k in ((1 << 32) - 1, 1 << 32):
        step.fill_(k)
        assert torch.equal(cattn.dropout_fwd(x, 0.25, 4, 2, step), cattn.dropout_fwd(x, 0.25, 4, 2, k))
    step.fill_(10)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = cattn.dropout_fwd(x, 0.25, 4, 2, step)
        dx = cattn.dropout_bwd(y, 0.25, 4, 2, step)
        step += 1
    seen = []
    for k in range(10, 14):
        graph.replay()
        eager = cattn.dropout_fwd(x, 0.25, 4, 2, k)
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(dx, cattn.dropout_bwd(eager, 0.25, 4, 2, k))
        seen.append(y.clone())
    assert int(step) == 14 and not any(torch.equal(seen[0], s) for s in seen[1:])


def test_two_streams(cuda):
    x = randn(gen(8), 333, 1000, dtype="bf16").to(cuda)
    first = cattn.dropout_fwd(x, 0.2, 7)
    torch.cuda.synchronize()
    out = []
    for s in [torch.cuda.Stream(), torch.cuda.Stream()] * 2:
        with torch.cuda.stream(s):
            out.append(cattn.dropout_fwd(x, 0.2, 7))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in out)


def test_elements_past_32_bits_of_bytes(cuda):
    """2^31 + 13 elements: the last ones against the oracle."""
    n = (1 << 31) + 13
    x = torch.ones(n, device=cuda, dtype=torch.bfloat16)
    cattn.dropout_fwd(x, 0.5, 6, 1, 2, y=x)
    for first, m in ((0, 4000), ((1 << 31) - 4000, 4013), (1 << 30, 4000)):
        assert np.array_equal((x[first:first + m] != 0).cpu().numpy(), orc.dropout_keep(m, 0.5, 6, 1, 2, first=first))
