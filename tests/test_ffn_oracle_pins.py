"""What pins the feed-forward operators' oracle: closed forms, published vectors, central differences, torch's
float64 autograd, planted mistakes."""

import numpy as np
import pytest
import torch

import oracle.ffn_oracle as orc


def data(T=5, C=7, F=6, seed=0):
    g = np.random.default_rng(seed)
    return g.standard_normal((T, C)), g.standard_normal((F, C)), g.standard_normal((F, C)), g.standard_normal((T, F))


def test_closed_forms():
    """act(0) = 0, act'(0) = 1/2, act -> identity and 0 far out; silu(ln 3) = 3/4 ln 3."""
    for kind in ("silu", "gelu"):
        assert orc.activation(0.0, kind) == 0 and orc.slope(0.0, kind) == 0.5
        assert orc.activation(50.0, kind) == 50 and orc.slope(50.0, kind) == pytest.approx(1, abs=1e-15)
        assert abs(orc.activation(-50.0, kind)) < 1e-19 and abs(orc.slope(-50.0, kind)) < 1e-19
    assert orc.activation(np.log(3.0), "silu") == pytest.approx(0.75 * np.log(3.0), rel=1e-15)
    assert orc.slope(np.log(3.0), "silu") == pytest.approx(0.75 + np.log(3.0) * 3 / 16, rel=1e-15)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activations_against_torch_and_differences(kind):
    g = np.linspace(-8, 8, 401)
    t = torch.tensor(g)
    ref = torch.nn.functional.silu(t) if kind == "silu" else torch.nn.functional.gelu(t, approximate="tanh")
    assert np.allclose(orc.activation(g, kind), ref.numpy(), rtol=0, atol=1e-14)
    d = 1e-6
    fd = (orc.activation(g + d, kind) - orc.activation(g - d, kind)) / (2 * d)
    assert np.allclose(orc.slope(g, kind), fd, rtol=0, atol=1e-8)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gradients_against_differences_and_autograd(kind):
    x, wg, wu, dh = data()
    h, gate, up = orc.gated_fwd(x, wg, wu, kind)
    grads = orc.gated_bwd(x, wg, wu, gate, up, dh, kind)
    for t, grad in zip((x, wg, wu), grads):
        for i in np.ndindex(t.shape):
            keep, d = t[i], 1e-6
            t[i] = keep + d
            hi = np.sum(orc.gated_fwd(x, wg, wu, kind)[0] * dh)
            t[i] = keep - d
            lo = np.sum(orc.gated_fwd(x, wg, wu, kind)[0] * dh)
            t[i] = keep
            assert (hi - lo) / (2 * d) == pytest.approx(grad[i], rel=1e-6, abs=1e-7)
    tx, tg, tu = (torch.tensor(t, requires_grad=True) for t in (x, wg, wu))
    a = torch.nn.functional.silu(tx @ tg.T) if kind == "silu" else torch.nn.functional.gelu(tx @ tg.T, approximate="tanh")
    out = a * (tx @ tu.T)
    assert np.allclose(h, out.detach().numpy(), rtol=0, atol=1e-12)
    out.backward(torch.tensor(dh))
    for t, grad in zip((tx, tg, tu), grads):
        assert np.allclose(grad, t.grad.numpy(), rtol=0, atol=1e-12)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_planted_mistakes_are_seen(kind):
    x, wg, wu, dh = data(seed=1)
    h, gate, up = orc.gated_fwd(x, wg, wu, kind)
    dx, dwg, dwu = orc.gated_bwd(x, wg, wu, gate, up, dh, kind)
    tol = 1e-3
    assert np.abs(h - orc.gated_fwd(x, wu, wg, kind)[0]).max() > tol                               # roles exchanged
    assert np.abs(h - gate * up).max() > tol                                                       # no activation
    assert np.abs(dwg - (dh * orc.slope(gate, kind)).T @ x).max() > tol                            # u left out of dg
    assert np.abs(dwu - (dh * up).T @ x).max() > tol                                               # act left out of du
    assert np.abs(dx - (dh * up * orc.slope(gate, kind)) @ wg).max() > tol                         # half of dx
    assert np.abs(orc.slope(gate, "silu") - orc.slope(gate, "gelu")).max() > tol
    assert np.abs(dwg - (dh * up * orc.activation(gate, kind) / gate).T @ x).max() > tol           # slope without its second term


def test_philox_published_vectors():
    """The known answers that the generator's authors publish for ten rounds."""
    for c, k, want in [
        ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
        ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
        ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
         [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
    ]:
        assert [int(v) for v in orc.philox(c, k)] == want


def test_dropout():
    n, p = 40000, 0.3
    keep = orc.dropout_keep(n, p, 12345, 7, 1 << 40)
    # 40000 draws: a standard deviation of 0.0023
    assert abs(keep.mean() - 0.7) < 0.0115
    others = [orc.dropout_keep(n, p, 12346, 7, 1 << 40), orc.dropout_keep(n, p, 12345 + (1 << 32), 7, 1 << 40),
              orc.dropout_keep(n, p, 12345, 8, 1 << 40), orc.dropout_keep(n, p, 12345, 7, (1 << 40) + 1),
              orc.dropout_keep(n, p, 12345, 7, 1)]
    for o in others:  # independent masks agree in 0.7^2 + 0.3^2 of the places
        assert abs((keep == o).mean() - 0.58) < 0.0125
    assert np.array_equal(orc.dropout_keep(96, p, 12345, 7, 1 << 40, first=400), keep[400:496])
    assert orc.dropout_keep(100, 0.0, 3).all() and not orc.dropout_keep(100, 1 - 2.0 ** -32, 3).any()
    x, r = np.arange(1.0, 9.0), np.full(8, 100.0)
    y = orc.dropout(x, 0.5, 9, residual=r)
    assert set((y - r) / x) <= {0.0, 2.0} and np.array_equal(y - r, orc.dropout(x, 0.5, 9))
