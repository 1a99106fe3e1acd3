"""Pins of the decoder-block oracle: closed forms, differences, an independent
implementation (torch in float64 with autograd) and planted mistakes."""

import math

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc

rng = np.random.default_rng(7)


def difference(f, x, w, eps=1e-6):
    """Central differences of sum(w f(x)) for every entry of x."""
    g = np.empty_like(x)
    for i in np.ndindex(*x.shape):
        old = x[i]
        x[i] = old + eps
        hi = np.sum(w * f(x))
        x[i] = old - eps
        lo = np.sum(w * f(x))
        x[i] = old
        g[i] = (hi - lo) / (2 * eps)
    return g


def test_rmsnorm_closed_forms():
    y, h, rstd = orc.rmsnorm_fwd([[3.0, 4.0]], [1.0, 2.0], eps=0.0)
    assert np.allclose(rstd, 1 / math.sqrt(12.5)) and np.allclose(y, [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]])
    x, r = rng.standard_normal((2, 3, 8))
    y, h, _ = orc.rmsnorm_fwd(x, np.ones(8), r, 0.0)
    assert np.allclose(h, x + r) and np.allclose((y * y).mean(1), 1.0)


def test_rmsnorm_backward_by_differences():
    x, dy = rng.standard_normal((2, 3, 8))
    gamma, dh = 1 + 0.3 * rng.standard_normal(8), rng.standard_normal((3, 8))
    _, h, rstd = orc.rmsnorm_fwd(x, gamma)
    dx, dgamma = orc.rmsnorm_bwd(h, gamma, rstd, dy, dh)
    assert np.allclose(dx - dh, difference(lambda t: orc.rmsnorm_fwd(t, gamma)[0], x.copy(), dy), atol=1e-7)
    assert np.allclose(dgamma, difference(lambda t: orc.rmsnorm_fwd(x, t)[0], gamma.copy(), dy), atol=1e-7)
    # planted: the mean without xhat, a missing gamma
    xhat, g = h * rstd[:, None], dy * gamma
    assert not np.allclose(dx - dh, rstd[:, None] * (g - g.mean(1, keepdims=True)))
    assert not np.allclose(dx - dh, rstd[:, None] * (dy - xhat * (dy * xhat).mean(1, keepdims=True)))


def test_q8_scales():
    y = np.array([[1.0, -448.0, 2.0, 0.0, 0.0, 0.0]])
    assert np.allclose(orc.q8_scales(y, 2), [[1.0, 2 / 448, 2.0 ** -126]]) and np.allclose(orc.q8_scales(y), [[1.0]])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_turns(interleaved):
    f = orc.rope_frequencies(8)
    assert f[0] == 1.0 and np.allclose(f[1], 10000 ** -0.25)
    x = rng.standard_normal((1, 2, 3, 12))
    pos = np.array([[0, 5, 11]])
    y = orc.rope(x, pos, f, interleaved)
    assert np.array_equal(y[:, :, 0], x[:, :, 0]) and np.array_equal(y[..., 8:], x[..., 8:])
    assert np.allclose((y * y).sum(-1), (x * x).sum(-1))
    assert np.allclose(orc.rope(y, pos, f, interleaved, inverse=True), x)
    # the product of a query and a key depends on the distance of their positions alone
    q, k = rng.standard_normal((2, 1, 1, 1, 8))
    d = [np.sum(orc.rope(q, [[p + 3]], f, interleaved) * orc.rope(k, [[p]], f, interleaved)) for p in (0, 1000)]
    assert np.allclose(d[0], d[1])
    # one pair as a complex product
    a, b = (0, 1) if interleaved else (0, 4)
    z = (x[0, 0, 1, a] + 1j * x[0, 0, 1, b]) * np.exp(5j)
    assert np.allclose([y[0, 0, 1, a], y[0, 0, 1, b]], [z.real, z.imag])


def test_rope_scalings():
    f = orc.rope_frequencies(16)
    assert np.allclose(orc.rope_frequencies(16, scaling="linear", factor=4), f / 4)
    ntk = orc.rope_frequencies(16, scaling="ntk", factor=4)
    assert ntk[0] == 1.0 and np.allclose(ntk[-1], f[-1] / 4)  # the slowest pair as if interpolated
    ramp = orc.rope_frequencies(16, scaling="ramp", factor=4, context=1000, low=1, high=16)
    turns = 1000 * f / (2 * np.pi)
    assert np.allclose(ramp[turns >= 16], f[turns >= 16]) and np.allclose(ramp[turns <= 1], f[turns <= 1] / 4)
    assert ((ramp <= f + 1e-18) & (ramp >= f / 4 - 1e-18)).all()


def test_rolling_cache_holds_what_a_window_sees():
    for n in (0, 1, 4, 5, 9, 10, 23):
        held = orc.cache_slots(n, 9, window=5, sinks=4, rolling=True)
        assert sorted(held) == (list(np.flatnonzero(orc.visible(n, 5, 4)[n - 1])) if n else [])
        assert sorted(held.values()) == list(range(len(held)))  # the first slots, each once


def test_visible():
    want = ["1......", "11.....", "111....", "1111...", "1.111..", "1..111.", "1...111"]
    assert ["".join("1" if x else "." for x in row) for row in orc.visible(7, 3, 1)] == want
    assert np.array_equal(orc.visible(9, 9, 0), np.tril(np.ones((9, 9), bool)))
    assert np.array_equal(orc.visible(9, 1, 0), np.eye(9, dtype=bool))


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 2), (4, 20), (20, 0)])
def test_swa_against_torch(window, sinks):
    B, Hq, Hkv, S, D = 2, 4, 2, 11, 4
    lens = [11, 7]
    q, do = (torch.from_numpy(rng.standard_normal((B, Hq, S, D))) for _ in range(2))
    k, v = (torch.from_numpy(rng.standard_normal((B, Hkv, S, D))) for _ in range(2))
    r = orc.swa(q, k, v, 0.6, window, sinks, lens, do)
    for b, n in enumerate(lens):
        qq, kk, vv = (t[b, :, :n].clone().requires_grad_() for t in (q, k, v))
        z = 0.6 * qq @ kk.repeat_interleave(2, 0).transpose(1, 2)
        z = z.masked_fill(~torch.from_numpy(orc.visible(n, window, sinks)), -math.inf)
        o = torch.softmax(z, -1) @ vv.repeat_interleave(2, 0)
        (o * do[b, :, :n]).sum().backward()
        assert np.allclose(r["o"][b, :, :n], o.detach()) and np.allclose(r["lse"][b, :, :n], z.logsumexp(-1).detach())
        for name, t in (("dq", qq), ("dk", kk), ("dv", vv)):
            assert np.allclose(r[name][b, :, :n], t.grad), name
            assert not r[name][b, :, n:].any()
        assert not r["o"][b, :, n:].any() and np.isneginf(r["lse"][b, :, n:]).all()
    for m, t in (("m_o", "o"), ("m_dv", "dv")):
        assert (np.abs(r[t]) <= r[m] + 1e-12).all()
    assert (np.abs(r["dq"]) <= 0.6 * r["g_dq"] + 1e-12).all() and (np.abs(r["dk"]) <= 0.6 * r["g_dk"] + 1e-12).all()


def test_swa_backward_by_differences():
    q, do = (rng.standard_normal((1, 2, 6, 3)) for _ in range(2))
    k, v = (rng.standard_normal((1, 1, 6, 3)) for _ in range(2))
    r = orc.swa(q, k, v, 0.7, 2, 1, do=do)
    f = lambda q_, k_, v_: orc.swa(q_, k_, v_, 0.7, 2, 1)["o"]  # noqa: E731
    assert np.allclose(r["dq"], difference(lambda t: f(t, k, v), q.copy(), do), atol=1e-7)
    assert np.allclose(r["dk"], difference(lambda t: f(q, t, v), k.copy(), do), atol=1e-7)
    assert np.allclose(r["dv"], difference(lambda t: f(q, k, t), v.copy(), do), atol=1e-7)


def test_decode_is_the_last_row():
    q, k, v = rng.standard_normal((1, 4, 9, 4)), rng.standard_normal((1, 2, 9, 4)), rng.standard_normal((1, 2, 9, 4))
    r = orc.swa(q, k, v, 0.5, 4, 2)
    o, lse, _ = orc.swa_decode(q[0, :, 8], k[0], v[0], 0.5, 4, 2)
    assert np.allclose(o, r["o"][0, :, 8]) and np.allclose(lse, r["lse"][0, :, 8])


def test_planted_masks_are_caught():
    q, k, v = (rng.standard_normal((1, 1, 9, 4)) for _ in range(3))
    good = orc.swa(q, k, v, 0.5, 3, 1)["o"]
    for window, sinks in ((4, 1), (2, 1), (3, 0), (3, 2)):  # off by one at either end, sinks left out or one more
        assert not np.allclose(good, orc.swa(q, k, v, 0.5, window, sinks)["o"])
