"""Refusals of the decoder-block entry points, on the host before any launch:
fake addresses, never dereferenced."""

import ctypes

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc
import paper_2608_00029_amd as cattn
from paper_2608_00029_amd import binding as b
from paper_2608_00029_amd import block

P = [0x10000000 * (i + 1) for i in range(12)]
BAD, NO, OK = b.CATTN_ERR_INVALID_ARG, b.CATTN_ERR_UNSUPPORTED, b.CATTN_OK


@pytest.fixture(scope="module")
def lib():
    return b.lib()


def longs(values):
    return None if values is None else (ctypes.c_longlong * len(values))(*values)


# Each helper's defaults are a call that would be launched; a test changes what makes it refused.
def norm(x=P[0], residual=P[1], gamma=P[2], y=P[3], h=P[4], rstd=P[5], rows=4, C=64, eps=1e-5, dtype=1):
    return b.lib().cattn_rmsnorm_fwd(x, residual, gamma, y, h, rstd, rows, C, eps, dtype, 0)


def norm_q8(x=P[0], residual=P[1], gamma=P[2], q=P[3], scale=P[6], h=P[4], rstd=P[5], rows=4, C=64, group=32, eps=1e-5,
            dtype=1):
    return b.lib().cattn_rmsnorm_fwd_q8(x, residual, gamma, q, scale, h, rstd, rows, C, group, eps, dtype, 0)


def norm_bwd(h=P[0], gamma=P[1], rstd=P[2], dy=P[3], dh=P[4], dx=P[5], dgamma=P[6], ws=P[7], rows=4, C=64, dtype=1):
    return b.lib().cattn_rmsnorm_bwd(h, gamma, rstd, dy, dh, dx, dgamma, ws, rows, C, dtype, 0)


def rope(q=P[0], k=P[1], qo=P[2], ko=P[3], pos=P[4], freqs=P[5], B=2, S=3, Hq=4, Hkv=2, D=64, rot=32, batched=1,
         strides=None, layout=0, interleaved=0, inverse=0, amplitude=1.0, dtype=1):
    return b.lib().cattn_rope(q, k, qo, ko, pos, freqs, B, S, Hq, Hkv, D, rot, batched, longs(strides), layout,
                              interleaved, inverse, amplitude, dtype, 0)


def append(q=P[0], k=P[1], v=P[2], qo=P[3], ko=P[4], kc=P[5], vc=P[6], lens=P[7], counts=P[8], freqs=P[9], B=2, S=3,
           Hq=4, Hkv=2, D=64, rot=32, cap=8, window=4, sinks=2, rolling=1, strides=None, layout=0, amplitude=1.0,
           dtype=1):
    return b.lib().cattn_rope_append(q, k, v, qo, ko, kc, vc, lens, counts, freqs, B, S, Hq, Hkv, D, rot, cap, window,
                                     sinks, rolling, longs(strides), layout, 0, amplitude, dtype, 0)


def swa(q=P[0], k=P[1], v=P[2], o=P[3], lse=P[4], lens=P[5], B=2, Hq=4, Hkv=2, S=40, D=64, window=8, sinks=2,
        scale=0.125, strides=None, layout=0, dtype=1):
    return b.lib().cattn_swa_fwd(q, k, v, o, lse, lens, B, Hq, Hkv, S, D, window, sinks, scale, longs(strides), layout,
                                 dtype, 0)


def swa_bwd(q=P[0], k=P[1], v=P[2], o=P[3], do=P[4], lse=P[5], lens=P[6], dq=P[7], dk=P[8], dv=P[9], ws=P[10], B=2,
            Hq=4, Hkv=2, S=40, D=64, window=8, sinks=2, scale=0.125, strides=None, layout=0, dtype=1):
    return b.lib().cattn_swa_bwd(q, k, v, o, do, lse, lens, dq, dk, dv, ws, B, Hq, Hkv, S, D, window, sinks, scale,
                                 longs(strides), layout, dtype, 0)


def decode(q=P[0], kc=P[1], vc=P[2], o=P[3], lse=P[4], lens=P[5], ws=P[6], B=2, Hq=4, Hkv=2, cap=4096, D=64, window=8,
           sinks=2, rolling=1, scale=0.125, strides=None, layout=0, dtype=1):
    return b.lib().cattn_swa_decode(q, kc, vc, o, lse, lens, ws, B, Hq, Hkv, cap, D, window, sinks, rolling, scale,
                                    longs(strides), layout, dtype, 0)


@pytest.mark.parametrize("call,changes,status", [
    (norm, dict(rows=-1), BAD), (norm, dict(C=-8), BAD), (norm, dict(dtype=2), BAD), (norm, dict(eps=-1.0), BAD),
    (norm, dict(eps=float("nan")), BAD), (norm, dict(C=60), NO), (norm, dict(C=16392), NO),
    (norm, dict(x=0), BAD), (norm, dict(h=0), BAD), (norm, dict(residual=0), BAD), (norm, dict(gamma=0), BAD),
    (norm, dict(y=P[3] + 2), BAD), (norm, dict(rstd=P[5] + 2), BAD), (norm, dict(y=P[0]), BAD), (norm, dict(h=P[1]), BAD),
    (norm, dict(y=P[4] + 16), BAD), (norm, dict(rstd=P[3] + 64), BAD),
    (norm_q8, dict(group=24), BAD), (norm_q8, dict(group=1024), BAD), (norm_q8, dict(group=-8), BAD),
    (norm_q8, dict(scale=0), BAD), (norm_q8, dict(scale=P[3] + 16), BAD),
    (norm_bwd, dict(dx=P[0]), BAD), (norm_bwd, dict(ws=0), BAD), (norm_bwd, dict(ws=P[5] + 16), BAD),
    (norm_bwd, dict(dgamma=P[6] + 4), BAD), (norm_bwd, dict(C=12), NO), (norm_bwd, dict(dtype=-1), BAD),
    (rope, dict(B=-1), BAD), (rope, dict(layout=2), BAD), (rope, dict(dtype=7), BAD), (rope, dict(rot=0), BAD),
    (rope, dict(rot=33), BAD), (rope, dict(rot=66), BAD), (rope, dict(D=514, rot=32), NO), (rope, dict(D=33), NO),
    (rope, dict(amplitude=float("inf")), BAD), (rope, dict(q=0), BAD), (rope, dict(ko=0), BAD), (rope, dict(freqs=0), BAD),
    (rope, dict(q=P[0] + 1), BAD), (rope, dict(freqs=P[5] + 4), BAD), (rope, dict(B=1 << 16, S=1 << 16), NO),
    (rope, dict(qo=P[0] + 64), BAD), (rope, dict(qo=P[1]), BAD), (rope, dict(qo=P[3]), BAD), (rope, dict(pos=P[2]), BAD),
    (rope, dict(Hq=0), BAD),
    (rope, dict(strides=[-64] + [64] * 11), BAD),
    (rope, dict(strides=[768, 192, 64, 384, 192, 64, 768, 64, 0, 384, 192, 64]), BAD),  # q_out's rows on one another
    (append, dict(cap=5), BAD), (append, dict(window=0), BAD), (append, dict(sinks=-1), BAD), (append, dict(cap=-1), BAD),
    (append, dict(window=2 ** 31 - 1), BAD), (append, dict(lens=0), BAD), (append, dict(kc=P[6]), BAD),
    (append, dict(kc=P[1]), BAD), (append, dict(vc=P[2]), BAD), (append, dict(Hkv=0), BAD), (append, dict(cap=0, rolling=0), BAD),
    (append, dict(lens=P[5]), BAD),
    (swa, dict(Hq=3), BAD), (swa, dict(Hkv=0), BAD), (swa, dict(Hq=0), BAD), (swa, dict(window=0), BAD),
    (swa, dict(sinks=-1), BAD), (swa, dict(scale=0.0), BAD), (swa, dict(scale=float("nan")), BAD), (swa, dict(scale=1e7), BAD),
    (swa, dict(D=96), NO), (swa, dict(D=0), BAD), (swa, dict(S=(1 << 26) + 1), NO), (swa, dict(B=1 << 16, Hq=1 << 14, Hkv=1), NO),
    (swa, dict(layout=3), BAD), (swa, dict(dtype=5), BAD), (swa, dict(k=0), BAD), (swa, dict(o=P[0]), BAD),
    (swa, dict(o=P[0] + 16), BAD), (swa, dict(k=P[1] + 8), BAD), (swa, dict(lse=P[3]), BAD), (swa, dict(lse=P[4] + 2), BAD),
    (swa, dict(lens=P[3] + 4), BAD),
    (swa, dict(strides=[10240, 2560, 60] + [5120, 2560, 64] * 2 + [10240, 2560, 64]), BAD),       # rows of 120 bytes
    (swa, dict(strides=[10240, 2560, 1 << 23] + [5120, 2560, 64] * 2 + [10240, 2560, 64]), NO),   # a row stride too large
    (swa_bwd, dict(dq=P[0]), BAD), (swa_bwd, dict(dk=P[9]), BAD), (swa_bwd, dict(ws=0), BAD), (swa_bwd, dict(ws=P[9] + 16), BAD),
    (swa_bwd, dict(ws=P[10] + 4), BAD), (swa_bwd, dict(do=0), BAD), (swa_bwd, dict(lse=P[7]), BAD), (swa_bwd, dict(D=32), NO),
    (swa_bwd, dict(B=64, Hq=8, Hkv=8, S=1 << 23, sinks=1 << 23), NO), (swa_bwd, dict(B=4, Hq=8, Hkv=8, S=1 << 19, sinks=1 << 19), NO),
    (swa_bwd, dict(B=1 << 20, Hq=12, Hkv=12, S=2, window=1, sinks=1), NO),
    (swa, dict(B=64, Hq=8, Hkv=8, S=1 << 20), NO), (decode, dict(B=1 << 20, Hq=16, Hkv=1), NO),
    (decode, dict(cap=9), BAD), (decode, dict(ws=0, window=4000, sinks=0), BAD), (decode, dict(lens=0), BAD), (decode, dict(o=P[0]), BAD),
    (decode, dict(cap=0, rolling=0), BAD), (decode, dict(Hq=5), BAD), (decode, dict(ws=P[3], window=4000), BAD),
    (decode, dict(cap=-1), BAD),
])
def test_refusals(lib, call, changes, status):
    assert call(**changes) == status, b.last_error_string()
    assert b.last_error_string() != ""


@pytest.mark.parametrize("call,changes", [
    (norm, dict(rows=0)), (norm, dict(C=0)), (norm_q8, dict(rows=0)), (norm_bwd, dict(rows=0)),
    (rope, dict(B=0)), (rope, dict(S=0)), (append, dict(B=0)), (append, dict(S=0)),
    (swa, dict(B=0)), (swa, dict(S=0)), (swa_bwd, dict(B=0)), (decode, dict(B=0)),
])
def test_empty_problems(lib, call, changes):
    assert call(**changes) == OK


def test_views_of_one_allocation_are_told_apart(lib):
    """Outputs that are other heads' columns of the allocation that holds the inputs are not an overlap;
    shared columns are.  (The NULL freqs / workspace makes a call that passes the check refused after it.)"""
    B, S, Hq, Hkv, D = 2, 3, 4, 2, 64
    row = (Hq + 2 * Hkv) * D
    st = [S * row, D, row]
    q, k = P[0], P[0] + Hq * D * 2
    assert rope(q=q, k=k, qo=q, ko=k, strides=st * 4, layout=1, pos=q + 64) == BAD
    assert "an output overlaps an input" in b.last_error_string()  # the positions, not the views
    assert rope(q=q, k=k, qo=q, ko=k + D * 2, strides=st * 4, layout=1) == BAD
    assert "overlaps" in b.last_error_string()
    # q_out one head further: in place no more, and on other heads' inputs
    assert rope(q=q, k=k, qo=q + D * 2, ko=k, strides=st * 4, layout=1) == BAD
    # heads-major views of one allocation [B, Hq + 2 Hkv, S, D]
    hm = [(Hq + 2 * Hkv) * S * D, S * D, D]
    assert rope(q=q, k=q + Hq * S * D * 2, qo=q, ko=q + Hq * S * D * 2, strides=hm * 4, pos=q + 64) == BAD
    assert "an output overlaps an input" in b.last_error_string()


def test_workspace_sizes(lib):
    assert cattn.rmsnorm_bwd_workspace_bytes(10000, 64) == 512 * 64 * 4
    assert cattn.rmsnorm_bwd_workspace_bytes(9, 64) == 3 * 64 * 4 and cattn.rmsnorm_bwd_workspace_bytes(0, 64) == 0
    assert cattn.rmsnorm_bwd_workspace_bytes(9, 4096) == 9 * 4096 * 4
    rows = 2 * 2 * 4 * 64 * 4
    assert cattn.swa_bwd_workspace_bytes(2, 4, 2, 40, 64, 40, 2) == rows  # the window covers the sequence
    assert cattn.swa_bwd_workspace_bytes(2, 4, 2, 40, 64, 8, 0) == rows   # no sinks
    assert cattn.swa_bwd_workspace_bytes(2, 4, 2, 40, 64, 8, 2) == rows   # few queries that only the sinks see
    rows = 2 * 2 * 4 * 608 * 4
    assert cattn.swa_bwd_workspace_bytes(2, 4, 2, 600, 64, 400, 2) == rows
    far = cattn.swa_bwd_workspace_bytes(2, 4, 2, 600, 64, 8, 2) - rows
    assert far > 0 and far % (2 * 2 * 2 * 32 * 64 * 4) == 0
    assert cattn.swa_bwd_workspace_bytes(2, 4, 2, 600, 64, 8, 2 ** 40) > rows  # clamped to the sequence
    assert cattn.swa_bwd_workspace_bytes(2, 3, 2, 40, 64, 8, 2) == 0
    assert cattn.swa_decode_workspace_bytes(300, 8, 8, 4096, 64, 4000) == 0  # work groups enough without parts
    for dtype in (torch.float32, torch.bfloat16):
        one = cattn.swa_decode_workspace_bytes(1, 8, 2, 4096, 64, 4000, 0, dtype)
        assert one > 0 and one % (8 * 66 * 4) == 0
        assert cattn.swa_decode_workspace_bytes(1, 8, 2, 4096, 64, 200, 50, dtype) == 0  # few slots
    assert cattn.swa_decode_workspace_bytes(40, 8, 2, 4096, 64, 4000, 0, torch.bfloat16) == 0
    few, either = (cattn.swa_decode_workspace_bytes(40, 8, 2, 4096, 64, 4000, 0, t) for t in (torch.float32, None))
    assert few == either == 3 * 40 * 8 * 66 * 4


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=3.0), dict(scaling="ntk", factor=8.0, base=5e5),
                                dict(scaling="ramp", factor=8.0, context=8192.0),
                                dict(scaling="ramp", factor=4.0, context=1000.0, low=1.0, high=4.0)])
@pytest.mark.parametrize("rot", [4, 24, 128])
def test_rope_frequencies(lib, rot, kw):
    f = cattn.rope_frequencies(rot, **kw)
    assert f.dtype == torch.float64 and f.shape == (rot // 2,)
    # pow is within an ulp or two; the blend cancels nothing
    assert np.allclose(f.numpy(), orc.rope_frequencies(rot, **kw), rtol=1e-14, atol=0)


def test_rope_frequencies_refusals(lib):
    for kw in (dict(rot=0), dict(rot=7), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, scaling="linear", factor=0.5),
               dict(rot=2, scaling="ntk", factor=2.0), dict(rot=8, scaling="ramp", factor=2.0),
               dict(rot=8, scaling="ramp", factor=2.0, context=100.0, low=3.0, high=3.0), dict(rot=8, base=float("nan"))):
        with pytest.raises(cattn.CattnError):
            cattn.rope_frequencies(**kw)
    with pytest.raises(ValueError):
        cattn.rope_frequencies(8, scaling="other")


def test_binding_refuses_host_tensors(lib):
    t = torch.zeros(2, 4, 8, 64)
    f = cattn.rope_frequencies(64)
    n = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: cattn.rmsnorm_fwd(t, torch.ones(64)), lambda: cattn.rmsnorm_fwd_q8(t, torch.ones(64)),
                 lambda: cattn.rmsnorm_bwd(t, torch.ones(64), torch.ones(64), t), lambda: cattn.rope_fwd(t, t, f),
                 lambda: cattn.rope_append(t, t, t, t, t, n, f), lambda: cattn.swa_fwd(t, t, t, 0.1, 4),
                 lambda: cattn.swa_bwd(t, t, t, t, t, t[..., 0], 0.1, 4), lambda: cattn.swa_decode(t[:, :, 0], t, t, n, 0.1, 4)):
        with pytest.raises(ValueError, match="HIP device"):
            call()


def test_strides_argument():
    """What the binding hands over: nothing for contiguous tensors, else batch, head and row strides."""
    qkv = torch.zeros(2, 5, 8, 64)
    q, k = qkv[:, :, :4], qkv[:, :, 4:6]
    o = torch.zeros(2, 5, 4, 64)
    assert block._strides((qkv, o), "bshd") is None
    assert list(block._strides((q, k, o), "bshd")) == [2560, 64, 512, 2560, 64, 512, 1280, 64, 256]
    assert list(block._strides((q.transpose(1, 2),), "bhsd")) == [2560, 64, 512]
    assert list(block._strides((q[:, 0],), "bhsd")) == [2560, 64, 0]
