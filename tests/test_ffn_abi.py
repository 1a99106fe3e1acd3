"""Refusals of the feed-forward entry points, on the host before any launch (fake addresses, never dereferenced), and
what the Python entry points refuse."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from paper_2608_00029_amd import binding as b
from paper_2608_00029_amd import ffn

P = [0x10000000 * (i + 1) for i in range(12)]
BAD, NO, OK = b.CATTN_ERR_INVALID_ARG, b.CATTN_ERR_UNSUPPORTED, b.CATTN_OK
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    return b.lib()


# Each helper's defaults are a call that would be launched; a test changes what makes it refused.
def gated(x=P[0], wg=P[1], wu=P[2], h=P[3], gate=P[4], up=P[5], T=4, C=64, F=32, act=0, dtype=1):
    return b.lib().cattn_gated_fwd(x, wg, wu, h, gate, up, T, C, F, act, dtype, 0)


def gated_bwd(x=P[0], wg=P[1], wu=P[2], gate=P[3], up=P[4], dh=P[5], dx=P[6], dwg=P[7], dwu=P[8], ws=P[9], T=4, C=64, F=32,
              act=0, dtype=1):
    return b.lib().cattn_gated_bwd(x, wg, wu, gate, up, dh, dx, dwg, dwu, ws, T, C, F, act, dtype, 0)


def dropout(x=P[0], r=P[1], y=P[2], n=100, p=0.1, seed=1, site=2, step=3, at=P[3], dtype=1):
    return b.lib().cattn_dropout_fwd(x, r, y, n, p, seed, site, step, at, dtype, 0)


def dropout_bwd(dy=P[0], dx=P[2], n=100, p=0.1, seed=1, site=2, step=3, at=P[3], dtype=1):
    return b.lib().cattn_dropout_bwd(dy, dx, n, p, seed, site, step, at, dtype, 0)


@pytest.mark.parametrize("call,changes,status", [
    (gated, dict(T=-1), BAD), (gated, dict(C=-8), BAD), (gated, dict(F=-8), BAD), (gated, dict(dtype=2), BAD),
    (gated, dict(act=2), BAD), (gated, dict(act=-1), BAD), (gated, dict(C=60), NO), (gated, dict(F=36), NO),
    (gated, dict(C=(1 << 18) + 8), NO), (gated, dict(F=(1 << 18) + 8), NO), (gated, dict(T=1 << 30, C=16, F=8), NO),
    (gated, dict(T=1 << 30, C=8, F=16), NO), (gated, dict(T=1, C=1 << 17, F=(1 << 16) + 8), NO), (gated, dict(x=0), BAD), (gated, dict(wg=0), BAD), (gated, dict(wu=0), BAD),
    (gated, dict(h=0), BAD), (gated, dict(gate=0), BAD), (gated, dict(up=0), BAD), (gated, dict(x=P[0] + 8), BAD),
    (gated, dict(gate=P[4] + 2), BAD), (gated, dict(h=P[0]), BAD), (gated, dict(h=P[1] + 4080), BAD), (gated, dict(gate=P[5] + 16), BAD),
    (gated, dict(up=P[3] + 240), BAD), (gated, dict(gate=P[2]), BAD),
    (gated_bwd, dict(T=-1), BAD), (gated_bwd, dict(act=3), BAD), (gated_bwd, dict(dtype=-1), BAD), (gated_bwd, dict(C=4), NO),
    (gated_bwd, dict(ws=0), BAD), (gated_bwd, dict(dh=0), BAD), (gated_bwd, dict(dwu=0), BAD), (gated_bwd, dict(ws=P[9] + 4), BAD),
    (gated_bwd, dict(dx=P[0]), BAD), (gated_bwd, dict(dwg=P[1]), BAD), (gated_bwd, dict(dwu=P[7] + 16), BAD),
    (gated_bwd, dict(ws=P[5]), BAD), (gated_bwd, dict(ws=P[6] + 64), BAD), (gated_bwd, dict(dx=P[3]), BAD),
    (dropout, dict(n=-1), BAD), (dropout, dict(dtype=3), BAD), (dropout, dict(p=-0.1), BAD), (dropout, dict(p=1.0), BAD),
    (dropout, dict(p=NAN), BAD), (dropout, dict(p=1 - 2.0 ** -33), BAD), (dropout, dict(n=(1 << 33) + 1), NO),
    (dropout, dict(x=0), BAD), (dropout, dict(y=0), BAD), (dropout, dict(x=P[0] + 2), BAD), (dropout, dict(r=P[1] + 8), BAD),
    (dropout, dict(y=P[2] + 4), BAD), (dropout, dict(at=P[3] + 4), BAD), (dropout, dict(y=P[0] + 16), BAD),
    (dropout, dict(y=P[1] - 16), BAD), (dropout, dict(at=P[2] + 8), BAD),
    (dropout_bwd, dict(dx=P[0] + 16), BAD), (dropout_bwd, dict(dy=0), BAD), (dropout_bwd, dict(p=1.5), BAD),
    (dropout_bwd, dict(dtype=-1), BAD),
])
def test_refusals(lib, call, changes, status):
    assert call(**changes) == status, b.last_error_string()
    assert b.last_error_string() != ""


@pytest.mark.parametrize("call,changes", [
    (gated, dict(T=0)), (gated, dict(C=0)), (gated, dict(F=0)), (gated_bwd, dict(T=0)), (gated_bwd, dict(C=0)),
    (gated_bwd, dict(F=0)), (dropout, dict(n=0)), (dropout_bwd, dict(n=0)), (gated, dict(T=0, x=0, h=0)), (dropout, dict(n=0, x=0, y=0)),
])
def test_empty_problems(lib, call, changes):
    assert call(**changes) == OK


def test_workspaces(lib):
    f = lib.cattn_gated_bwd_workspace_bytes
    assert f(100, 64, 32, b.CATTN_BF16) >= 2 * 100 * 32 * 2 and f(100, 64, 32, b.CATTN_F32) >= 2 * 100 * 32 * 4
    for T, C, F, dtype in ((0, 64, 32, 1), (-1, 64, 32, 1), (4, 60, 32, 1), (4, 64, 36, 1), (4, 64, 32, 2), (1 << 30, 64, 64, 1),
                           (4, 1 << 19, 32, 1)):
        assert f(T, C, F, dtype) == 0
    big = 1 << 32
    assert cattn.gated_bwd_workspace_bytes(big + 4, 64, 32) == cattn.gated_bwd_workspace_bytes(4, big + 64, 32) == 0
    assert cattn.gated_bwd_workspace_bytes(4, 64, 32, torch.bfloat16) == f(4, 64, 32, 1)


BF, F32 = torch.bfloat16, torch.float32


def t(*shape, dtype=BF):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.fixture
def host(monkeypatch):
    """The Python entry points as they are, but for the device they ask for and the stream."""
    def run(where, device, *args):
        st = getattr(b.lib(), where)(*args, 0)
        if st != OK:
            raise cattn.CattnError(st, where, b.last_error_string())
    monkeypatch.setattr(ffn, "_on_hip", lambda name, x: None)
    monkeypatch.setattr(ffn, "_run", run)


def call_fwd(T=4, C=64, F=32):
    return cattn.gated_fwd(t(T, C), t(F, C), t(F, C))


def call_bwd(T=4, C=64, F=32):
    return cattn.gated_bwd(t(T, C), t(F, C), t(F, C), t(T, F), t(T, F), t(T, F))


WRAP = 1 << 32


@pytest.mark.parametrize("call,sizes", [(c, s) for c in (call_fwd, call_bwd) for s in (dict(T=WRAP + 4), dict(C=WRAP + 64), dict(F=WRAP + 32))]
                         + [(lambda n: cattn.dropout_fwd(t(n), 0.1, 1), dict(n=WRAP * 4)),
                            (lambda n: cattn.dropout_bwd(t(n), 0.1, 1), dict(n=WRAP * 4))])
def test_sizes_beyond_an_int_are_refused(host, call, sizes):
    with pytest.raises(cattn.CattnError) as e:
        call(**sizes)
    assert "NULL" not in str(e.value)


def test_the_calls_are_otherwise_taken(host):
    for call in (call_fwd, call_bwd, lambda: cattn.dropout_fwd(t(9), 0.1, 1), lambda: cattn.dropout_bwd(t(9), 0.1, 1)):
        with pytest.raises(cattn.CattnError, match="NULL"):
            call()


def test_python_refusals(host):
    x, w, h = t(4, 64), t(32, 64), t(4, 32)
    for bad, err in [
        (lambda: cattn.gated_fwd(x, w, w, "relu"), ValueError), (lambda: cattn.gated_fwd(x, w, t(24, 64)), ValueError),
        (lambda: cattn.gated_fwd(x, w, t(32, 64, dtype=F32)), TypeError), (lambda: cattn.gated_fwd(x, t(64), w), TypeError),
        (lambda: cattn.gated_fwd(t(4, 64, dtype=torch.float16), w, w), TypeError), (lambda: cattn.gated_fwd(t(64, 4).t(), w, w), ValueError),
        (lambda: cattn.gated_fwd(x, t(64, 32).t(), w), ValueError), (lambda: cattn.gated_fwd(x, w, None), TypeError),
        (lambda: cattn.gated_fwd(t(), w, w), ValueError),
        (lambda: cattn.gated_bwd(x, w, w, None, h, h), TypeError), (lambda: cattn.gated_bwd(x, w, w, h, h, t(4, 24)), ValueError),
        (lambda: cattn.gated_bwd(x, w, w, h, h, h, workspace=t(8, dtype=F32)), ValueError),
        (lambda: cattn.gated_bwd_workspace_bytes(4, 64, 32, torch.float16), KeyError),
        (lambda: cattn.dropout_fwd(x, 0.1, -1), ValueError), (lambda: cattn.dropout_fwd(x, 0.1, 1 << 64), ValueError),
        (lambda: cattn.dropout_fwd(x, 0.1, 1.5), ValueError), (lambda: cattn.dropout_fwd(x, 0.1, 1, site=1 << 32), ValueError),
        (lambda: cattn.dropout_fwd(x, 0.1, 1, step=-1), ValueError), (lambda: cattn.dropout_fwd(x, 0.1, 1, step=t(2, dtype=torch.int64)), ValueError),
        (lambda: cattn.dropout_fwd(x, 0.1, 1, step=t(1, dtype=torch.int32)), TypeError), (lambda: cattn.dropout_fwd(x.t(), 0.1, 1), ValueError),
        (lambda: cattn.dropout_fwd(x, 0.1, 1, residual=h), ValueError), (lambda: cattn.dropout_bwd(x, 0.1, 1, dx=h), ValueError),
        (lambda: cattn.dropout_fwd(t(4, 64, dtype=torch.float16), 0.1, 1), TypeError),
    ]:
        with pytest.raises(err):
            bad()


def test_tensors_on_the_host_are_refused():
    x, w, h = torch.ones(4, 64), torch.ones(32, 64), torch.ones(4, 32)
    for call in (lambda: cattn.gated_fwd(x, w, w), lambda: cattn.gated_bwd(x, w, w, h, h, h), lambda: cattn.dropout_fwd(x, 0.1, 1),
                 lambda: cattn.dropout_bwd(x, 0.1, 1)):
        with pytest.raises(ValueError, match="HIP device"):
            call()
