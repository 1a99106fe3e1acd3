"""Sizes beyond a C int, at the Python entry points of the decoder-block operators: refused, never cut to their
low 32 bits.  Tensors without memory; the library refuses the sizes before it looks at an address."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from paper_2608_00029_amd import binding, block

BF, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
WRAP = 1 << 32  # and a size of its own left in the low 32 bits


def t(*shape, dtype=BF):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.fixture
def host(monkeypatch):
    """The entry points as they are, but for the device they ask for and the stream."""
    def run(where, device, *args):
        st = getattr(binding.lib(), where)(*args, 0)
        if st != binding.CATTN_OK:
            raise cattn.CattnError(st, where, binding.last_error_string())
    monkeypatch.setattr(block, "_on_hip", lambda name, x: None)
    monkeypatch.setattr(block, "_run", run)


def append(B=2, Hq=2, Hkv=1, S=1, D=2, cap=8, rot=2, **kw):
    k = t(B, Hkv, S, D)
    return cattn.rope_append(t(B, Hq, S, D), k, k, t(B, Hkv, cap, D), t(B, Hkv, cap, D), t(B, dtype=I32), t(rot // 2, dtype=F64), **kw)


def decode(B=2, Hq=2, Hkv=1, cap=64, D=64):
    return cattn.swa_decode(t(B, Hq, D), t(B, Hkv, cap, D), t(B, Hkv, cap, D), t(B, dtype=I32), 0.125, 8)


def swa(B=2, Hq=2, Hkv=1, S=4, D=64):
    return cattn.swa_fwd(t(B, Hq, S, D), t(B, Hkv, S, D), t(B, Hkv, S, D), 0.125, 8)


def swa_bwd(B=2, Hq=2, Hkv=1, S=4, D=64):
    q, k = t(B, Hq, S, D), t(B, Hkv, S, D)
    return cattn.swa_bwd(q, k, k, q, q, t(B, Hq, S, dtype=F32), 0.125, 8, 2)


def rope(B=2, Hq=2, Hkv=1, S=4, D=2, rot=2):
    return cattn.rope_fwd(t(B, Hq, S, D), t(B, Hkv, S, D), t(rot // 2, dtype=F64))


def norm(R=2, C=64):
    return cattn.rmsnorm_fwd(t(R, C), t(C, dtype=F32))


def norm_q8(R=2, C=64):
    return cattn.rmsnorm_fwd_q8(t(R, C), t(C, dtype=F32))


def norm_bwd(R=2, C=64):
    return cattn.rmsnorm_bwd(t(R, C), t(C, dtype=F32), t(R, dtype=F32), t(R, C))


@pytest.mark.parametrize("call,sizes", [
    (norm, dict(C=WRAP + 64)), (norm, dict(R=WRAP + 2)), (norm_q8, dict(C=WRAP + 64)), (norm_bwd, dict(C=WRAP + 64)),
    (norm_bwd, dict(R=WRAP + 2)),
    (rope, dict(B=WRAP + 2)), (rope, dict(Hq=WRAP + 2)), (rope, dict(Hkv=WRAP + 1)), (rope, dict(S=WRAP + 4)),
    (rope, dict(D=WRAP + 2)), (rope, dict(rot=WRAP + 2)),
    (append, dict(B=WRAP + 2)), (append, dict(Hq=WRAP + 2)), (append, dict(Hkv=WRAP + 1)), (append, dict(S=WRAP + 1)),
    (append, dict(D=WRAP + 2)), (append, dict(rot=WRAP + 2)),
    (append, dict(cap=WRAP + 8)), (append, dict(cap=1 << 31)),  # (taken as 2^31 - 1, a sequence's cache would begin too early)
    (swa, dict(B=WRAP + 2)), (swa, dict(Hq=WRAP + 2)), (swa, dict(Hq=WRAP + 2, Hkv=WRAP + 2)), (swa, dict(S=WRAP + 4)),
    (swa, dict(D=WRAP + 64)),
    (swa_bwd, dict(B=WRAP + 2)), (swa_bwd, dict(Hq=WRAP + 2)), (swa_bwd, dict(S=WRAP + 4)), (swa_bwd, dict(D=WRAP + 64)),
    (decode, dict(B=WRAP + 2)), (decode, dict(Hq=WRAP + 2)), (decode, dict(cap=WRAP + 64)), (decode, dict(D=WRAP + 64)),
])
def test_refused(host, call, sizes):
    with pytest.raises(cattn.CattnError) as e:
        call(**sizes)
    assert "NULL" not in str(e.value)  # (refused for its size, not for the addresses it does not have)


def test_the_calls_are_otherwise_taken(host):
    """What is refused above is refused for that size: the same calls get as far as the addresses."""
    for call in (norm, norm_q8, norm_bwd, rope, append, swa, swa_bwd, decode):
        with pytest.raises(cattn.CattnError, match="NULL"):
            call()


def test_frequencies_of_a_size_beyond_an_int(monkeypatch):
    """Refused before anything of that size is allocated."""
    monkeypatch.setattr(block.ctypes, "c_double", None)
    for rot in (1 << 31, WRAP + 64):
        with pytest.raises(cattn.CattnError, match="2\\^31"):
            cattn.rope_frequencies(rot)


def test_workspaces_of_refused_sizes():
    """None, and no overflow on the way."""
    big = (1 << 31) - 1
    for n in (big, WRAP + 1, WRAP + 64):
        assert cattn.rmsnorm_bwd_workspace_bytes(n, 64) == 0 and cattn.rmsnorm_bwd_workspace_bytes(2, n) == 0
        assert cattn.swa_bwd_workspace_bytes(1, 2, 2, n, 64, 8, 2) == cattn.swa_bwd_workspace_bytes(n, 2, 2, 40, 64, 8, 2) == 0
        assert cattn.swa_bwd_workspace_bytes(1, n, n, 40, 64, 8, 2) == 0
        assert cattn.swa_decode_workspace_bytes(1, 2, 2, n, 64, 8000, 2) == cattn.swa_decode_workspace_bytes(n, 2, 2, 4096, 64, 8000) == 0
        assert cattn.swa_bwd_workspace_bytes(1, 2, 2, 1 << 20, 64, n, n) > 0  # (window and sinks are clamped to S)
    assert cattn.rmsnorm_bwd_workspace_bytes(1 << 30, 64) == 512 * 64 * 4
    assert cattn.rmsnorm_bwd_workspace_bytes(2, 60) == cattn.swa_bwd_workspace_bytes(1, 2, 2, 4096, 96, 8, 2) == 0
    assert cattn.swa_decode_workspace_bytes(1, 2, 2, 4096, 96, 4000) == 0
