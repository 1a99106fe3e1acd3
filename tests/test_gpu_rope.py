"""Rotary positions and the append to a cache on the GPU against the float64
oracle (bounds: block_util)."""

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import E, TINY, U, gen, randn, within
from parity_util import say, to64

pytestmark = pytest.mark.gpu


def order(t, layout):
    return t if layout == "bhsd" else t.transpose(1, 2)


def check(name, got, x, ref, amplitude, freqs, interleaved, dtype):
    """got against the turned x: 10 E of |a| + |b| of the element's pair, and its rounding; copies exact."""
    x, half = np.abs(to64(x)), len(freqs)
    size = np.zeros_like(x)
    a_at, b_at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    size[..., a_at] = size[..., b_at] = x[..., a_at] + x[..., b_at]
    within(name, got, ref, 10 * E * abs(amplitude) * size + (U[dtype] * np.abs(ref) + TINY) * (size > 0))


CASES = [  # B, Hq, Hkv, S, D, rot, interleaved, layout
    (1, 1, 1, 1, 64, 64, False, "bhsd"), (2, 4, 2, 5, 128, 128, False, "bshd"), (2, 3, 1, 33, 64, 32, True, "bhsd"),
    (1, 8, 2, 17, 128, 24, False, "bhsd"), (3, 2, 2, 7, 64, 6, True, "bshd"), (1, 5, 5, 3, 70, 70, False, "bhsd"),
    (2, 40, 8, 9, 128, 64, True, "bshd"), (1, 2, 1, 4, 512, 512, False, "bhsd"), (1, 1, 1, 3, 512, 2, True, "bhsd"),
    (4, 12, 4, 700, 64, 64, False, "bhsd"), (2, 4, 4, 6000, 64, 48, False, "bshd"), (1, 300, 20, 2, 16, 8, False, "bhsd"),
    (2, 4, 2, 30, 128, 20, True, "bhsd"), (2, 4, 2, 300, 64, 24, False, "bshd"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,S,D,rot,interleaved,layout", CASES)
def test_forward_and_backward(cuda, B, Hq, Hkv, S, D, rot, interleaved, layout, dtype):
    say(f"rope B{B} Hq{Hq} Hkv{Hkv} S{S} D{D} rot{rot} {interleaved} {layout} {dtype}")
    g = gen(B + S + D + rot)
    q, k = randn(g, B, Hq, S, D, dtype=dtype), randn(g, B, Hkv, S, D, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (B, S), generator=g).to(torch.int32)
    f = cattn.rope_frequencies(rot, scaling="ramp", factor=4.0, context=4096.0)
    amplitude = 1.14
    fd, pd = f.to(cuda), pos.to(cuda)
    qd, kd = order(q, layout).contiguous().to(cuda), order(k, layout).contiguous().to(cuda)
    for fn, inverse in ((cattn.rope_fwd, False), (cattn.rope_bwd, True)):
        qo, ko = fn(qd, kd, fd, pd, layout=layout, interleaved=interleaved, amplitude=amplitude)
        for n, got, x in (("q", qo, q), ("k", ko, k)):
            ref = orc.rope(to64(x), pos.numpy(), f.numpy(), interleaved, amplitude, inverse)
            check(n, order(got, layout), x, ref, amplitude, f, interleaved, dtype)
    # in place: the same bits
    q2, k2 = qd.clone(), kd.clone()
    a = cattn.rope_bwd(q2, k2, fd, pd, layout=layout, interleaved=interleaved, amplitude=amplitude, dq_out=q2, dk_out=k2)
    assert a[0] is q2 and torch.equal(q2, qo) and torch.equal(k2, ko)


def test_positions_far_negative_default_and_shared(cuda):
    f = cattn.rope_frequencies(64)
    q = randn(gen(1), 2, 2, 3, 64)
    far = torch.tensor([[0, 2 ** 31 - 1, 123456789], [-5, -(2 ** 31), 16777217]], dtype=torch.int32)
    got, none = cattn.rope_fwd(q.to(cuda), None, f.to(cuda), far.to(cuda))
    assert none is None
    # the oracle's own angle is off by 2^31 2^-53 radians: nothing against 10 E
    check("q", got, q, orc.rope(to64(q), far.numpy(), f.numpy()), 1.0, f, False, "f32")
    want, _ = cattn.rope_fwd(q.to(cuda), None, f.to(cuda), torch.arange(3, dtype=torch.int32, device=cuda))
    assert torch.equal(want, cattn.rope_fwd(q.to(cuda), None, f.to(cuda))[0])
    assert torch.equal(want[:, :, 0], q.to(cuda)[:, :, 0])


@pytest.mark.parametrize("offset", [0, 1])
def test_views_of_a_projection_in_place(cuda, offset):
    """q and k are columns of one [B, S, Hq + 2 Hkv, D] tensor, rotated in place; the rest stays.  With an odd
    first element nothing is 16-byte aligned."""
    B, S, Hq, Hkv, D = 2, 9, 4, 2, 64
    flat = randn(gen(2), B * S * (Hq + 2 * Hkv) * D + offset, dtype="bf16").to(cuda)
    qkv = flat[offset:].view(B, S, Hq + 2 * Hkv, D)
    before = qkv.clone()
    f = cattn.rope_frequencies(32).to(cuda)
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    want = cattn.rope_fwd(q.contiguous(), k.contiguous(), f, layout="bshd")
    cattn.rope_fwd(q, k, f, layout="bshd", q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, Hq + Hkv:], before[:, :, Hq + Hkv:])
    with pytest.raises(cattn.CattnError):  # q's results onto k
        cattn.rope_fwd(q[:, :, :Hkv], k, f, layout="bshd", q_out=k, k_out=k)


@pytest.mark.parametrize("layout", ["bhsd", "bshd"])
@pytest.mark.parametrize("dtype,D,rot,interleaved", [("bf16", 128, 128, False), ("bf16", 64, 32, True), ("f32", 64, 64, False),
                                                     ("bf16", 66, 22, False)])
@pytest.mark.parametrize("rolling", [False, True])
def test_append(cuda, rolling, dtype, D, rot, interleaved, layout):
    """Prompts of uneven length (more tokens than the window, fewer, none), then single tokens; the cache's slots
    against the oracle's, all others as they were."""
    say(f"rope_append rolling={rolling} {dtype} D{D} rot{rot} {interleaved} {layout}")
    B, Hq, Hkv, S, cap, window, sinks = 5, 4, 2, 13, 16, 6, 3
    g = gen(D + rot)
    f = cattn.rope_frequencies(rot)
    kc, vc = randn(g, B, Hkv, cap, D, dtype=dtype), randn(g, B, Hkv, cap, D, dtype=dtype)
    kcd, vcd = (order(t, layout).contiguous().to(cuda) for t in (kc, vc))
    held = [{} for _ in range(B)]  # position: (key, value, bound of the key)
    lens = torch.zeros(B, dtype=torch.int32)
    for step, counts in enumerate(([13, 2, 0, 7, 9], [1, 1, 1, 1, 0], None, [1, 1, 1, 1, 1], [-3, 1, 0, 1, 99])):
        n = S if step == 0 else 1
        cnt = [n] * B if counts is None else [min(max(c, 0), n) for c in counts]
        lens += torch.tensor(cnt, dtype=torch.int32)
        q, k, v = randn(g, B, Hq, n, D, dtype=dtype), randn(g, B, Hkv, n, D, dtype=dtype), randn(g, B, Hkv, n, D, dtype=dtype)
        for b in range(B):  # rows past the count may hold anything
            q[b, :, cnt[b]:] = k[b, :, cnt[b]:] = v[b, :, cnt[b]:] = float("nan")
        qd, kd, vd = (order(t, layout).contiguous().to(cuda) for t in (q, k, v))
        qo, ko = cattn.rope_append(qd, kd, vd, kcd, vcd, lens.to(cuda), f.to(cuda),
                                   None if counts is None else torch.tensor(counts, dtype=torch.int32, device=cuda), window, sinks,
                                   rolling, layout, interleaved)
        pos = np.stack([np.arange(n) + int(lens[b]) - cnt[b] for b in range(B)])
        for name, got, x in (("q", qo, q), ("k", ko, k)):
            x = torch.nan_to_num(x, nan=0.0)
            ref = orc.rope(to64(x), pos, f.numpy(), interleaved)
            check(name, order(got, layout), x, ref, 1.0, f, interleaved, dtype)
        rows = order(ko, layout).cpu()
        for b in range(B):
            for i in range(cnt[b]):
                held[b][int(pos[b, i])] = (rows[b, :, i], v[b, :, i])
            slots = orc.cache_slots(int(lens[b]), cap, window, sinks, rolling)
            for p, s in slots.items():
                kc[b, :, s], vc[b, :, s] = held[b][p]
        assert torch.equal(order(kcd, layout).cpu(), kc) and torch.equal(order(vcd, layout).cpu(), vc), step


def test_empty_sizes_and_a_replayed_graph(cuda):
    f = cattn.rope_frequencies(64).to(cuda)
    for shape in ((0, 2, 3, 64), (2, 2, 0, 64)):
        e = torch.empty(shape, device=cuda)
        assert cattn.rope_fwd(e, e, f)[1].shape == shape
        cache = torch.empty(shape[0], 2, 8, 64, device=cuda)
        lens = torch.zeros(shape[0], dtype=torch.int32, device=cuda)
        assert cattn.rope_append(e, e, e, cache, cache.clone(), lens, f)[0].shape == shape
    q, k = (randn(gen(30), 2, h, 70, 64, dtype="bf16").to(cuda) for h in (4, 2))
    pos = torch.arange(70, dtype=torch.int32, device=cuda)

    def run():
        turned = cattn.rope_fwd(q, k, f, pos)
        return turned + cattn.rope_bwd(*turned, f, pos)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(3):
        pos += 1000
        q.copy_(torch.roll(q, 1, 2))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_more_tokens_than_one_grid_dimension_takes(cuda):
    """2^27 and some tokens of one pair: over 2^24 work groups of 8 tokens (a launch counts a dimension's threads
    in 32 bits).  The sine and cosine of an angle, float32 from the 64-bit turns, are off by under 1e-6."""
    S = (1 << 27) + 11
    q = torch.ones(1, 1, S, 2, dtype=torch.float32, device=cuda)
    f = cattn.rope_frequencies(2).to(cuda) * 1e-3
    say(f"rope S{S} D2")
    o, _ = cattn.rope_fwd(q, None, f, q_out=q)
    third = (S + 7) // 8 // 3 * 8  # about where a third of the work groups ends
    at = torch.cat([torch.arange(64), *(torch.arange(third * i - 64, third * i + 64) for i in (1, 2)), torch.arange(S - 64, S)])
    got, angle = o[0, 0, at.to(cuda)].cpu().double(), at.double() * float(f[0])
    ref = torch.stack([angle.cos() - angle.sin(), angle.cos() + angle.sin()], -1)
    assert (got - ref).abs().max() <= 2e-6
    n = o.double().square_().sum(-1)
    assert (n - 2).abs().max() <= 1e-5  # every row was turned once or not at all
    assert int((o[0, 0, 1:] == 1).all(-1).sum()) <= 9  # ... at all: 9 angles have |sin| < 2e-7, whose row may be (1, 1) again


def test_offsets_past_32_bits(cuda):
    S, step = 600, 1 << 22
    q = randn(gen(31), 1, 2, S, 64, dtype="bf16").to(cuda)
    memory = torch.empty(S * step, dtype=q.dtype, device=cuda)
    view = memory.as_strided((1, 2, S, 64), (128, 64, step, 1))
    view.copy_(q)
    f = cattn.rope_frequencies(32).to(cuda)
    say("rope strides past 32 bits")
    want, _ = cattn.rope_fwd(q, None, f)
    assert torch.equal(cattn.rope_fwd(view, None, f, q_out=view)[0], want)


def test_append_past_a_linear_cache_is_dropped(cuda):
    g = gen(9)
    q, k, v = (randn(g, 2, 1, 1, 64).to(cuda) for _ in range(3))
    kc, vc = (randn(g, 2, 1, 4, 64).to(cuda) for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    f = cattn.rope_frequencies(64).to(cuda)
    cattn.rope_append(q, k, v, kc, vc, torch.tensor([5, 2 ** 31 - 1], dtype=torch.int32, device=cuda), f)
    assert torch.equal(kc, k0) and torch.equal(vc, v0)
    qo, ko = cattn.rope_append(q, k, v, kc, vc, torch.tensor([0, -7], dtype=torch.int32, device=cuda), f)
    assert torch.equal(kc, k0) and not qo.any() and not ko.any()


def test_refusals(cuda):
    q = torch.zeros(2, 4, 3, 64, device=cuda)
    f = cattn.rope_frequencies(64).to(cuda)
    with pytest.raises(TypeError):
        cattn.rope_fwd(q, None, f.float())
    with pytest.raises(TypeError):
        cattn.rope_fwd(q, None, f, torch.zeros(2, 3, dtype=torch.int64, device=cuda))
    with pytest.raises(ValueError):
        cattn.rope_fwd(q, None, f, torch.zeros(3, 2, dtype=torch.int32, device=cuda))
    with pytest.raises(ValueError):
        cattn.rope_fwd(q, q[:, :, :2], f)
    with pytest.raises(TypeError):
        cattn.rope_fwd(q.half(), None, f)
    with pytest.raises(ValueError):
        cattn.rope_fwd(q.transpose(2, 3), None, f)
    with pytest.raises(ValueError):
        cattn.rope_fwd(q, None, f, layout="sbhd")
    with pytest.raises(cattn.CattnError):
        cattn.rope_fwd(q[..., :32], None, f)
    with pytest.raises(cattn.CattnError):
        cattn.rope_append(q, q, q, q.clone(), q.clone(), torch.zeros(2, dtype=torch.int32, device=cuda), f, window=3, sinks=1,
                          rolling=True)
