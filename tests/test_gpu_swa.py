"""Sliding-window attention with sinks, forward and backward, on the GPU against
the float64 oracle (bounds: block_util)."""

import math

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import gen, randn, swa_bounds, within
from parity_util import max_abs, say, to64

pytestmark = pytest.mark.gpu


def order(t, layout):
    return t if layout == "bhsd" else t.transpose(1, 2)


def inputs(seed, B, Hq, Hkv, S, D, dtype, lens=None, sigma=1.0):
    g = gen(seed)
    q, k = randn(g, B, Hq, S, D, dtype=dtype, scale=sigma), randn(g, B, Hkv, S, D, dtype=dtype, scale=sigma)
    v, do = randn(g, B, Hkv, S, D, dtype=dtype), randn(g, B, Hq, S, D, dtype=dtype)
    if lens is not None:  # padding holds anything
        for b, n in enumerate(lens):
            for t in (q, k, v, do):
                t[b, :, max(n, 0):] = float("nan")
    return q, k, v, do


def check(cuda, B, Hq, Hkv, S, D, window, sinks, dtype, lens=None, layout="bhsd", sigma=1.0, scale=None):
    say(f"swa B{B} Hq{Hq} Hkv{Hkv} S{S} D{D} window{window} sinks{sinks} {dtype} {lens} {layout}")
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    q, k, v, do = inputs(S * 7 + window, B, Hq, Hkv, S, D, dtype, lens, sigma)
    qd, kd, vd, dod = (order(t, layout).contiguous().to(cuda) for t in (q, k, v, do))
    ld = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=cuda)
    o = torch.full_like(qd, float("nan"))
    lse = torch.full((B, Hq, S), float("nan"), device=cuda)
    cattn.swa_fwd(qd, kd, vd, scale, window, sinks, ld, layout, o=o, lse=lse)
    g = {"dq": torch.full_like(qd, float("nan")), "dk": torch.full_like(kd, float("nan")), "dv": torch.full_like(vd, float("nan"))}
    n = cattn.swa_bwd_workspace_bytes(B, Hq, Hkv, S, D, window, sinks) // 4
    ws = torch.full((n + 64,), float("nan"), device=cuda)
    cattn.swa_bwd(qd, kd, vd, o, dod, lse, scale, window, sinks, ld, layout, workspace=ws, **g)
    assert ws[n:].isnan().all()  # the workspace's size is enough
    ref = orc.swa(to64(q), to64(k), to64(v), scale, window, sinks, lens, to64(do))
    finite = ~np.isinf(ref["lse"])
    err = max_abs(np.where(finite, to64(lse), 0.0), np.where(finite, ref["lse"], 0.0))
    bounds = swa_bounds(ref, q, k, v, do, scale, dtype, err, min(S, window + sinks) * (Hq // Hkv) + S // 32 * (sinks > 0))
    within("lse", lse, ref["lse"], bounds["lse"])
    for name, got in (("o", o), *g.items()):
        within(name, order(got, layout), ref[name], bounds[name])
    return o, lse, g


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,window,sinks", [(70, 1, 0), (1, 5, 3)])
def test_one_visible_key_has_no_gradient(cuda, S, window, sinks, dtype):
    """Its probability is 1 whatever its score: dq and dk are 0 exactly, dv the sum of the group's do."""
    o, lse, g = check(cuda, 2, 4, 2, S, 64, window, sinks, dtype)
    assert not g["dq"].any() and not g["dk"].any() and g["dv"].any()


# window and sinks where tiles of 32 begin and end; S of one token, one tile, several
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,window,sinks", [
    (1, 1, 0), (2, 1, 1), (31, 5, 2), (32, 32, 0), (33, 32, 1), (64, 1, 0), (65, 31, 32), (97, 33, 4), (128, 64, 0),
    (129, 2, 3), (160, 160, 5), (200, 1000, 0), (257, 40, 33), (300, 3, 200), (333, 100, 64), (420, 128, 1)])
def test_lengths_windows_sinks(cuda, S, window, sinks, D, dtype):
    check(cuda, 1, 2, 1, S, D, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 3, 3), (64, 8, 2), (128, 4, 4), (128, 7, 1), (64, 16, 8)])
def test_head_groups_and_storage_order(cuda, D, Hq, Hkv, dtype):
    check(cuda, 2, Hq, Hkv, 150, D, 45, 3, dtype, layout="bshd")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(17, 0), (17, 5), (64, 40), (500, 0)])
def test_padded_batches(cuda, D, window, sinks, dtype):
    """NaN in the padding; sequences that end on and inside tiles, of one token, none, and lens out of range."""
    check(cuda, 7, 2, 1, 161, D, window, sinks, dtype, lens=[161, 160, 97, 64, 1, 0, 33])
    q, k, v, do = (t.to(cuda) for t in inputs(1, 2, 2, 1, 40, D, dtype, [40, -1]))
    ld = torch.tensor([99, -5], dtype=torch.int32, device=cuda)
    o, lse = cattn.swa_fwd(q, k, v, 0.1, window, sinks, ld)
    dq, dk, dv = cattn.swa_bwd(q, k, v, o, do, lse, 0.1, window, sinks, ld)
    want = cattn.swa_fwd(q[:1].contiguous(), k[:1].contiguous(), v[:1].contiguous(), 0.1, window, sinks)
    assert torch.equal(o[:1], want[0]) and torch.equal(lse[:1], want[1])
    assert not o[1].any() and torch.isneginf(lse[1]).all() and not dq[1].any() and not dk[1].any() and not dv[1].any()


@pytest.mark.parametrize("D,B,Hq,Hkv,S,window,sinks", [
    (64, 4, 48, 12, 513, 130, 2), (128, 2, 64, 16, 520, 200, 40), (64, 2, 32, 8, 1000, 64, 0), (128, 3, 40, 8, 400, 1, 1),
    (64, 1, 72, 72, 500, 300, 1), (128, 1, 65, 13, 700, 90, 3)])
def test_grids_of_every_split(cuda, D, B, Hq, Hkv, S, window, sinks):
    """Grids large enough for the unsplit work groups, and the two-part ones, ragged."""
    check(cuda, B, Hq, Hkv, S, D, window, sinks, "bf16", lens=[S - 7 * b for b in range(B)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,S,window,sinks", [
    (2, 2, 520, 8, 1), (2, 2, 521, 8, 1),      # 512 far queries and one more: without and with a grid of their own
    (2, 1, 300, 100, 2), (2, 1, 302, 101, 2),  # the same at 400, where float32 changes
    (4, 1, 700, 33, 40), (3, 3, 900, 128, 70), (8, 1, 350, 1, 32)])
def test_far_queries_of_the_sinks(cuda, Hq, Hkv, S, window, sinks, D, dtype):
    check(cuda, 1, Hq, Hkv, S, D, window, sinks, dtype)
    check(cuda, 3, Hq, Hkv, S, D, window, sinks, dtype, lens=[S, window, S // 2 + 3])  # far queries in some sequences only


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,B", [(64, 8), (128, 8), (128, 16), (64, 20)])
def test_far_queries_beside_or_within_the_windows_grid(cuda, D, B, dtype):
    """320 work groups, 256 of them the window's (one round of the GPU's CUs at D = 128), and whole rounds of them."""
    check(cuda, B, 4, 2, 500, D, 100, 3, dtype, [500 - 31 * (i % 3) for i in range(B)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ends_of_the_softmax(cuda, dtype):
    """Uniform rows, and rows near one-hot whose offset moves."""
    check(cuda, 1, 2, 2, 140, 64, 50, 2, dtype, scale=1e-20)
    check(cuda, 1, 2, 2, 140, 64, 50, 2, dtype, scale=0.4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_a_full_window_is_causal_attention(cuda, D, dtype):
    q, k, v, do = (t.to(cuda) for t in inputs(4, 2, 3, 3, 230, D, dtype))
    scale = 1 / math.sqrt(D)
    o, lse = cattn.swa_fwd(q, k, v, scale, 230)
    o2, lse2 = cattn.attn_fwd(q, k, v, scale)
    g = cattn.swa_bwd(q, k, v, o, do, lse, scale, 230)
    g2 = cattn.attn_bwd(q, k, v, o, do, lse, scale)
    tol = 1e-2 if dtype == "bf16" else 2e-6  # both within half of the type's tolerance of the truth
    assert torch.allclose(lse, lse2, atol=1e-5, rtol=0)
    for a, b in ((o, o2), *zip(g, g2)):
        assert (a.float() - b.float()).norm() <= tol * b.float().norm()
    # sinks that the window covers, and any window beyond the sequence, change nothing
    for window, sinks in ((230, 40), (10 ** 12, 0), (231, 10 ** 12)):
        assert torch.equal(cattn.swa_fwd(q, k, v, scale, window, sinks)[0], o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_views(cuda, dtype):
    """q, k, v as columns of one projection's output, results into views of others: the same bits as contiguous."""
    B, S, Hq, Hkv, D, window, sinks = 2, 150, 4, 2, 64, 40, 2
    qkv = randn(gen(8), B, S, Hq + 2 * Hkv, D, dtype=dtype).to(cuda)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    do = randn(gen(9), B, S, Hq, D, dtype=dtype).to(cuda)
    lens = torch.tensor([150, 71], dtype=torch.int32, device=cuda)
    o, lse = cattn.swa_fwd(q, k, v, 0.125, window, sinks, lens, "bshd")
    dqkv = torch.full_like(qkv, float("nan"))
    views = dqkv[:, :, :Hq], dqkv[:, :, Hq:Hq + Hkv], dqkv[:, :, Hq + Hkv:]
    cattn.swa_bwd(q, k, v, o, do, lse, 0.125, window, sinks, lens, "bshd", *views)
    qc, kc, vc = (t.contiguous() for t in (q, k, v))
    o2, lse2 = cattn.swa_fwd(qc, kc, vc, 0.125, window, sinks, lens, "bshd")
    want = cattn.swa_bwd(qc, kc, vc, o2, do, lse2, 0.125, window, sinks, lens, "bshd")
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(a, b) for a, b in zip(views, want)) and dqkv.isfinite().all()
    # heads-major views of the same memory, and a key/value head broadcast over the batch
    o3, _ = cattn.swa_fwd(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2), 0.125, window, sinks, lens)
    assert torch.equal(o3.transpose(1, 2), o2)
    kb, vb = (t[:1].expand(B, S, Hkv, D) for t in (kc, vc))
    o4, _ = cattn.swa_fwd(qc, kb, vb, 0.125, window, sinks, None, "bshd")
    assert torch.equal(o4, cattn.swa_fwd(qc, kb.contiguous(), vb.contiguous(), 0.125, window, sinks, None, "bshd")[0])
    with pytest.raises(cattn.CattnError):
        cattn.swa_bwd(qc, kb, vb, o2, do, lse2, 0.125, window, sinks, lens, "bshd", dk=kb)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_expanded_inputs_and_empty_sizes(cuda, dtype):
    """One key/value sequence for the whole batch, one gradient for all heads: views of stride 0."""
    q, k, v, do = (t.to(cuda) for t in inputs(8, 3, 4, 2, 90, 64, dtype))
    k, v, do = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1), do[:, :1].expand(-1, 4, -1, -1)
    o, lse = cattn.swa_fwd(q, k, v, 0.125, 20, 2)
    got = cattn.swa_bwd(q, k, v, o, do, lse, 0.125, 20, 2)
    k, v, do = (t.contiguous() for t in (k, v, do))
    want_o, want_lse = cattn.swa_fwd(q, k, v, 0.125, 20, 2)
    assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
    assert all(torch.equal(a, b) for a, b in zip(got, cattn.swa_bwd(q, k, v, o, do, lse, 0.125, 20, 2)))
    for shape in ((0, 4, 5, 64), (2, 4, 0, 64)):
        e = q.new_empty(shape)
        o, lse = cattn.swa_fwd(e, e, e, 0.125, 4, 1)
        g = cattn.swa_bwd(e, e, e, o, e, lse, 0.125, 4, 1)
        assert o.shape == shape and lse.shape == shape[:3] and all(t.shape == shape for t in g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(cuda, dtype):
    """Rows 2^22 elements apart, q, k, v, o and do side by side in them: the same bits as contiguous tensors give."""
    S, step = 600, 1 << 22
    t = inputs(9, 1, 2, 1, S, 64, dtype)
    q, k, v, do = (x.to(cuda) for x in t)
    memory = torch.empty(S * step, dtype=q.dtype, device=cuda)
    at, views = 0, []
    for x in (q, k, v, do, q):
        heads = x.shape[1]
        views.append(memory.as_strided((1, heads, S, 64), (heads * 64, 64, step, 1), at))
        views[-1].copy_(x)
        at += heads * 64
    say(f"swa strides past 32 bits {dtype}")
    o, lse = cattn.swa_fwd(q, k, v, 0.125, 90, 3)
    got, got_lse = cattn.swa_fwd(*views[:3], 0.125, 90, 3, o=views[4])
    assert torch.equal(got, o) and torch.equal(got_lse, lse)
    want = cattn.swa_bwd(q, k, v, o, do, lse, 0.125, 90, 3)
    dq = views[4]
    o2 = o.clone()
    got = cattn.swa_bwd(*views[:3], o2, views[3], lse, 0.125, 90, 3, dq=dq)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_repeats_and_streams(cuda):
    """The same bits every time, on another stream, and on two streams at once with workspaces of their own."""
    q, k, v, do = (t.to(cuda) for t in inputs(5, 2, 8, 2, 700, 64, "bf16"))

    def run():
        o, lse = cattn.swa_fwd(q, k, v, 0.125, 100, 5)
        return (o, lse) + cattn.swa_bwd(q, k, v, o, do, lse, 0.125, 100, 5)

    first = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = []
    for s in streams * 2:
        with torch.cuda.stream(s):
            results.append(run())
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(first, r))


def test_captured_and_replayed(cuda):
    """Forward and backward in a graph: every replay equals the eager results on the inputs it finds."""
    q, k, v, do = (t.to(cuda) for t in inputs(6, 1, 4, 2, 300, 64, "bf16"))
    lens = torch.tensor([300], dtype=torch.int32, device=cuda)

    def run():
        o, lse = cattn.swa_fwd(q, k, v, 0.125, 64, 4, lens)
        return (o, lse) + cattn.swa_bwd(q, k, v, o, do, lse, 0.125, 64, 4, lens)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for i, n in enumerate((300, 211, 40)):
        q.copy_(randn(gen(20 + i), 1, 4, 300, 64, dtype="bf16"))
        lens.fill_(n)
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), i


def test_refusals(cuda):
    q, k = torch.zeros(2, 4, 40, 64, device=cuda), torch.zeros(2, 2, 40, 64, device=cuda)
    for kw in (dict(window=0), dict(window=-3), dict(window=4, sinks=-1), dict(window=4, scale=0.0)):
        with pytest.raises(cattn.CattnError):
            cattn.swa_fwd(q, k, k, kw.pop("scale", 0.125), **kw)
    with pytest.raises(cattn.CattnError):
        cattn.swa_fwd(q[:, :3].contiguous(), k, k, 0.125, 4)
    with pytest.raises(cattn.CattnError):
        cattn.swa_fwd(q[..., :32].contiguous(), k[..., :32].contiguous(), k[..., :32].contiguous(), 0.125, 4)
    with pytest.raises(cattn.CattnError):
        cattn.swa_fwd(q, k, k, 0.125, 4, o=q)
    with pytest.raises(TypeError):
        cattn.swa_fwd(q, k.bfloat16(), k, 0.125, 4)
    with pytest.raises(TypeError):
        cattn.swa_fwd(q, k, k, 0.125, 4, lens=torch.zeros(2, dtype=torch.int64, device=cuda))
    with pytest.raises(ValueError):
        cattn.swa_fwd(q, k, k, 0.125, 4, lens=torch.zeros(3, dtype=torch.int32, device=cuda))
    with pytest.raises(ValueError):
        cattn.swa_bwd(q, k, k, q, q, torch.zeros(2, 4, 40, device=cuda), 0.125, 4, 2, workspace=torch.zeros(8, device=cuda))
    e = torch.zeros(0, 4, 40, 64, device=cuda)
    o, lse = cattn.swa_fwd(e, e, e, 0.125, 4)
    assert o.shape == e.shape and lse.shape == (0, 4, 40)
