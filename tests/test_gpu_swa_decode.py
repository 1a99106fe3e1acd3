"""Single-token attention over caches on the GPU against the float64 oracle, and
a decoder step of all operators together (bounds: block_util)."""

import math

import numpy as np
import pytest
import torch

import oracle.block_oracle as orc
import paper_2608_00029_amd as cattn
from block_util import E, TYPES, U, gen, randn, swa_bounds, within
from parity_util import say, to64

pytestmark = pytest.mark.gpu


def order(t, layout):
    return t if layout == "bhsd" else t.transpose(1, 2)


def check(cuda, lens, Hq, Hkv, cap, D, window, sinks, rolling, dtype, layout="bhsd"):
    """Caches laid out from whole sequences; slots that hold nothing visible are NaN."""
    say(f"decode lens={lens} Hq{Hq} Hkv{Hkv} cap{cap} D{D} window{window} sinks{sinks} rolling={rolling} {dtype} {layout}")
    B, scale, g = len(lens), 1 / math.sqrt(D), gen(cap + D)
    q = randn(g, B, Hq, D, dtype=dtype)
    kc, vc = (torch.full((B, Hkv, cap, D), float("nan"), dtype=TYPES[dtype]) for _ in range(2))
    want, sequences = [], []
    for b, n in enumerate(lens):
        k, v = randn(g, Hkv, n, D, dtype=dtype), randn(g, Hkv, n, D, dtype=dtype)
        sequences.append((k, v))
        slots = orc.cache_slots(n, cap, window, sinks, rolling)
        for p in np.flatnonzero(orc.visible(n, window, sinks)[n - 1]) if n else []:
            kc[b, :, slots[p]], vc[b, :, slots[p]] = k[:, p], v[:, p]
        want.append(orc.swa_decode(to64(q[b]), to64(k), to64(v), scale, window, sinks) if n else
                    (np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D))))
    kd, vd = (order(t, layout).contiguous().to(cuda) for t in (kc, vc))
    n = cattn.swa_decode_workspace_bytes(B, Hq, Hkv, cap, D, window, sinks, TYPES[dtype]) // 4
    ws = torch.full((n + 64,), float("nan"), device=cuda)
    o = torch.full((B, Hq, D), float("nan"), dtype=TYPES[dtype], device=cuda)
    lse = torch.full((B, Hq), float("nan"), device=cuda)
    ld = torch.tensor(lens, dtype=torch.int32, device=cuda)
    cattn.swa_decode(q.to(cuda), kd, vd, ld, scale, window, sinks, rolling, layout, o, lse, ws)
    assert ws[n:].isnan().all()
    ref = {"o": np.stack([w[0] for w in want]), "lse": np.stack([w[1] for w in want]), "m_o": np.stack([w[2] for w in want])}
    if max(lens):
        keys, values = (torch.cat([s[i].flatten(0, 1) for s in sequences]) for i in (0, 1))
        bounds = swa_bounds(ref, q, keys, values, None, scale, dtype, 0.0, window + sinks)
        within("o", o, ref["o"], bounds["o"])
        within("lse", lse, ref["lse"], bounds["lse"])
    else:
        assert not o.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,window,sinks,lens", [
    (1, 1, 0, [1, 0]), (40, 33, 2, [1, 2, 3, 31, 32, 33, 34, 35, 36, 40, 0]), (300, 64, 5, [300, 69, 70, 68, 5, 6, 200]),
    (200, 500, 0, [200, 199, 129, 128, 127]), (700, 300, 40, [700, 340, 341, 300, 12]), (150, 1, 1, [150, 1, 2]),
    (90, 10, 60, [90, 75, 60, 61, 10, 9])])
@pytest.mark.parametrize("rolling", [False, True])
def test_caches(cuda, rolling, cap, window, sinks, lens, D, dtype):
    if rolling:  # a cache of just what is visible, and sequences longer than it
        cap = window + sinks
        lens = lens + [2 * cap + 3]
    check(cuda, lens, 4, 2, cap, D, window, sinks, rolling, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (3, 1, 128), (40, 1, 64), (64, 2, 128), (33, 1, 128), (16, 16, 64)])
def test_head_groups(cuda, Hq, Hkv, D, dtype):
    check(cuda, [77, 5], Hq, Hkv, 100, D, 50, 4, False, dtype, "bshd")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts(cuda, dtype):
    """One long sequence over many work groups, some without a slot; many sequences, one each."""
    check(cuda, [3000], 8, 2, 3000, 64, 2500, 3, False, dtype)
    check(cuda, [3000, 200], 8, 1, 4000, 128, 5000, 0, False, dtype)
    check(cuda, [70 + i for i in range(64)], 8, 4, 160, 64, 60, 2, False, dtype)
    check(cuda, [930 + i for i in range(100)], 6, 3, 1030, 64, 1024, 0, False, dtype)  # over a work group per CU
    check(cuda, [700, 650, 1], 8, 8, 700, 128, 600, 1, True, dtype)


def test_strides_and_lens_past_a_linear_cache(cuda):
    g = gen(2)
    kc, vc = randn(g, 2, 2, 50, 64).to(cuda), randn(g, 2, 2, 50, 64).to(cuda)
    qkv = randn(g, 2, 8, 64).to(cuda)
    q = qkv[:, :4]
    lens = torch.tensor([50, 33], dtype=torch.int32, device=cuda)
    o, lse = cattn.swa_decode(q, kc, vc, lens, 0.125, 20, 1)
    o2, lse2 = cattn.swa_decode(q.contiguous(), kc, vc, torch.tensor([77, 33], dtype=torch.int32, device=cuda), 0.125, 20, 1)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # caches as views of larger ones: a part of the slots, heads of another order
    big = torch.full((2, 64, 3, 64), float("nan"), device=cuda)
    kv, vv = big[:, 5:55, :2], big.clone()[:, 5:55, 1:]
    kv.copy_(kc.transpose(1, 2))
    vv.copy_(vc.transpose(1, 2))
    out = torch.full((2, 6, 64), float("nan"), device=cuda)
    cattn.swa_decode(q, kv, vv, lens, 0.125, 20, 1, layout="bshd", o=out[:, 1:5])
    assert torch.equal(out[:, 1:5], o) and out[:, 0].isnan().all() and out[:, 5].isnan().all()


def test_offsets_past_32_bits(cuda):
    """A cache of more than 2^31 elements per sequence's head stride: slots at its far end."""
    cap, D = (1 << 24) + 40, 128
    kc = torch.zeros(1, 1, cap, D, dtype=torch.bfloat16, device=cuda)
    vc = torch.zeros(1, 1, cap, D, dtype=torch.bfloat16, device=cuda)
    assert kc.numel() > 2 ** 31
    g = gen(4)
    n = cap - 3
    k, v, q = randn(g, 1, 50, D, dtype="bf16"), randn(g, 1, 50, D, dtype="bf16"), randn(g, 1, 2, D, dtype="bf16")
    kc[0, 0, n - 50:n], vc[0, 0, n - 50:n] = k[0].to(cuda), v[0].to(cuda)
    lens = torch.tensor([n], dtype=torch.int32, device=cuda)
    o, lse = cattn.swa_decode(q.to(cuda), kc, vc, lens, 0.1, 50)
    ro, rl, m = orc.swa_decode(to64(q[0]), to64(k), to64(v), 0.1, 50)
    b = swa_bounds({"o": ro, "lse": rl, "m_o": m}, q, k, v, None, 0.1, "bf16", 0.0, 50)
    within("o", o[0], ro, b["o"])
    within("lse", lse[0], rl, b["lse"])
    # and a token appended there
    f = cattn.rope_frequencies(D).to(cuda)
    t = randn(g, 1, 1, 1, D, dtype="bf16").to(cuda)
    lens += 1
    _, kr = cattn.rope_append(t, t, t, kc, vc, lens, f)
    assert torch.equal(kc[0, 0, n], kr[0, 0, 0]) and torch.equal(vc[0, 0, n], t[0, 0, 0]) and not kc[0, 0, n + 1:].any()


def test_empty_batch_and_an_expanded_cache(cuda):
    """No sequences; and one cache read by every sequence of a batch (stride 0)."""
    q, kc, vc = (randn(gen(50 + i), 3, h, 64, dtype="bf16").to(cuda) for i, h in enumerate((4, 2, 2)))
    kc, vc = (t[:1, :, None].expand(3, 2, 40, 64) + torch.arange(40, device=cuda)[:, None] % 3 for t in (kc, vc))
    lens = torch.tensor([40, 7, 0], dtype=torch.int32, device=cuda)
    want = cattn.swa_decode(q, kc, vc, lens, 0.125, 20, 2)
    got = cattn.swa_decode(q, kc[:1].expand(3, -1, -1, -1), vc[:1].expand(3, -1, -1, -1), lens, 0.125, 20, 2)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    o, lse = cattn.swa_decode(q[:0], kc[:0].contiguous(), vc[:0].contiguous(), lens[:0], 0.125, 20, 2)
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_refusals(cuda):
    q, c = torch.zeros(2, 4, 64, device=cuda), torch.zeros(2, 2, 40, 64, device=cuda)
    lens = torch.ones(2, dtype=torch.int32, device=cuda)
    with pytest.raises(cattn.CattnError):
        cattn.swa_decode(q, c, c, lens, 0.125, 40, 1, rolling=True)
    with pytest.raises(cattn.CattnError):
        cattn.swa_decode(q, c, c, lens, 0.125, 0)
    with pytest.raises(ValueError):
        cattn.swa_decode(q[:, :, None], c, c, lens, 0.125, 4)
    with pytest.raises(ValueError):
        cattn.swa_decode(q, c, c[:, :, :30], lens, 0.125, 4)
    with pytest.raises(TypeError):
        cattn.swa_decode(q, c, c, lens.long(), 0.125, 4)
    big = torch.zeros(1, 1, 4000, 64, device=cuda)
    with pytest.raises(ValueError):
        cattn.swa_decode(q[:1, :1].contiguous(), big, big, lens[:1], 0.125, 4000, workspace=torch.zeros(8, device=cuda))


# ---------------------------------------------------------------------------
# All operators together
# ---------------------------------------------------------------------------
class Block:
    """The attention half of a decoder block: norm with the residual, projection, rotary positions, windowed attention,
    projection.  `ops` computes the five operators; the products are torch's in both."""

    def __init__(self, seed, C=256, Hq=4, Hkv=2, D=64, window=24, sinks=2):
        g = gen(seed)
        self.C, self.Hq, self.Hkv, self.D, self.window, self.sinks = C, Hq, Hkv, D, window, sinks
        self.gamma = 1 + 0.1 * randn(g, C)
        self.w = randn(g, (Hq + 2 * Hkv) * D, C) / math.sqrt(C)
        self.wo = randn(g, C, Hq * D) / math.sqrt(Hq * D)
        self.freqs = cattn.rope_frequencies(48)
        self.scale = 1 / math.sqrt(D)

    def to(self, device):
        self.gamma, self.w, self.wo, self.freqs = (t.to(device) for t in (self.gamma, self.w, self.wo, self.freqs))
        return self

    def heads(self, n):
        """The projection's rows [B, S, (Hq + 2 Hkv) D] of a normalised n [B, S, C] as q, k, v views."""
        p = (n @ self.w.t()).unflatten(-1, (self.Hq + 2 * self.Hkv, self.D))
        return p[:, :, :self.Hq], p[:, :, self.Hq:self.Hq + self.Hkv], p[:, :, self.Hq + self.Hkv:]


def reference_block(blk, x, r, lens):
    """The block in float64 with autograd over every input, from the definitions."""
    h = x + r
    n = h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * blk.gamma
    q, k, v = (t.transpose(1, 2) for t in blk.heads(n))
    S = x.shape[1]
    ang = torch.arange(S, dtype=torch.float64)[:, None] * blk.freqs

    def turn(t):
        a, b, rest = t[..., :24], t[..., 24:48], t[..., 48:]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin(), rest], -1)

    q, k = turn(q), turn(k)
    z = blk.scale * q @ k.repeat_interleave(blk.Hq // blk.Hkv, 1).transpose(2, 3)
    z = z.masked_fill(~torch.from_numpy(orc.visible(S, blk.window, blk.sinks)), -math.inf)
    o = torch.softmax(z, -1) @ v.repeat_interleave(blk.Hq // blk.Hkv, 1)
    y = o.transpose(1, 2).flatten(2) @ blk.wo.t()
    mask = torch.stack([(torch.arange(S) < m) for m in lens])[..., None]
    return h, torch.where(mask, y, torch.zeros_like(y))


def test_a_training_step_and_its_gradients(cuda):
    """Forward and backward through all operators, against autograd in float64 on the CPU."""
    B, S = 2, 70
    lens = [70, 41]
    g = gen(11)
    x, r, dy, dh = (randn(g, B, S, 256) for _ in range(4))
    ref = Block(1)
    ref.gamma, ref.w, ref.wo = (t.double().requires_grad_() for t in (ref.gamma, ref.w, ref.wo))
    xr, rr = x.double().requires_grad_(), r.double().requires_grad_()
    h_ref, y_ref = reference_block(ref, xr, rr, lens)
    ((y_ref * dy.double()).sum() + (h_ref * dh.double()).sum()).backward()

    blk = Block(1).to(cuda)
    xd, rd, dyd, dhd = (t.to(cuda) for t in (x, r, dy, dh))
    ld = torch.tensor(lens, dtype=torch.int32, device=cuda)
    n, h, rstd = cattn.rmsnorm_fwd(xd, blk.gamma, rd)
    q, k, v = blk.heads(n)
    cattn.rope_fwd(q, k, blk.freqs, layout="bshd", q_out=q, k_out=k)  # in place in the projection's output
    o, lse = cattn.swa_fwd(q, k, v, blk.scale, blk.window, blk.sinks, ld, "bshd")
    y = o.flatten(2) @ blk.wo.t()
    do = (dyd @ blk.wo).view_as(o)
    dp = torch.empty(B, S, blk.Hq + 2 * blk.Hkv, blk.D, device=cuda)
    dq, dk, dv = dp[:, :, :blk.Hq], dp[:, :, blk.Hq:blk.Hq + blk.Hkv], dp[:, :, blk.Hq + blk.Hkv:]
    cattn.swa_bwd(q, k, v, o, do, lse, blk.scale, blk.window, blk.sinks, ld, "bshd", dq, dk, dv)
    cattn.rope_bwd(dq, dk, blk.freqs, layout="bshd", dq_out=dq, dk_out=dk)
    dn = dp.flatten(2) @ blk.w
    dx, dgamma = cattn.rmsnorm_bwd(h, blk.gamma, rstd, dn, dhd)
    dw = dp.flatten(0, 1).flatten(1).t() @ n.flatten(0, 1)
    # float32 throughout: some thousand roundings of sums of at most 512 terms, 2^-24 each; 1e-5 of the norm is ample
    # for one that adds up and far below any wrong term
    for name, got, want in (("y", y, y_ref), ("h", h, h_ref), ("dx", dx, xr.grad), ("dgamma", dgamma, ref.gamma.grad),
                            ("dw", dw, ref.w.grad)):
        want = want.detach()
        err = (got.cpu().double() - want).norm() / want.norm()
        assert err <= 1e-5, (name, float(err))
    assert torch.equal(xr.grad, rr.grad)  # one gradient for both: dx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_and_single_tokens_equal_the_whole_sequence(cuda, dtype):
    """Prompts of uneven length through training's operators into a rolling cache, then token by token: each step's
    attention equals the whole sequence's at that row, within the two computations' bounds."""
    B, S, prompt = 3, 60, [37, 20, 1]
    blk = Block(2).to(cuda)
    g = gen(12)
    x = randn(g, B, S, 256, dtype=dtype).to(cuda)
    blk.w = blk.w.to(TYPES[dtype])
    n, _, _ = cattn.rmsnorm_fwd(x, blk.gamma)
    q, k, v = (t.contiguous() for t in blk.heads(n))
    qr, kr = cattn.rope_fwd(q, k, blk.freqs, layout="bshd")
    whole, whole_lse = cattn.swa_fwd(qr, kr, v, blk.scale, blk.window, blk.sinks, layout="bshd")

    cap = blk.window + blk.sinks
    kc, vc = (torch.full((B, cap, blk.Hkv, blk.D), float("nan"), dtype=TYPES[dtype], device=cuda) for _ in range(2))
    lens = torch.tensor(prompt, dtype=torch.int32, device=cuda)
    P = max(prompt)
    q0, k0 = cattn.rope_append(q[:, :P].contiguous(), k[:, :P].contiguous(), v[:, :P].contiguous(), kc, vc, lens, blk.freqs,
                               counts=lens, window=blk.window, sinks=blk.sinks, rolling=True, layout="bshd")
    o, _ = cattn.swa_fwd(q0, k0, v[:, :P].contiguous(), blk.scale, blk.window, blk.sinks, lens, "bshd")
    for b, m in enumerate(prompt):
        assert torch.equal(q0[b, :m], qr[b, :m]) and torch.equal(k0[b, :m], kr[b, :m])
    tol = 2 * (2 * U[dtype] + 400 * E)  # two computations, each within 2 U + (keys + D + 80) E + 2 eps_s (about 50 E) of the terms' sum
    m_o = float(v.float().abs().max())
    for b, m in enumerate(prompt):
        assert (o[b, :m].float() - whole[b, :m].float()).abs().max() <= tol * m_o
    for step in range(S - P):
        at = lens.long()  # the row of each sequence's next token
        lens += 1
        rows = [t[torch.arange(B, device=cuda), at][:, None].contiguous() for t in (q, k, v)]
        qn, _ = cattn.rope_append(*rows, kc, vc, lens, blk.freqs, window=blk.window, sinks=blk.sinks, rolling=True, layout="bshd")
        o, lse = cattn.swa_decode(qn[:, 0], kc, vc, lens, blk.scale, blk.window, blk.sinks, rolling=True, layout="bshd")
        want = whole[torch.arange(B, device=cuda), at]
        assert (o.float() - want.float()).abs().max() <= tol * m_o, step
        want = torch.stack([whole_lse[b, :, int(at[b])] for b in range(B)])
        assert (lse - want).abs().max() <= 2 * 600 * E * 8, step


def test_a_captured_decoding_step(cuda):
    """Append and attention in one graph, replayed over a growing sequence: every step equals the eager one."""
    B, Hq, Hkv, D, window, sinks = 2, 4, 2, 64, 30, 2
    g = gen(13)
    f = cattn.rope_frequencies(D).to(cuda)
    q, k, v = (randn(g, B, h, 1, D, dtype="bf16").to(cuda) for h in (Hq, Hkv, Hkv))
    caches = [torch.zeros(B, Hkv, 32, D, dtype=torch.bfloat16, device=cuda) for _ in range(4)]
    lens = torch.ones(B, dtype=torch.int32, device=cuda)

    def step(kc, vc):
        qr, _ = cattn.rope_append(q, k, v, kc, vc, lens, f, window=window, sinks=sinks, rolling=True)
        return cattn.swa_decode(qr[:, :, 0], kc, vc, lens, 0.125, window, sinks, rolling=True)

    step(*caches[2:])
    torch.cuda.synchronize()
    for c in caches:
        c.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step(*caches[:2])
    for c in caches:
        c.zero_()
    lens.zero_()
    for i in range(70):
        for t in (q, k, v):
            t.copy_(randn(g, *t.shape, dtype="bf16"))
        lens += 1
        graph.replay()
        want, want_lse = step(*caches[2:])
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lse, want_lse), i
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
