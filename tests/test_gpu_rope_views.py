"""Rotary positions and the append to a cache on views that fit no access wider than an element: an odd first
element, or odd strides of the caches.  The same bits as contiguous tensors give, and nothing beside the views
written."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from block_util import gen, randn
from parity_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_a_projection_from_any_element_on(cuda, offset, dtype, interleaved):
    say(f"rope view offset{offset} {dtype} {interleaved}")
    B, S, Hq, Hkv, D = 2, 9, 4, 2, 64
    flat = randn(gen(2), B * S * (Hq + 2 * Hkv) * D + offset, dtype=dtype).to(cuda)
    qkv = flat[offset:].view(B, S, Hq + 2 * Hkv, D)
    before = flat.clone()
    f = cattn.rope_frequencies(32).to(cuda)
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    for fn, outs in ((cattn.rope_fwd, ("q_out", "k_out")), (cattn.rope_bwd, ("dq_out", "dk_out"))):
        want = fn(q.contiguous(), k.contiguous(), f, layout="bshd", interleaved=interleaved)
        fn(q, k, f, layout="bshd", interleaved=interleaved, **dict(zip(outs, (q, k))))
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    kept = before[offset:].view_as(qkv)
    assert torch.equal(qkv[:, :, Hq + Hkv:], kept[:, :, Hq + Hkv:]) and torch.equal(flat[:offset], before[:offset])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 3])  # columns between the caches' rows: odd row, head and batch strides
def test_append_to_caches_of_any_stride(cuda, pad, dtype, interleaved):
    say(f"rope_append cache pad{pad} {dtype} {interleaved}")
    B, Hq, Hkv, S, D, cap = 2, 4, 2, 5, 64, 9
    g = gen(3)
    q, k, v = (randn(g, B, h, S, D, dtype=dtype).to(cuda) for h in (Hq, Hkv, Hkv))
    f = cattn.rope_frequencies(48).to(cuda)
    lens = torch.tensor([5, 8], dtype=torch.int32, device=cuda)
    memory = [randn(g, B, Hkv, cap, D + pad, dtype=dtype).to(cuda) for _ in range(2)]
    before = [m.clone() for m in memory]
    caches = [m[..., pad:] for m in memory]
    plain = [c.contiguous() for c in caches]
    # results too in rows of odd strides
    outs = [torch.zeros(B, h, S, D + pad, dtype=q.dtype, device=cuda)[..., pad:] for h in (Hq, Hkv)]
    want = cattn.rope_append(q, k, v, *plain, lens, f, interleaved=interleaved)
    got = cattn.rope_append(q, k, v, *caches, lens, f, interleaved=interleaved, q_out=outs[0], k_out=outs[1])
    assert all(torch.equal(a, b) for a, b in zip((*got, *caches), (*want, *plain)))
    assert all(torch.equal(m[..., :pad], b[..., :pad]) for m, b in zip(memory, before))
    assert not torch.equal(caches[0], before[0][..., pad:])
