"""The codes of RMSNorm's 8-bit output, one by one: e4m3, to nearest even, of the float32 quotient y / scale."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from block_util import TYPES, gen, randn
from parity_util import say

pytestmark = pytest.mark.gpu


def rule(y, scale, group):
    """The codes of float32 y [rows, C]; a quotient on or beside the middle of two codes shows any other arithmetic."""
    wide = scale.repeat_interleave(group or y.shape[1], 1)[:, :y.shape[1]]
    return (y / wide).to(torch.float8_e4m3fn)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C,group", [(40, 1024, 0), (2000, 512, 64), (300, 2056, 0), (9, 16384, 128), (70, 4096, 512)])
def test_codes_of_whole_numbers(cuda, rows, C, group, dtype):
    """Rows of whole numbers whose largest is 448, 224 or 300: every quotient is near one, and many are in the middle of
    two codes.  (The float32 input of the same values takes the same steps to the same y.)"""
    say(f"rmsnorm codes rows={rows} C={C} group={group} {dtype}")
    top = torch.tensor([448.0, 224.0, 300.0])[torch.arange(rows) % 3, None]
    g = gen(rows + C)
    # (bfloat16 holds whole numbers to 256 and even ones to 512)
    x = (torch.randint(-224, 225, (rows, C), generator=g) * 2).float().clamp(-top, top)
    x[:, ::8] = top
    gamma = torch.ones(C)
    q, scale, _, _ = cattn.rmsnorm_fwd_q8(x.to(TYPES[dtype]).to(cuda), gamma.to(cuda), None, 1e-5, group)
    y, _, _ = cattn.rmsnorm_fwd(x.to(cuda), gamma.to(cuda))
    want = rule(y.cpu(), scale.cpu(), group)
    off = q.cpu().view(torch.uint8) != want.view(torch.uint8)
    at = off.nonzero()[:1]
    assert not off.any(), (int(off.sum()), at, y.cpu()[off][0], q.cpu().float()[off][0], want.float()[off][0])


@pytest.mark.parametrize("rows,C,group,scale", [(2100, 2048, 0, 1.0), (1030, 768, 128, 1e-37), (64, 4096, 0, 1e30), (64, 4096, 0, 1e-20),
                                                (300, 1600, 16, 1e-34), (50, 2056, 64, 3e19), (5, 512, 0, 1.4e38)])
def test_codes_of_random_rows(cuda, rows, C, group, scale):
    """Random rows, and gammas of both signs that bring y to the smallest and near the largest float32 values."""
    say(f"rmsnorm codes rows={rows} C={C} group={group} gamma {scale}")
    g = gen(rows)
    x, gamma = randn(g, rows, C), (1 + 0.2 * randn(g, C)) * scale * (1 - 2 * (torch.arange(C) % 2))
    x[:, :64] = 0  # zeros of both signs
    q, s, _, _ = cattn.rmsnorm_fwd_q8(x.to(cuda), gamma.to(cuda), None, 1e-5, group)
    y, _, _ = cattn.rmsnorm_fwd(x.to(cuda), gamma.to(cuda))
    want = rule(y.cpu(), s.cpu(), group)
    off = q.cpu().view(torch.uint8) != want.view(torch.uint8)
    assert not off.any(), (int(off.sum()), y.cpu()[off][0], q.cpu().float()[off][0], want.float()[off][0])


def test_an_infinite_scale(cuda):
    """A gamma that takes one y past the largest float32: its scale is infinite, finite values over it are 0, that one NaN."""
    x, gamma = torch.ones(3, 512), torch.ones(512)
    x[1, 5], gamma[5] = 300.0, 3e38
    q, s, _, _ = cattn.rmsnorm_fwd_q8(x.to(cuda), gamma.to(cuda), None, 1e-5, 0)
    q, s = q.cpu().float(), s.cpu()
    assert torch.isinf(s[1, 0]) and q[1, 5].isnan() and not q[1, :5].any() and not q[1, 6:].any()
    assert s[0, 0].isfinite() and q[[0, 2]].isfinite().all() and q[0, 5] == 448
