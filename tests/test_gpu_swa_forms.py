"""Every form of the bf16 sliding-window kernels, forward and backward, on the GPU against the float64 oracle.  The
cases' forms are derived on the CPU (test_swa_forms.py)."""

import pytest

from test_gpu_swa import check

pytestmark = pytest.mark.gpu

# D, B, Hq, Hkv, S, window, sinks, lens
CASES = [
    # undivided dK/dV (over 1024 groups of 32 keys): without sinks, with their far queries in the walk, in another grid
    (128, 4, 24, 12, 700, 90, 0, [700, 641, 33, 699]),
    (128, 3, 17, 17, 650, 200, 3, [650, 609, 450]),
    (128, 4, 24, 12, 700, 330, 3, [700, 699, 338, 612]),
    (128, 3, 36, 18, 620, 45, 40, [620, 550, 1]),
    (64, 4, 12, 12, 690, 131, 0, [690, 500, 32, 689]),
    (64, 3, 17, 17, 650, 200, 3, [650, 609, 450]),
    (64, 4, 24, 12, 700, 90, 33, [700, 641, 100, 699]),
    # two parts
    (128, 2, 16, 16, 530, 100, 0, [530, 417]),
    (128, 2, 16, 16, 530, 100, 3, [530, 417]),
    (128, 2, 32, 16, 530, 100, 35, [530, 200]),
    (128, 2, 16, 16, 530, 400, 3, [530, 517]),
    (64, 2, 16, 16, 530, 100, 0, [530, 417]),
    (64, 2, 16, 16, 530, 100, 3, [530, 417]),
    (64, 2, 32, 16, 530, 100, 35, [530, 200]),
    # four parts, the far queries in a grid of their own or in the window's
    (128, 8, 4, 2, 500, 100, 3, [500, 469, 438, 500, 129, 64, 0, 499]),
    (128, 2, 8, 2, 500, 60, 0, [500, 333]),
    (128, 2, 2, 2, 500, 60, 20, [500, 333]),
    (128, 2, 8, 2, 500, 60, 2, [500, 333]),
    (64, 8, 32, 4, 500, 100, 3, [500, 469, 438, 500, 129, 64, 0, 499]),
    (64, 2, 8, 2, 500, 60, 0, [500, 333]),
    (64, 2, 2, 2, 500, 60, 20, [500, 333]),
    (64, 2, 8, 2, 500, 60, 2, [500, 333]),
    # undivided forward at D = 128: a ring of four (up to 512 work groups of 128 queries), else of three
    (128, 3, 40, 8, 400, 150, 1, [399, 400, 290]),
]


@pytest.mark.parametrize("D,B,Hq,Hkv,S,window,sinks,lens", CASES)
def test_against_the_oracle(cuda, D, B, Hq, Hkv, S, window, sinks, lens):
    check(cuda, B, Hq, Hkv, S, D, window, sinks, "bf16", lens=lens)
