"""Which form of the bf16 sliding-window kernels a call takes (paper_2608_00029_amd/csrc/swa_sched.h, compiled with
the host C++ compiler): the cases that the GPU compares with the oracle take every one."""

import os
import shutil
import subprocess

import pytest

from test_gpu_swa_forms import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "swa_sched.h"
using namespace cattn;
int main() {
  int D, B, Hq, Hkv, S, window, sinks;
  while (std::scanf("%d %d %d %d %d %d %d", &D, &B, &Hq, &Hkv, &S, &window, &sinks) == 7) {
    const int w = window < S ? window : S, k = sinks < S ? sinks : S, run = swa_run(S, w, k);
    const int fwd = swa_form(Pass::kFwd, D, (int64_t)B * Hq, S, run), dq = swa_form(Pass::kDq, D, (int64_t)B * Hq, S, run);
    const int dkdv = swa_form(Pass::kDkdv, D, (int64_t)B * Hkv, S, run * (Hq / Hkv));
    const bool shared = dkdv == 4 && swa_far_shares(true, B, Hq, Hkv, S, D, w, k);
    std::printf("%d %d %d %d %d %d\n", fwd, fwd == 1 ? swa_fwd_ring(D, (int64_t)B * Hq, S) : 0, dq, dkdv,
                swa_has_far(true, Hq, Hkv, S, w, k), shared);
  }
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    """{(D, kernel, parts, what else)} of each case: the ring's slots of an undivided forward; in dK/dV where the
    sinks' far queries go."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("forms")
    src, exe = d / "forms.cpp", str(d / "forms")
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2608_00029_amd", "csrc"), str(src),
                    "-o", exe], check=True)
    text = "".join("%d %d %d %d %d %d %d\n" % c[:7] for c in CASES)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(CASES)
    got = []
    for c, line in zip(CASES, out):
        fwd, ring, dq, dkdv, far, shared = map(int, line.split())
        sinks = "no sinks" if c[6] == 0 else "within" if not far else "shared grid" if shared else "own grid"
        got.append({(c[0], "fwd", fwd, ring), (c[0], "dq", dq, 0), (c[0], "dkdv", dkdv, sinks)})
    return got


EVERY = {(D, "fwd", n, ring) for D in (64, 128) for n, ring in ((4, 0), (2, 0), (1, 4), (1, 3)) if (D, ring) != (64, 3)} \
    | {(D, "dq", n, 0) for D in (64, 128) for n in (1, 2, 4)} \
    | {(D, "dkdv", n, s) for D in (64, 128) for n in (1, 2, 4) for s in ("no sinks", "within", "own grid", "shared grid")
       if n == 4 or s != "shared grid"}


def test_every_form_is_compared(forms):
    reached = set().union(*forms)
    assert reached == EVERY, (EVERY - reached, reached - EVERY)


def test_ragged_and_padded():
    """Every case ends inside a tile, and the sequences of a batch in different ones."""
    for D, B, Hq, Hkv, S, window, sinks, lens in CASES:
        assert S % 32 and len(lens) == B and all(0 <= n <= S for n in lens) and (B == 1 or len(set(lens)) > 1)
