"""Which form of the gated projections' kernels a product takes (paper_2608_00029_amd/csrc/ffn_sched.h, compiled with the
host C++ compiler): the cases that the GPU compares with the oracle take every one."""

import os
import shutil
import subprocess

import pytest

from test_gpu_gated_forms import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "ffn_sched.h"
using namespace cattn;
int main() {
  long long T, C, F, bf16;
  while (std::scanf("%lld %lld %lld %lld", &T, &C, &F, &bf16) == 4) {
    const FfnPlan f = ffn_plan(FWD, T, F, C, bf16), x = ffn_plan(DX, T, C, F, bf16), w = ffn_plan(DW, F, C, T, bf16);
    std::printf("%d %d %d %d %d %d %d %lld\n", T < (1LL << 31) ? gated_rows_columns((int)T, (int)F, bf16) : 0, f.form, f.parts,
                x.form, x.parts, w.form, w.parts, (long long)ffn_part_floats(T, C, F, bf16));
  }
}
"""
NAMES = ["256x256", "192x256", "256x128", "128x128", "64x128", "64x64", "128x64"]
BF16, F32 = NAMES[:4] + ["64x64"], NAMES[3:6]  # (128x64: the forward alone)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("forms")
    src, exe = d / "forms.cpp", str(d / "forms")
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2608_00029_amd", "csrc"), str(src), "-o", exe], check=True)

    def run(cases):
        text = "".join("%d %d %d %d\n" % (T, C, F, dtype == "bf16") for T, C, F, dtype in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [tuple(map(int, line.split())) for line in out]
    return run


def forms_of(case, p):
    T, C, F, dtype = case
    rows, ff, fp, xf, xp, wf, wp, _ = p
    assert fp == 1
    fwd = (dtype, "rows", rows, T > 16) if rows else (dtype, "fwd", NAMES[ff], False)
    return {fwd, (dtype, "dx", NAMES[xf], xp > 1), (dtype, "dw", NAMES[wf], wp > 1)}


EVERY = {(d, "rows", n, many) for d, n in (("bf16", 8), ("f32", 8), ("f32", 16)) for many in (False, True)} \
    | {("bf16", "fwd", n, False) for n in BF16 + ["128x64"]} | {("f32", "fwd", n, False) for n in F32} \
    | {("bf16", p, n, parts) for p in ("dx", "dw") for n in BF16 for parts in (False, True)} \
    | {("f32", p, n, parts) for p in ("dx", "dw") for n in F32 for parts in (False, True)}


def test_every_form_is_compared(plan):
    reached = set().union(*(forms_of(c, p) for c, p in zip(CASES, plan(CASES))))
    assert reached == EVERY, (EVERY - reached, reached - EVERY)


def test_a_plan_fits_its_product(plan):
    """No part of k is empty, and the partial sums are counted for the largest of the two products."""
    cases = [(T, C, F, d) for d in ("bf16", "f32") for T in (1, 33, 777, 8192, 65536, 1 << 20) for C in (8, 768, 1600, 8192, 1 << 18)
             for F in (8, 2048, 4288, 1 << 18) if T * C <= 1 << 33 and T * F <= 1 << 33]
    for (T, C, F, d), (_, ff, fp, xf, xp, wf, wp, floats) in zip(cases, plan(cases)):
        chunk = 64 if d == "bf16" else 32
        assert fp == 1 and 1 <= xp <= 2 * -(-F // chunk) and 1 <= wp <= -(-T // chunk)
        assert floats == max(xp * T * C if xp > 1 else 0, 2 * wp * F * C if wp > 1 else 0)
        assert {ff, xf, wf} <= ({0, 1, 2, 3, 5, 6} if d == "bf16" else {3, 4, 5}) and 6 not in (xf, wf)


def test_limits_of_a_launch(plan):
    """The largest shapes that are taken: tiles that an int counts, work items of a launch below 2^32."""
    E = 1 << 33
    for T, C, F in ((1 << 30, 8, 8), (E >> 18, 1 << 18, 1 << 15), (1, 1 << 15, 1 << 18), (E >> 18, 8, 1 << 18), (1 << 25, 256, 8)):
        assert T * C <= E and T * F <= E and F * C <= E
        (_, ff, _, xf, xp, wf, wp, floats), = plan([(T, C, F, "f32")])
        for M, N, parts, two in ((T, F, 1, 1), (T, C, xp, 1), (F, C, wp, 2)):
            assert two * parts * -(-M // 64) * -(-N // 64) < 1 << 31
            assert M * N // 4 < 1 << 32
        assert T * F // 8 < 1 << 32
