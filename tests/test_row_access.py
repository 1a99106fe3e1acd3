"""The accesses of rows that may begin at any element (paper_2608_00029_amd/csrc/row_access.h), compiled for the
host with the alignment sanitizer: an access wider than the elements at an address that is no multiple of its
width traps."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#define __device__
#define __forceinline__ inline
#include "row_access.h"
using namespace cattn;
template <int V, bool NT> int check(int offset) {
  alignas(16) static float in[16], out[16];
  for (int i = 0; i < 16; ++i) in[i] = i + 1, out[i] = 0;
  store_v<float, V, NT>(out + offset, load_v<float, V>(in + offset));
  int bad = 0;
  for (int i = 0; i < 16; ++i) bad += out[i] != (i >= offset && i < offset + V ? in[i] : 0.f);
  return bad;
}
int main() {
  int bad = check<4, false>(0) + check<4, true>(4);
  for (int offset = 0; offset < 8; ++offset)
    bad += check<1, false>(offset) + check<1, true>(offset) + check<2, false>(offset) + check<2, true>(offset);
  std::printf("bad=%d\n", bad);
}
"""


def test_elements_at_any_address(tmp_path):
    cxx = shutil.which("clang++", path="/opt/rocm/llvm/bin:" + os.environ.get("PATH", ""))
    if cxx is None:
        pytest.skip("no clang++ (the header uses its vector types)")
    src, exe = tmp_path / "row_access.cpp", str(tmp_path / "row_access")
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fsanitize=alignment", "-fsanitize-trap=alignment", "-I",
                    os.path.join(ROOT, "paper_2608_00029_amd", "csrc"), str(src), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "bad=0\n", (out.returncode, out.stdout)
