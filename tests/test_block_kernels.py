"""What the compiler made of the decoder-block operators' kernels, read from the metadata of the built library's
gfx950 code objects (as test_residency.py does)."""

import re
import subprocess

import pytest

from paper_2608_00029_amd.binding import library_path
from test_residency import READELF, _code_objects

FAMILIES = "rmsnorm_|rope_|swa_"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: (spilled vector registers, bytes of scratch)}"""
    if READELF is None:
        pytest.skip("llvm-readelf not found")
    with open(library_path(), "rb") as f:
        blob = f.read()
    out = {}
    for i, elf in enumerate(_code_objects(blob)):
        path = tmp_path_factory.mktemp("co") / f"{i}.elf"
        path.write_bytes(elf)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for k in re.split(r"\n  - \.agpr_count:", notes)[1:]:
            name = re.search(r"\.name:\s+(\S+)", k)[1]
            if re.search(FAMILIES, name):
                out[name] = tuple(int(re.search(rf"\.{f}:\s+(\d+)", k)[1]) for f in ("vgpr_spill_count", "private_segment_fixed_size"))
    assert len(out) > 50
    return out


def test_no_form_without_a_call(kernels):
    """The forward's ring of three is D = 128's: the rule takes four slots at D = 64 on every grid."""
    rings = {(int(m[1]), int(m[2]), int(m[3])) for m in (re.search(r"swa_fwd_bf16_kernelILi(\d+)ELi(\d)ELi(\d)E", n) for n in kernels) if m}
    assert rings == {(64, 1, 4), (64, 2, 4), (64, 4, 2), (128, 1, 4), (128, 1, 3), (128, 2, 2), (128, 4, 2)}


def test_no_kernel_spills(kernels):
    """All operands of a row or a tile stay in vector registers: nothing goes through scratch memory."""
    assert {n: k for n, k in kernels.items() if k != (0, 0)} == {}
