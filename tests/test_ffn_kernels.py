"""What the compiler made of the feed-forward operators' kernels, read from the built library's code objects as
test_block_kernels.py does."""

import pytest

import test_block_kernels as base


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    base.FAMILIES, keep = "ffn_|dropout_|swa_", base.FAMILIES
    try:
        found = base.kernels.__wrapped__(tmp_path_factory)
    finally:
        base.FAMILIES = keep
    return {n: k for n, k in found.items() if "ffn_" in n or "dropout_" in n}


def test_no_kernel_spills(kernels):
    """All operands of a tile stay in vector registers: nothing goes through scratch memory."""
    assert len(kernels) > 25
    assert {n: k for n, k in kernels.items() if k != (0, 0)} == {}
