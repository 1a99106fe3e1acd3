"""Types that the feed-forward operators do not know are refused alike by all of them: TypeError, "unsupported dtype"."""

import pytest
import torch

import paper_2608_00029_amd as cattn
from paper_2608_00029_amd import ffn


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8])
def test_unsupported_types(monkeypatch, dtype):
    monkeypatch.setattr(ffn, "_on_hip", lambda name, t: None)
    x, w = torch.empty(4, 64, dtype=dtype, device="meta"), torch.empty(32, 64, dtype=dtype, device="meta")
    h = torch.empty(4, 32, dtype=dtype, device="meta")
    for call in (lambda: cattn.gated_bwd_workspace_bytes(4, 64, 32, dtype), lambda: cattn.gated_fwd(x, w, w),
                 lambda: cattn.gated_bwd(x, w, w, h, h, h), lambda: cattn.dropout_fwd(x, 0.1, 1), lambda: cattn.dropout_bwd(x, 0.1, 1)):
        with pytest.raises(TypeError, match=f"unsupported dtype {dtype}"):
            call()
