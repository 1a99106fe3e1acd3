"""MI355X (gfx950) fused causal multi-head attention, forward and backward,
plus the fused loss head and the memory-bound operators (LayerNorm, GELU,
softmax cross entropy) of the same training step, and the operators of a
decoder block's attention half: RMSNorm with the residual added, rotary
positions, sliding-window attention with sinks, in training and for single
tokens.

The compute lives in libcattn.so (HIP kernels behind the C ABI of
include/cattn.h); this package only marshals torch tensors into that ABI.
"""
from .binding import (  # noqa: F401
    CattnError, attn_bwd, attn_bwd_dkdv, attn_bwd_dq, attn_fwd, last_error_string, library_path, status_string, workspace_bytes,
    lmhead_fwd, lmhead_workspace_bytes,
    layernorm_fwd, layernorm_bwd, layernorm_bwd_workspace_bytes, gelu_fwd, gelu_bwd, sce_fwd, sce_bwd,
    CATTN_BF16, CATTN_F32, CATTN_OK, CATTN_ERR_HIP, CATTN_ERR_INVALID_ARG, CATTN_ERR_UNSUPPORTED, CATTN_BHSD, CATTN_BSHD,
)
from .block import (  # noqa: F401
    rmsnorm_fwd, rmsnorm_fwd_q8, rmsnorm_bwd, rmsnorm_bwd_workspace_bytes,
    rope_frequencies, rope_fwd, rope_bwd, rope_append,
    swa_fwd, swa_bwd, swa_bwd_workspace_bytes, swa_decode, swa_decode_workspace_bytes,
)
