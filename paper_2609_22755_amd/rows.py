"""The calls on rows (rotary positions, norms of rows, token log probabilities,
embedding, log probabilities from hidden rows, distillation) on torch tensors: the
part of the binding that
``paper_2609_22755_amd.nsp`` offers under the same names, compiled
(binding/rows_module.cpp) because a small call's time is its binding's.

Sizes, strides and types come from the tensors: a wrong one raises TypeError or
ValueError; what the C ABI refuses raises NspError.  A call goes to the GPU that
holds the tensors, by default on its current stream; a Stream of another GPU
raises ValueError.
"""
from __future__ import annotations

import torch


def _current_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


# the handle of a GPU's current stream (without a Stream object around it, where torch has that)
raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)

try:
    from ._rows import (nsp_distill_bwd, nsp_distill_fwd, nsp_embedding_bwd, nsp_embedding_fwd,  # noqa: E402,F401
                        nsp_linear_logp_bwd, nsp_linear_logp_fwd, nsp_norm_bwd, nsp_norm_fwd, nsp_rotary_bwd,
                        nsp_rotary_fwd, nsp_token_logp_bwd, nsp_token_logp_fwd)
except ImportError as e:
    raise ImportError(f"{e}: build it with `python -m paper_2609_22755_amd.build` (there is no non-HIP fallback)") from e
