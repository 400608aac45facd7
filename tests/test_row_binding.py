"""The row calls' binding refuses what its C arguments do not hold, before anything
is asked of a GPU (which these stand-ins for tensors are not on)."""
import types

import pytest
import torch

from paper_2609_22755_amd import nsp


class OnGpu:
    """What the binding asks of a tensor, on a GPU that need not be there."""

    def __init__(self, shape, dtype, gpu=0):
        self.shape, self.dtype, self.gpu = tuple(shape), dtype, gpu

    def stride(self):
        s, out = 1, []
        for n in reversed(self.shape):
            out.insert(0, s)
            s *= n
        return tuple(out)

    def numel(self):
        n = 1
        for d in self.shape:
            n *= d
        return n

    def get_device(self):
        return self.gpu

    def data_ptr(self):
        return 0x10000

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.dtype.itemsize


F = torch.float32


def _stream(gpu):
    return types.SimpleNamespace(cuda_stream=0, device_index=gpu)


def test_a_stream_of_another_gpu_is_refused():
    if torch.cuda.device_count() > 0:
        pytest.skip("stand-ins for tensors, for a machine without a GPU")
    x, z, v = OnGpu((4, 64), F, 1), OnGpu((4, 90), F, 1), OnGpu((4,), F, 1)
    for call in (lambda s: nsp.nsp_norm_fwd(x, None, None, x, stream=s), lambda s: nsp.nsp_token_logp_fwd(z, None, None, v, stream=s),
                 lambda s: nsp.nsp_token_logp_bwd(z, None, v, z, stream=s)):
        for gpu in (0, 2):
            with pytest.raises(ValueError, match=f"stream: of GPU {gpu}, the tensors are on GPU 1"):
                call(_stream(gpu))


def test_numbers_past_32_bits_are_refused():
    x, w = torch.zeros(4, 2, 64), torch.zeros(64)
    pos, freqs = torch.zeros(4, dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
    for n in (1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 31):
        with pytest.raises(ValueError, match="kind"):
            nsp.nsp_norm_fwd(x, w, None, x, kind=n)
        with pytest.raises(ValueError, match="kind"):
            nsp.nsp_norm_bwd(x, w, x, None, torch.zeros(8), x, None, None, None, kind=n)
        with pytest.raises(ValueError, match="layout"):
            nsp.nsp_rotary_fwd(pos, freqs, x, x, layout=n)
