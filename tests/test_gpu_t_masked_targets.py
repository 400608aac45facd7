"""A masked target (a logit of -2^126 and below, finite or not) has probability
0 and so a log probability of -inf, whatever the scale makes of its logit."""
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [9, 5000])
@pytest.mark.parametrize("scale", [2.0 ** -64, 0.25, 1.0, 2.0])
def test_a_masked_target(scale, V, dtype):
    z = torch.zeros(6, V, dtype=dtype, device="cuda")
    z[:, 4] = torch.tensor([torch.finfo(dtype).min, -(2.0 ** 126), -1e38, float("-inf"), -1e38, -1e38], device="cuda").to(dtype)
    z[4, 0] = float("nan")
    y = torch.full((6,), 4, device="cuda")
    y[5] = -1
    logp, lse = torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda")
    ws = torch.empty(nsp.nsp_token_logp_workspace(6, V), dtype=torch.uint8, device="cuda")
    nsp.nsp_token_logp_fwd(z, y, logp, lse, workspace=ws, scale=scale)
    torch.cuda.synchronize()
    assert bool((logp[:4] == float("-inf")).all()) and bool(logp[4].isnan()) and float(logp[5]) == 0, logp
