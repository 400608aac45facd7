"""Norms without eps of rows whose variance float32 holds as a subnormal number.

Tolerance: a square and the mean's last product are each off by half a step of
the subnormal numbers at most (2^-150), sums of such numbers are exact, so v is
off by 2^-149 and N = 64 + n / 1024 roundings of 2^-24, and rstd by half of
both; y by rstd's and three roundings, and with a mean by the mean's N roundings
of the row's largest number."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import F32, as64, draw, half_step, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("rms", [True, False])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [5, 128, 1000, 5000, 16384, 20000])
def test_variances_below_the_normal_numbers(n, dtype, rms):
    rng = np.random.default_rng(n)
    x = draw(rng, (6, n), dtype)
    x *= torch.tensor([2.0 ** -e for e in (60, 64, 65, 66, 68, 0)], device="cuda")[:, None].to(dtype)
    y = torch.empty_like(x)
    mean, rstd = (torch.empty(6, dtype=F, device="cuda") for _ in range(2))
    nsp.nsp_norm_fwd(x, None, None, y, mean, rstd, eps=0.0, kind=nsp.NSP_NORM_RMS if rms else nsp.NSP_NORM_LAYER)
    torch.cuda.synchronize()
    x64 = as64(x)
    want, m, r = R.norm(x64, None, None, 0.0, rms)
    v = r ** -2.0
    assert v[0] > 2.0 ** -126 > v[2] and v[4] > 2.0 ** -140
    u = (64 + n / 1024) * F32
    off = 0.0 if rms else u * np.abs(x64).max(-1)
    tol = r * (u + 0.5 * (2.0 ** -149 + off ** 2) / v)
    within("rstd", as64(rstd), r, tol)
    d = np.abs(x64 - m[:, None])
    within("y", as64(y), want, half_step(dtype) * np.abs(want) + d * tol[:, None] + r[:, None] * (3 * F32 * d + np.broadcast_to(off, r.shape)[:, None]))
