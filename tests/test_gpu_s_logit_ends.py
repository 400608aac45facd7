"""Logits whose scaled size passes float32, and targets that are masked.

A row's largest logit m with |m scale log2(e)| of 2^128 and more has no lse in
float32: everything that depends on it is NaN, forward and backward, instead of
a number that looks like a result.  Up to there lse is within 2^-21 of itself
(the product with log2(e), its constant, the sum, the product with ln 2)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
INF = float("inf")
LIMIT = math.log(2.0) * 2.0 ** 128               # of m scale: 2.36e38


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _forward(z, y, scale, top=2):
    T, V = z.shape
    o = {n: torch.zeros(T, device="cuda") for n in ("logp", "lse", "entropy")}
    o["top_logp"], o["top_index"] = torch.zeros(T, top, device="cuda"), torch.zeros(T, top, dtype=torch.int64, device="cuda")
    ws = torch.empty(nsp.nsp_token_logp_workspace(T, V, top), dtype=torch.uint8, device="cuda")
    nsp.nsp_token_logp_fwd(z, y, *o.values(), ws, scale=scale)
    torch.cuda.synchronize()
    return o


def _backward(z, y, o, scale, lse=None):
    dz = torch.zeros_like(z)
    g = torch.ones(z.shape[0], device="cuda")
    nsp.nsp_token_logp_bwd(z, y, o["lse"] if lse is None else lse, dz, g_logp=g, g_entropy=g, entropy=o["entropy"], scale=scale)
    torch.cuda.synchronize()
    return dz


# m, scale: past the limit above, below it, at both ends of the scales
PAST = [(3e38, 1.0, F), (3e38, 1.0, BF), (2.0 ** 70, 2.0 ** 64, F), (1e38, 4.0, BF), (-1e37, 2.0 ** 10, F), (-8e37, 4.0, BF), (-2.0 ** 70, 2.0 ** 64, F)]


@pytest.mark.parametrize("V", [7, 5000, 40000])    # (in one part and in several)
@pytest.mark.parametrize("m,scale,dtype", PAST)
def test_past_float32(m, scale, dtype, V):
    z = torch.full((3, V), m * (0.5 if m > 0 else 1.25), device="cuda").clamp_min(-8.4e37).to(dtype)
    z[0, V // 2] = m                             # the others far below
    z[1] = -INF
    z[1, V - 1] = m                              # the others masked
    z[2] = 0.25                                  # (a row with results, and not the others' business)
    y = torch.tensor([V // 2, V - 1, 3], device="cuda")
    o = _forward(z, y, scale)
    for n in ("logp", "lse", "entropy"):
        assert bool(o[n][:2].isnan().all()) and bool(o[n][2].isfinite()), (n, o[n])
    assert bool(o["top_logp"][0].isnan().all()) and bool(o["top_logp"][1, 0].isnan())
    assert o["top_index"][0, 0] == V // 2 and o["top_index"][1].tolist() == [V - 1, -1] and float(o["top_logp"][1, 1]) == -INF
    dz = _backward(z, y, o, scale)
    assert bool(dz[:2].isnan().all()) and bool(dz[2].isfinite().all())
    off = _forward(z, torch.full_like(y, -1), scale)
    assert not off["logp"].any()                 # (an ignored target's stays 0)
    # whoever hands on an lse of infinity gets no plausible gradient for it
    assert bool(_backward(z, y, o, scale, torch.full((3,), INF, device="cuda")).isnan().all())


@pytest.mark.parametrize("V", [7, 5000, 40000])
@pytest.mark.parametrize("m,scale", [(2.0 ** 126, 1.0), (2.3e38, 1.0), (1.1e38, 2.0), (-8e37, 2.0), (-(2.0 - 2.0 ** -23) * 2.0 ** 125, 2.0),
                                     (-(2.0 - 2.0 ** -23) * 2.0 ** 125, 2.7)])
def test_up_to_float32(m, scale, V):
    """The last number above the masked ones among them."""
    assert abs(m) * scale < LIMIT
    z = torch.full((2, V), m, device="cuda")
    z[1, 1:] = -INF
    y = torch.tensor([V - 1, 0], device="cuda")
    o = _forward(z, y, scale)
    want = float(z[0, 0]) * scale
    assert np.abs(as64(o["lse"]) / want - 1).max() <= 2.0 ** -21, (o["lse"], want)
    near = 2.0 ** -20 * (1 + math.log(V))
    assert abs(float(o["logp"][0]) + math.log(V)) <= near and float(o["logp"][1]) == 0
    assert abs(float(o["entropy"][0]) - math.log(V)) <= near and float(o["entropy"][1]) == 0
    assert o["top_index"].tolist() == [[0, 1], [0, -1]]
    assert bool(_backward(z, y, o, scale).isfinite().all())
