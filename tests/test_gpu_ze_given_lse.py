"""Backward calls with an lse that is not the forward's: of a part of the vocabulary, or
of other logits.  p = exp(z - lse) is taken as at most 1, as the header says of all
three operators on the vocabulary's logits.

The tolerances count p's errors, 2^-20 (1 + |z| + |lse|) of p (its exponent's product with
log2(e) and the exponential), the logit's own, dim 2^-23 of the terms' sizes, the weights'
(top + 16) 2^-21, and what the kernels round: the gradient of the logits to bf16 (2^-8),
the result to its type."""
import numpy as np
import pytest
import torch

from oracle import vocab as O
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, draw, half_step, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,dim,V", [(5, 16, 300), (200, 64, 700), (300, 1544, 257)])
def test_hidden_rows(T, dim, V, dtype):
    rng = np.random.default_rng(T)
    x, w = draw(rng, (T, dim), BF), draw(rng, (V, dim), BF, 2.0 / dim ** 0.5)
    x64, w64 = as64(x), as64(w)
    z = x64 @ w64.T
    lse = torch.from_numpy(np.quantile(z, 0.9, axis=1).astype(np.float32)).cuda()      # a tenth of the logits lies above
    y = rng.integers(-1, V, T)
    g = [rng.standard_normal(T).astype(np.float32) for _ in range(3)]
    ent = rng.random(T).astype(np.float32)
    t = lambda v: torch.from_numpy(v).cuda()                                           # noqa: E731
    dx, dw = (torch.full(v.shape, float("nan"), dtype=dtype, device="cuda") for v in (x, w))
    ws = torch.full((nsp.nsp_linear_logp_bwd_workspace(T, dim, V),), 255, dtype=torch.uint8, device="cuda")
    nsp.nsp_linear_logp_bwd(x, w, t(y), lse, dx, dw, ws, g_logp=t(g[0]), g_lse=t(g[1]), g_entropy=t(g[2]), entropy=t(ent))
    torch.cuda.synchronize()
    a, b, c = (v.astype(np.float64)[:, None] for v in g)
    a = np.where(y[:, None] >= 0, a, 0.0)
    l64 = as64(lse)[:, None]
    d = z - l64
    p = np.exp(np.minimum(d, 0.0))
    assert 0.05 < (d > 0).mean() < 0.2 and d.max() > 1
    da = (b - a) * p - c * p * (d + ent.astype(np.float64)[:, None])
    size = (np.abs(a) + np.abs(b) + np.abs(c) * (np.abs(d) + ent[:, None] + 1)) * p
    rows = np.flatnonzero(y >= 0)
    da[rows, y[rows]] += a[rows, 0]
    ez = dim * 2.0 ** -23 * (np.abs(x64) @ np.abs(w64).T)
    off = 2.0 ** -8 * np.abs(da) + size * (2.0 ** -20 * (1 + np.abs(z) + np.abs(l64)) + 2 * ez) + 2.0 ** -22 * np.abs(a)
    for name, got, want, tol, sizes, n in (("dx", dx, da @ w64, off @ np.abs(w64), np.abs(da) @ np.abs(w64), V),
                                           ("dw", dw, da.T @ x64, off.T @ np.abs(x64), np.abs(da).T @ np.abs(x64), T)):
        within(name, as64(got), want, tol + (n + 8) * 2.0 ** -23 * sizes + half_step(dtype) * np.abs(want))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,V,K", [(3, 700, 5), (40, 9001, 64)])
def test_distillation(T, V, K, dtype):
    rng = np.random.default_rng(V)
    z = torch.from_numpy((rng.standard_normal((T, V)) * 3).astype(np.float32)).to(dtype).cuda()
    lse = torch.quantile(z.float(), 0.9, dim=1)
    index, t = rng.integers(0, V, (T, K)), (rng.standard_normal((T, K)) - 4).astype(np.float32)
    g = rng.standard_normal(T).astype(np.float32)
    c = lambda v: torch.from_numpy(v).cuda()                                           # noqa: E731
    dz = torch.empty_like(z)
    nsp.nsp_distill_bwd(z, c(index), c(t), lse, c(g), dz)
    torch.cuda.synchronize()
    z64, l64 = as64(z), as64(lse)[:, None]
    p = np.exp(np.minimum(z64 - l64, 0.0))
    assert (z64 > l64 + 1).any()
    q, _, _ = O.weights(index, t, V)
    want = p * q.sum(1, keepdims=True)
    off = want * (2.0 ** -20 * (1 + np.abs(z64) + np.abs(l64)) + (K + 16) * 2.0 ** -21)
    for r in range(T):
        np.subtract.at(want[r], index[r], q[r])
        np.add.at(off[r], index[r], q[r] * (K + 16) * 2.0 ** -21)
    want *= g[:, None]
    within("dlogits", as64(dz), want, off * np.abs(g)[:, None] + half_step(dtype) * np.abs(want) + 2.0 ** -120)
    assert np.array_equal(O.distill_backward(z64, index, t, l64[:, 0], g), want)
