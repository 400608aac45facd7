"""Log probabilities from hidden rows: gradients where the vocabulary ends inside a
vector of eight, or inside a tile, with logits far below zero and a large scale.
What the kernels make of the columns past the end must not reach a result.

All logits of a row are the same number a, exact in bf16, with scale 2^s: z = a 2^s, lse
as the forward gives it (ln V is lost beside 2^s), so z - lse = 0 and p = 1 of the lse
given, and
    da = 2^s (g_logp (1[target] - 1) + g_lse - g_entropy H)
is one number for every column but the target's; past the end z would be 0 and its
exponent 2^s, times g_entropy 2^s past float32.  w differs from column to column in
elements that x is zero in, so every column counts in dx.

Tolerance: da's terms and their sum 4 steps of 2^-24, a rounding to bf16 (2^-8), V (or T)
additions of 2^-24 of the sizes' sum, half a step of the result's type, relative to the
sizes' sum."""
import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, half_step, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _ws(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None


# (the last four: sums of the logits in parts over the width)
@pytest.mark.parametrize("T,dim,V", [(1, 8, 1), (3, 16, 9), (40, 16, 255), (128, 64, 1003), (130, 16, 257), (300, 64, 1003), (600, 8, 5),
                                     (1, 1536, 3), (7, 2048, 300), (130, 1536, 513), (300, 2048, 1001)])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("s", [0, 20, 64])
def test_columns_past_the_end(T, dim, V, dtype, s):
    rng = np.random.default_rng(T + V + s)
    scale = 2.0 ** s
    x, w = np.zeros((T, dim), np.float32), np.zeros((V, dim), np.float32)
    x[:, 0] = rng.integers(1, 3, T)                      # logits of -1 and -2
    w[:, 0] = -1.0
    w[:, 1:] = rng.integers(-2, 3, (V, dim - 1))
    x, w = (torch.from_numpy(v).to(BF).cuda() for v in (x, w))
    y = torch.from_numpy(rng.integers(-1, V, T)).cuda()
    g = [torch.from_numpy((rng.integers(1, 5, T) * rng.choice([-1.0, 1.0], T)).astype(np.float32)).cuda() for _ in range(3)]
    o = [torch.empty(T, device="cuda") for _ in range(3)]
    nsp.nsp_linear_logp_fwd(x, w, y, *o, _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V)), scale=scale)
    logp, lse, ent = o
    ws = _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V))
    for use in ((1, 0, 0), (0, 0, 1), (1, 1, 1)):
        gl, gs, ge = (t if u else None for t, u in zip(g, use))
        dx, dw = (torch.full(v.shape, float("nan"), dtype=dtype, device="cuda") for v in (x, w))
        nsp.nsp_linear_logp_bwd(x, w, y, lse, dx, dw, ws, g_logp=gl, g_lse=gs, g_entropy=ge, entropy=ent if ge is not None else None, scale=scale)
        torch.cuda.synchronize()
        d = as64(x[:, 0]) * -scale - as64(lse)
        p = np.exp(np.minimum(d, 0.0))
        zero = np.zeros(T)
        yy = y.cpu().numpy()
        a, b, c = (zero if t is None else as64(t) for t in (gl, gs, ge))
        a = np.where(yy >= 0, a, 0.0)
        da = np.broadcast_to((scale * p * (b - a - c * (d + as64(ent))))[:, None], (T, V)).copy()
        size = np.broadcast_to((scale * p * (np.abs(a) + np.abs(b) + np.abs(c) * (np.abs(d) + np.abs(as64(ent)))))[:, None], (T, V)).copy()
        rows = np.flatnonzero(yy >= 0)
        da[rows, yy[rows]] += scale * a[rows]
        size[rows, yy[rows]] += scale * np.abs(a[rows])
        x64, w64 = as64(x), as64(w)
        # (p: the exponent's own steps, 2^-21 (1 + |z| + |lse|) where ln V is not lost)
        off = 2.0 ** -8 * np.abs(da) + size * (4 * 2.0 ** -24 + np.where(d == 0, 0.0, 2.0 ** -21 * (1 + 2 * np.abs(as64(lse)) + 2 * scale))[:, None])
        for name, got, want, tol, sizes, n in (("dx", dx, da @ w64, off @ np.abs(w64), size @ np.abs(w64), V),
                                               ("dw", dw, da.T @ x64, off.T @ np.abs(x64), size.T @ np.abs(x64), T)):
            within(f"{name} {use}", as64(got), want, tol + (n + 8) * 2.0 ** -24 * sizes + half_step(dtype) * np.abs(want) + 2.0 ** -120)
