"""Norms of rows against the float64 definition.

Tolerance: half a step of the type, and N = 64 roundings of float32 (2^-24) on
the size of the terms: a lane adds at most 32 elements one after another, then
at most 10 sums of lanes and waves follow, and the few roundings of the means,
the root, the products.  Rows wider than 16384 (8192 in float32) add n / 1024
one after another: N = 64 + n / 1024."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import F32, as64, draw, half_step, strided, untouched, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
LAYER, RMS = nsp.NSP_NORM_LAYER, nsp.NSP_NORM_RMS


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _roundings(n):
    return (64 + n / 1024) * F32


def _check_fwd(x, w, b, y, mean, rstd, eps, rms):
    x64, n = as64(x), x.shape[-1]
    w64, b64 = (None if t is None else as64(t) for t in (w, b))
    want, m, r = R.norm(x64, w64, b64, eps, rms)
    u, size = _roundings(n), np.abs(x64).mean(-1)
    aw, ab = (1.0 if w64 is None else np.abs(w64)), (0.0 if b64 is None else np.abs(b64))
    d = np.abs(x64 - m[..., None])
    off = (0.0 if rms else 1.0) * u * size
    tol = half_step(y.dtype) * np.abs(want) + u * ab + aw * r[..., None] * (u * d + (off[..., None] if not rms else 0.0))
    within("y", as64(y), want, tol)
    if mean is not None:
        within("mean", as64(mean), m.reshape(-1), u * size.reshape(-1))
    within("rstd", as64(rstd), r.reshape(-1), (r * (u + 0.5 * (off * r) ** 2)).reshape(-1))


def _check_bwd(x, w, dy, mean, rstd, dx, dw, db, rms):
    sh, n = x.shape[:-1], x.shape[-1]
    x64, g64, w64 = as64(x), as64(dy), None if w is None else as64(w)
    m = np.zeros(sh) if rms else as64(mean).reshape(sh)
    r = as64(rstd).reshape(sh)
    want, want_w, want_b = R.norm_backward(x64, w64, g64, m, r, rms)
    u = _roundings(n)
    xh = np.abs((x64 - m[..., None]) * r[..., None])
    h = np.abs(g64 * (1.0 if w64 is None else w64))
    size = h + xh * (h * xh).mean(-1, keepdims=True) + (0.0 if rms else h.mean(-1, keepdims=True))
    within("dx", as64(dx), want, half_step(dx.dtype) * np.abs(want) + u * r[..., None] * size)
    rows = int(np.prod(sh))
    us = (128 + rows / 256) * F32                 # rows of a workgroup, its groups, 32 strands of workgroups
    if dw is not None:
        within("dw", as64(dw), want_w, half_step(dw.dtype) * np.abs(want_w) + us * (np.abs(g64) * xh).reshape(-1, n).sum(0))
    if db is not None:
        within("db", as64(db), want_b, half_step(db.dtype) * np.abs(want_b) + us * np.abs(g64).reshape(-1, n).sum(0))


def _both(x, w, b, kind, eps=1e-6, dy=None, strides=None):
    """Forward and backward of one call, checked; returns every output."""
    n, rows = x.shape[-1], x.numel() // x.shape[-1]
    rms, f32 = kind == RMS, dict(dtype=F, device="cuda")
    rng = np.random.default_rng(rows * 7 + n)
    dy = draw(rng, x.shape, x.dtype) if dy is None else dy
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd = torch.full((rows,), float("nan"), **f32), torch.full((rows,), float("nan"), **f32)
    nsp.nsp_norm_fwd(x, w, b, y, mean, rstd, eps=eps, kind=kind)
    wt = x.dtype if w is None else w.dtype
    dw, db = (torch.full((n,), float("nan"), dtype=wt, device="cuda") for _ in range(2))
    T, H = x.shape[0], x.shape[1] if x.dim() == 3 else 1
    ws = torch.full((nsp.nsp_norm_bwd_workspace(T, H, n),), 255, dtype=torch.uint8, device="cuda")
    nsp.nsp_norm_bwd(x, w, dy, None if rms else mean, rstd, dx, dw, db, ws, kind=kind)
    torch.cuda.synchronize()
    _check_fwd(x, w, b, y, None if rms else mean, rstd, eps, rms)
    assert not rms or bool(mean.isnan().all())                     # not written
    _check_bwd(x, w, dy, mean, rstd, dx, dw, db, rms)
    return y, mean, rstd, dx, dw, db


WIDTHS = [1, 2, 7, 8, 9, 63, 64, 127, 128, 129, 255, 256, 500, 512, 1024, 1111, 2048, 2049, 4096, 5000, 8192, 8200, 16384, 16385, 40001, 65536]


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("dtype,wtype", [(BF, BF), (BF, F), (F, F), (F, BF)])
@pytest.mark.parametrize("n", WIDTHS)
def test_against_the_definition(n, dtype, wtype, kind):
    rng = np.random.default_rng(n)
    rows = 37 if n <= 8200 else 3
    x = draw(rng, (rows, n), dtype, 2.0, 0.7)
    w, b = draw(rng, (n,), wtype, 0.3, 1.0), draw(rng, (n,), wtype)
    _both(x, w, b, kind, eps=1e-5)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("rows,n,dtype", [(1, 128, BF), (1, 4096, F), (2, 64, F), (3001, 128, BF), (20011, 100, F), (5000, 1111, F), (2100, 2048, BF),
                                          (1500, 8192, BF)])
def test_few_and_many_rows(rows, n, dtype, kind):
    rng = np.random.default_rng(rows)
    _both(draw(rng, (rows, n), dtype), draw(rng, (n,), dtype, 0.3, 1.0), None, kind)


@pytest.mark.parametrize("dtype", [BF, F])
def test_without_weights(dtype):
    rng = np.random.default_rng(3)
    _both(draw(rng, (33, 200), dtype), None, None, LAYER)


def test_a_middle_far_from_zero():
    """Rows whose mean is 300 times their spread: the squares are of the
    differences, not differences of squares."""
    rng = np.random.default_rng(4)
    for n in (128, 1000, 20000):
        _both(draw(rng, (9, n), F, 1.0, 300.0), None, None, LAYER, eps=0.0)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [128, 100, 2056])
def test_heads_of_a_projection(n, dtype):
    """Heads where they lie, at any alignment, in place, gradients into a
    strided view; what lies between stays as it is."""
    rng = np.random.default_rng(5)
    x, dy = draw(rng, (21, 3, n), dtype), draw(rng, (21, 3, n), dtype)
    w = draw(rng, (n,), dtype, 0.3, 1.0)
    y, _, rstd, dx, dw, _ = _both(x, w, None, RMS, dy=dy)
    for lead, gap, token_gap in ((1, 5, 7), (8, 8, 64)):
        xv, xb, xm = strided(x, lead, gap, token_gap)
        gv, gb, gm = strided(dy, lead + 2, gap + 2, token_gap)
        ov, ob, om = strided(torch.zeros_like(x), lead + 1, gap + 1, token_gap)
        ws = torch.empty(nsp.nsp_norm_bwd_workspace(21, 3, n), dtype=torch.uint8, device="cuda")
        dw2 = torch.empty_like(dw)
        nsp.nsp_norm_bwd(xv, w, gv, None, rstd, ov, dw2, None, ws, kind=RMS)
        torch.cuda.synchronize()
        assert torch.equal(ov, dx) and torch.equal(dw2, dw) and torch.equal(xv, x)
        assert all(untouched(*t) for t in ((xb, xm), (gb, gm), (ob, om)))
        nsp.nsp_norm_bwd(xv, w, gv, None, rstd, gv, dw2, None, ws, kind=RMS)          # dx over dy
        torch.cuda.synchronize()
        assert torch.equal(gv, dx) and torch.equal(dw2, dw) and untouched(gb, gm)
        gv.copy_(dy)
        nsp.nsp_norm_fwd(xv, w, None, ov, eps=1e-6, kind=RMS)
        nsp.nsp_norm_fwd(xv, w, None, xv, eps=1e-6, kind=RMS)                         # y over x
        torch.cuda.synchronize()
        assert torch.equal(ov, y) and torch.equal(xv, y) and untouched(xb, xm) and untouched(ob, om)
        xv.copy_(x)
        nsp.nsp_norm_bwd(xv, w, gv, None, rstd, xv, None, None, None, kind=RMS)       # dx over x, no weights' gradient
        torch.cuda.synchronize()
        assert torch.equal(xv, dx) and untouched(xb, xm)


def test_a_broadcast_gradient():
    rng = np.random.default_rng(6)
    x, g = draw(rng, (40, 96), F), draw(rng, (1, 96), F)
    _both(x, draw(rng, (96,), F), None, LAYER, dy=g.expand(40, 96))


def test_no_rows():
    w = torch.ones(100, dtype=BF, device="cuda")
    e = torch.empty(0, 100, dtype=BF, device="cuda")
    f = torch.empty(0, dtype=F, device="cuda")
    dw, db = torch.full_like(w, 7.0), torch.full_like(w, 7.0)
    nsp.nsp_norm_fwd(e, w, None, e, f, f)
    nsp.nsp_norm_bwd(e, w, e, f, f, e, dw, db, None)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()


def test_a_nan_stays_in_its_row():
    rng = np.random.default_rng(12)
    x = draw(rng, (10, 130), BF)
    clean = torch.empty_like(x)
    nsp.nsp_norm_fwd(x, None, None, clean)
    x[4, 129] = float("nan")
    x[7, 3] = float("inf")
    y = torch.empty_like(x)
    nsp.nsp_norm_fwd(x, None, None, y)
    torch.cuda.synchronize()
    bad = torch.tensor([4, 7], device="cuda")
    assert bool(y[4].isnan().all()) and bool(y[7].isnan().any())
    keep = torch.ones(10, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(y[keep], clean[keep])


def test_repeatable_on_a_side_stream_and_replayed():
    """The same bits from every run, from a side stream and from a graph whose
    replays alternate with eager calls; two graphs with workspaces of their own."""
    rng = np.random.default_rng(13)
    n, rows = 384, 3000
    x, dy, w = draw(rng, (rows, n), BF), draw(rng, (rows, n), BF), draw(rng, (n,), BF, 0.3, 1.0)
    y, mean, rstd, dx, dw, db = _both(x, w, None, LAYER, dy=dy)
    size = nsp.nsp_norm_bwd_workspace(rows, 1, n)
    s = torch.cuda.Stream()
    sets = []
    for k in range(3):
        out = [torch.zeros_like(t) for t in (dx, dw, db)]
        sets.append((out, torch.empty(size, dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    out, ws = sets[0]
    nsp.nsp_norm_bwd(x, w, dy, mean, rstd, *out, ws, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, (dx, dw, db)))
    graphs = []
    for out, ws in sets[1:]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nsp.nsp_norm_fwd(x, w, None, y, mean, rstd)
            nsp.nsp_norm_bwd(x, w, dy, mean, rstd, *out, ws)
        graphs.append(g)
    for k in range(3):
        x.copy_(draw(rng, x.shape, BF))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        eager, ws = sets[0]
        nsp.nsp_norm_bwd(x, w, dy, mean, rstd, *eager, ws)
        torch.cuda.synchronize()
        _check_bwd(x, w, dy, mean, rstd, *eager, False)
        for out, _ in sets[1:]:
            assert all(torch.equal(a, b) for a, b in zip(out, eager))
