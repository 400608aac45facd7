"""Log probabilities from hidden rows against the float64 definition.

Tolerances, with A = max_v sum_k |x_k w_vk| of a token:
    logits   products of bf16 are exact in float32; dim additions, each within a
             step (2^-23) of at most A, and the scale: ez = scale (dim + 8) 2^-23 A
    lse      a lane adds 64 terms of a tile, tiles are joined 16 at a time: S = 64 +
             V / 4096 + 40 additions, each exponent within 2^-23 (|z| + |m| + |d|):
             ez + (S + 24) 2^-24 + 2^-21 (max|z| + ln V + 12)
    entropy  2 ez (ln V + 12) + (S + 64) 2^-22 (ln V + 12)
    logp     that of lse, ez and 2^-23 (|z| + |lse|)
    da       a rounding to bf16 (2^-8), and p (2^-21 (1 + |z| + |lse|) + 2 ez)
             times the sizes of its coefficients, and 2^-23 of the target's own
    dx, dw   the sums of da's with |w|, |x|; their own additions, one for each
             term and a step of 2^-23 of the sizes' sum; half a step of the type."""
import math

import numpy as np
import pytest
import torch

from oracle import vocab as O
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, draw, half_step, strided, untouched, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _inputs(T, dim, V, seed, spread=2.0):
    rng = np.random.default_rng(seed)
    x, w = draw(rng, (T, dim), BF), draw(rng, (V, dim), BF, spread / math.sqrt(dim))
    y = torch.from_numpy(rng.integers(-1, V + 1, T)).cuda()      # ignored ones on both sides
    return rng, x, w, y


def _ws(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None


def _forward(x, w, y, scale=1.0):
    T, (V, dim) = x.shape[0], w.shape
    o = {n: torch.full((T,), -7.0, device="cuda") for n in ("logp", "lse", "entropy")}
    nsp.nsp_linear_logp_fwd(x, w, y, o["logp"], o["lse"], o["entropy"], _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V)), scale=scale)
    return o


def _backward(x, w, y, o, g, scale=1.0, dtype=BF, dx=True, dw=True):
    """g: gradients of logp, lse, entropy, or None."""
    T, (V, dim) = x.shape[0], w.shape
    dx = torch.full((T, dim), NAN, dtype=dtype, device="cuda") if dx is True else dx
    dw = torch.full((V, dim), NAN, dtype=dtype, device="cuda") if dw is True else dw
    nsp.nsp_linear_logp_bwd(x, w, y, o["lse"], dx, dw, _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V)), g_logp=g[0], g_lse=g[1],
                            g_entropy=g[2], entropy=o["entropy"] if g[2] is not None else None, scale=scale)
    return dx, dw


def _logit_error(x64, w64, scale):
    A = np.abs(x64) @ np.abs(w64).T
    return scale * (x64.shape[1] + 8) * 2.0 ** -23 * A.max(1)


def _check_fwd(x, w, y, o, scale):
    x64, w64 = as64(x), as64(w)
    V = len(w64)
    want = O.linear_logp(x64, w64, y.cpu().numpy(), scale)
    ez = _logit_error(x64, w64, scale)
    S, ln = 64 + V / 4096 + 40, math.log(V) + 12
    big = np.abs(x64 @ w64.T).max(1) * scale
    tl = ez + (S + 24) * 2.0 ** -24 + 2.0 ** -21 * (big + ln)
    within("lse", as64(o["lse"]), want["lse"], tl)
    within("entropy", as64(o["entropy"]), want["entropy"], 2 * ez * ln + (S + 64) * 2.0 ** -22 * ln)
    within("logp", as64(o["logp"]), want["logp"], tl + ez + 2.0 ** -23 * (big + np.abs(want["lse"])))


def _check_bwd(x, w, y, o, g, dx, dw, scale):
    x64, w64, l64, e64 = as64(x), as64(w), as64(o["lse"]), as64(o["entropy"])
    gs = [None if t is None else as64(t) for t in g]
    t = None if y is None else y.cpu().numpy()
    want_dx, want_dw, da = O.linear_logp_backward(x64, w64, t, l64, e64, *gs, scale=scale)
    live = np.abs(da).max(1) > 0
    x64 = np.where(live[:, None], x64, 0.0)
    z = x64 @ w64.T * scale
    d = z - l64[:, None]
    p = np.exp(d) * live[:, None]
    c = np.zeros_like(p)
    for v in gs[:2]:
        if v is not None:
            c += np.abs(v)[:, None]
    if gs[2] is not None:
        c += np.abs(gs[2])[:, None] * (np.abs(d) + np.abs(e64)[:, None] + 1)
    ez = _logit_error(x64, w64, scale)[:, None]
    tol = 2.0 ** -8 * np.abs(da) + (2.0 ** -21 * (1 + np.abs(z) + np.abs(l64)[:, None]) + 2 * ez) * p * c * scale * 1.01
    if gs[0] is not None:
        for r, v in enumerate(t):
            if 0 <= v < len(w64):
                tol[r, v] += 2.0 ** -23 * abs(gs[0][r]) * scale
    T, V = da.shape
    for name, got, want, left, right, n in (("dx", dx, want_dx, (tol, np.abs(da)), np.abs(w64), V),
                                            ("dw", dw, want_dw, (tol.T, np.abs(da).T), np.abs(x64), T)):
        if got is not None:
            bound = left[0] @ right + (n + 8) * 2.0 ** -23 * (left[1] @ right) + half_step(got.dtype) * np.abs(want)
            within(name, as64(got), want, bound + 2.0 ** -120)


SIZES = [(1, 8, 1), (1, 64, 2), (3, 16, 257), (32, 40, 256), (33, 72, 300), (64, 64, 513), (65, 136, 1000), (100, 32, 31), (128, 256, 255),
         (129, 264, 511), (257, 64, 1025), (300, 1000, 777), (520, 72, 2100), (24, 512, 9001), (3000, 64, 300)]


@pytest.mark.parametrize("T,dim,V", SIZES)
def test_against_the_definition(T, dim, V):
    _, x, w, y = _inputs(T, dim, V, T + V)
    for scale in (1.0, 0.6):
        _check_fwd(x, w, y, _forward(x, w, y, scale), scale)


@pytest.mark.parametrize("T,dim,V", SIZES)
def test_gradient(T, dim, V):
    rng, x, w, y = _inputs(T, dim, V, T * V)
    o = _forward(x, w, y, 0.8)
    g = [torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda() for _ in range(3)]
    for use, dtype in (((1, 0, 0), BF), ((1, 1, 1), F), ((0, 0, 1), BF), ((0, 1, 0), F)):
        gg = [t if u else None for t, u in zip(g, use)]
        yy = y if use[0] else None
        dx, dw = _backward(x, w, yy, o, gg, 0.8, dtype)
        torch.cuda.synchronize()
        _check_bwd(x, w, yy, o, gg, dx, dw, 0.8)


# wide rows, few tiles of logits: sums in parts over dim
WIDE = [(1, 1024, 1), (7, 1032, 300), (33, 2056, 600), (70, 4104, 100), (130, 1536, 513), (300, 2048, 1000), (513, 1096, 257), (24, 8192, 3001)]


@pytest.mark.parametrize("T,dim,V", WIDE)
def test_wide_rows_of_few_tiles(T, dim, V):
    rng, x, w, y = _inputs(T, dim, V, T + dim)
    off = torch.from_numpy(rng.random(T) < 0.2).cuda()
    o = _forward(x, w, y, 0.8)
    _check_fwd(x, w, y, o, 0.8)
    again = _forward(x, w, y, 0.8)
    assert all(torch.equal(o[n], again[n]) for n in o)
    g = [torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda().masked_fill(off, 0.0) for _ in range(3)]
    for use, dtype in (((1, 0, 0), BF), ((1, 1, 1), F)):
        gg = [t if u else None for t, u in zip(g, use)]
        dx, dw = _backward(x, w, y, o, gg, 0.8, dtype)
        dx2, dw2 = _backward(x, w, y, o, gg, 0.8, dtype)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
        _check_bwd(x, w, y, o, gg, dx, dw, 0.8)


def test_wide_rows_that_are_lost():
    """As in test_rows_that_are_lost, with sums in parts."""
    rng, x, w, y = _inputs(50, 2048, 400, 12)
    y = y.clamp(0, 399)
    o = _forward(x, w, y)
    bad = x.clone()
    bad[7, 3], bad[20, 1500] = NAN, float("inf")
    o2 = _forward(bad, w, y)
    lost = torch.zeros(50, dtype=torch.bool, device="cuda")
    lost[[7, 20]] = True
    for n in o:
        assert o2[n][lost].isnan().all() and torch.equal(o2[n][~lost], o[n][~lost]), n
    g = torch.ones(50, device="cuda")
    dx, dw = _backward(bad, w, y, o2, (g, None, None))
    assert dx[lost].isnan().all() and not dx[~lost].isnan().any() and dw.isnan().all()
    # logits of -inf alone
    big = torch.full((1, 2048), 3e38, dtype=BF, device="cuda")
    o3 = _forward(big, torch.full_like(w, -1.0), y[:1].contiguous())
    assert o3["lse"].item() == -math.inf and o3["entropy"].item() == 0 and o3["logp"].item() == -math.inf
    # some of them
    wneg = torch.zeros_like(w)
    wneg[:200] = -1.0
    o4 = _forward(big, wneg, torch.tensor([3], device="cuda"))
    assert abs(o4["lse"].item() - math.log(200)) < 1e-5 and abs(o4["entropy"].item() - math.log(200)) < 1e-5 and o4["logp"].item() == -math.inf


@pytest.mark.parametrize("T,dim,V", [(1, 64, 700), (31, 72, 500), (33, 264, 1000), (64, 64, 3000), (65, 1032, 300), (127, 136, 1000), (128, 2048, 300)])
def test_gradients_of_few_tokens(T, dim, V):
    """Up to 128 tokens the gradient of the logits is kept to 2^-16 of itself (twice half a step
    of bf16); p's own errors, 2^-21 (1 + |z| + |lse|) and the logits', are below that at these
    sizes.  The sizes' sum of dx and dw is at most 4 times the result (a target's against the
    others'): relative 2-norms of float32 gradients within 4 (2^-16 + 2^-16) < 2^-12, a fifth
    of what one rounding to bf16 leaves.  All weights alike, so that its errors are too."""
    rng, x, w, y = _inputs(T, dim, V, 5 * T)
    y = y.clamp(0, V - 1)
    o = _forward(x, w, y)
    g = torch.full((T,), -1.0 / 3.0, device="cuda")
    dx, dw = _backward(x, w, y, o, (g, None, None), dtype=F)
    want_dx, want_dw, _ = O.linear_logp_backward(as64(x), as64(w), y.cpu().numpy(), as64(o["lse"]), as64(o["entropy"]), as64(g))
    for name, got, want in (("dx", dx, want_dx), ("dw", dw, want_dw)):
        off = float(np.linalg.norm(as64(got) - want) / np.linalg.norm(want))
        print(f"[rows] {name}: {off:.2e}", flush=True)
        assert off <= 2.0 ** -12, (name, off)


def test_gradient_against_differences():
    """Differences of the forward along a direction, by steps of x that bf16 holds: x on
    a grid of 2^-4 below 4, steps of 2^-4.  The third-order term is below
    step^3 / 6 times max|w . direction|^3 (sum of |g| = 2.2; coefficients 6 of its
    third derivative) and values round at 2^-21 of their size; the gradient itself is
    off by a rounding of da, 2^-8."""
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.integers(-16, 17, (4, 8)) / 16.0).to(BF).cuda()
    w = torch.from_numpy(rng.integers(-8, 9, (37, 8)) / 16.0).to(BF).cuda()
    y = torch.tensor([3, 36, 0, -1], device="cuda")
    c = [1.0, 0.5, -0.7]
    o = _forward(x, w, y)
    dx, _ = _backward(x, w, y, o, [torch.full((4,), v, device="cuda") for v in c], dtype=F)

    def f(v):
        r = _forward(v, w, y)
        return c[0] * as64(r["logp"]) + c[1] * as64(r["lse"]) + c[2] * as64(r["entropy"])
    h = 2.0 ** -4
    for k in range(8):
        up, down = x.clone(), x.clone()
        up[:, k] += h
        down[:, k] -= h
        d = (f(up) - f(down)) / (2 * h)
        assert np.abs(d - as64(dx)[:, k]).max() <= h ** 2 * 2.2 * 0.5 ** 3 + 2.0 ** -19 / h + 2.0 ** -8 * 2.2 * 2 * 0.5


def test_pieces_of_the_vocabulary():
    """More than one piece (2^28 elements of the gradient of the logits), against
    float64 on the GPU: relative 2-norms within the roundings of da (2^-8) and of the
    result (2^-8)."""
    T, dim, V = 20011, 24, 30011
    rng, x, w, y = _inputs(T, dim, V, 3)
    assert 3 * 2 ** 28 > T * V > 2 ** 29
    o = _forward(x, w, y)
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    dx, dw = _backward(x, w, y, o, (g, None, None))
    dx2, dw2 = _backward(x, w, y, o, (g, None, None))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    x64, w64 = x.double(), w.double()
    dx_ref, dw_ref = torch.empty_like(x64), torch.zeros_like(w64)
    for a in range(0, T, 4096):
        z = x64[a:a + 4096] @ w64.t()
        lse = torch.logsumexp(z, 1)
        assert (o["lse"][a:a + 4096].double() - lse).abs().max() < 1e-4
        yy = y[a:a + 4096]
        given = (yy >= 0) & (yy < V)
        gg = torch.where(given, g[a:a + 4096].double(), 0.0)[:, None]
        da = -gg * (z - lse[:, None]).exp()
        da.scatter_add_(1, yy.clamp(0, V - 1)[:, None], gg)
        dx_ref[a:a + 4096] = da @ w64
        dw_ref += da.t() @ x64[a:a + 4096]
    for got, ref in ((dx, dx_ref), (dw, dw_ref)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -7


def test_views_with_strides():
    rng, x, w, y = _inputs(70, 72, 300, 9)
    xs, _, _ = strided(x, 8, 24)
    ws, _, _ = strided(w, 16, 8)
    o, o2 = _forward(x, w, y), _forward(xs, ws, y)
    assert all(torch.equal(o[n], o2[n]) for n in o)
    g = [torch.from_numpy(rng.standard_normal(70).astype(np.float32)).cuda(), None, None]
    want = _backward(x, w, y, o, g)
    dx, bx, outx = strided(torch.zeros_like(x), 8, 16)
    dw, bw, outw = strided(torch.zeros_like(w), 24, 8)
    _backward(xs, ws, y, o, g, dx=dx, dw=dw)
    torch.cuda.synchronize()
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and untouched(bx, outx) and untouched(bw, outw)
    # one gradient at a time
    assert torch.equal(_backward(x, w, y, o, g, dw=None)[0], want[0]) and torch.equal(_backward(x, w, y, o, g, dx=None)[1], want[1])
    # the same row for every token
    one = x[:1].expand(70, 72)
    o3, o4 = _forward(one, w, y), _forward(one.contiguous(), w, y)
    assert all(torch.equal(o3[n], o4[n]) for n in o3)


@pytest.mark.parametrize("T", [40, 300])
def test_tokens_without_a_gradient(T):
    """Ignored tokens, whose rows hold NaN, change nothing; with none left dw is zero."""
    rng, x, w, y = _inputs(T, 64, 500, T)
    y = y.clamp(0, 499)
    off = torch.from_numpy(rng.random(T) < 0.4).cuda()
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    o = _forward(x, w, y)
    kept = ~off
    ok = {n: o[n][kept].contiguous() for n in o}
    wx, ww = _backward(x[kept].contiguous(), w, y[kept].contiguous(), ok, (g[kept].contiguous(), None, None))
    bad, yy = x.clone(), y.clone()
    bad[off] = NAN
    yy[off] = -100
    o["lse"][off] = NAN
    dx, dw = _backward(bad, w, yy, o, (g, None, None))
    torch.cuda.synchronize()
    assert not dx[off].any()
    # (fewer rows may be tiled and split another way: the same up to the roundings)
    assert float((dx[kept].double() - wx.double()).norm() / wx.double().norm()) <= 2.0 ** -7
    assert float((dw.double() - ww.double()).norm() / ww.double().norm()) <= 2.0 ** -7
    dx, dw = _backward(bad, w, torch.full_like(yy, -1), o, (g, None, None))
    assert not dx.any() and not dw.any()


def test_rows_that_are_lost():
    """A NaN or infinity in a row of x: that row's results are NaN, the others' what they were."""
    rng, x, w, y = _inputs(50, 32, 400, 12)
    y = y.clamp(0, 399)
    o = _forward(x, w, y)
    bad = x.clone()
    bad[7, 3], bad[20, 0] = NAN, float("inf")
    o2 = _forward(bad, w, y)
    lost = torch.zeros(50, dtype=torch.bool, device="cuda")
    lost[[7, 20]] = True
    for n in o:
        assert o2[n][lost].isnan().all() and torch.equal(o2[n][~lost], o[n][~lost]), n
    g = torch.ones(50, device="cuda")
    dx, dw = _backward(bad, w, y, o2, (g, None, None))
    assert dx[lost].isnan().all() and not dx[~lost].isnan().any() and dw.isnan().all()
    # logits of -inf: no probability; of nothing else: no lse
    big = torch.full((2, 32), 3e38, dtype=BF, device="cuda")
    big[1] = 0
    wneg = w.clone()
    wneg[5] = -1.0
    o3 = _forward(big[:1].contiguous(), torch.full_like(w, -1.0), y[:1].contiguous())
    assert o3["lse"].item() == -math.inf and o3["entropy"].item() == 0 and o3["logp"].item() == -math.inf
    dx, dw = _backward(big[:1].contiguous(), torch.full_like(w, -1.0), y[:1].contiguous(), o3, (g[:1].contiguous(), None, None))
    assert not dx.any() and not dw.any()


def test_large_logits():
    """Logits far from zero, and far apart: the largest takes all."""
    x = torch.full((3, 8), 2.0 ** 40, dtype=BF, device="cuda")
    w = torch.zeros((300, 8), dtype=BF, device="cuda")
    w[270] = 2.0 ** 20
    y = torch.tensor([270, 1, -1], device="cuda")
    o = _forward(x, w, y)
    z = 8 * 2.0 ** 60
    assert o["lse"].tolist() == [z] * 3 and o["logp"].tolist() == [0.0, -z, 0.0] and o["entropy"].tolist() == [0.0] * 3
    dx, dw = _backward(x, w, y, o, (torch.ones(3, device="cuda"), None, None))
    assert not dx[0].any() and dx[1].tolist() == [-2.0 ** 20] * 8 and dw[1].tolist() == [2.0 ** 40] * 8


def test_no_tokens():
    w = torch.ones((5, 16), dtype=BF, device="cuda")
    x, y, f = torch.empty((0, 16), dtype=BF, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    for dtype in (BF, F):
        dw = torch.full((5, 16), NAN, dtype=dtype, device="cuda")
        nsp.nsp_linear_logp_fwd(x, w, y, f, f, f)
        nsp.nsp_linear_logp_bwd(x, w, y, f, None, dw, None, g_logp=f)
        torch.cuda.synchronize()
        assert not dw.any()


@pytest.mark.parametrize("T,dim,V", [(24, 512, 9001), (300, 264, 2100)])
def test_repeats_streams_and_graphs(T, dim, V):
    rng, x, w, y = _inputs(T, dim, V, 21)
    g = [torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda() for _ in range(3)]
    o = _forward(x, w, y)
    dx, dw = _backward(x, w, y, o, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                # (its buffers are filled on that stream too)
        o2 = _forward(x, w, y)
        dx2, dw2 = _backward(x, w, y, o2, g)
    side.synchronize()
    assert all(torch.equal(o[n], o2[n]) for n in o) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    # captured, replayed on changed inputs with eager calls between
    xs = x.clone()
    ws1, ws2 = _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V)), _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V))
    og = {n: torch.empty(T, device="cuda") for n in o}
    dxg, dwg = torch.empty_like(x), torch.empty_like(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nsp.nsp_linear_logp_fwd(xs, w, y, og["logp"], og["lse"], og["entropy"], ws1)
        nsp.nsp_linear_logp_bwd(xs, w, y, og["lse"], dxg, dwg, ws2, g_logp=g[0], g_lse=g[1], g_entropy=g[2], entropy=og["entropy"])
    for k in range(3):
        xs.copy_(x * (1 + 0.25 * k))
        graph.replay()
        torch.cuda.synchronize()
        oe = _forward(xs, w, y)
        dxe, dwe = _backward(xs, w, y, oe, g)
        assert all(torch.equal(og[n], oe[n]) for n in o) and torch.equal(dxg, dxe) and torch.equal(dwg, dwe)
