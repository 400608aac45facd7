"""Gradients from hidden rows in float32, of any number of tokens: the gradient of the
logits goes into the products as two bf16 numbers, which keep it to 2^-16 of itself
(twice half a step of bf16).  p's own errors, 2^-21 (1 + |z| + |lse|) and the logits', are
below that at these sizes, and the products' additions grow as the square root of
their number (2^-24 (V or T)^(1/2) of the result and less).  The sizes' sum of dx and dw is
at most 4 times the result (a target's against the others'): relative 2-norms within
4 (2^-16 + 2^-16) = 2^-13, where one rounding to bf16 leaves some 2^-9.  All weights
alike, so that their errors are too."""
import math

import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import draw

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _ws(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def _reference(x, w, y, g, ignored=None):
    """dx, dw in float64, some tokens at a time."""
    x, w = x.double(), w.double()
    dx, dw = torch.empty_like(x), torch.zeros_like(w)
    wt = w.t().contiguous()
    for a in range(0, len(x), 4096):
        xx, yy = x[a:a + 4096], y[a:a + 4096, None]
        gg = torch.where(yy >= 0, g[a:a + 4096, None].double(), 0.0)
        z = xx @ wt
        da = -gg * (z - torch.logsumexp(z, 1, keepdim=True)).exp()
        da.scatter_add_(1, yy.clamp_min(0), gg)
        dx[a:a + 4096] = da @ w
        dw += da.t().contiguous() @ xx
    return dx, dw


def _check(T, dim, V, share=0.0):
    rng = np.random.default_rng(T + dim + V)
    x, w = draw(rng, (T, dim), BF), draw(rng, (V, dim), BF, 2.0 / math.sqrt(dim))
    y = torch.from_numpy(np.where(rng.random(T) < share, -1, rng.integers(0, V, T))).cuda()
    o = [torch.empty(T, device="cuda") for _ in range(3)]
    nsp.nsp_linear_logp_fwd(x, w, y, *o, _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V)))
    g = torch.full((T,), -1.0 / 3.0, device="cuda")
    ws = _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V))

    def run(dx=True, dw=True):
        out = [torch.full(t.shape, float("nan"), device="cuda") if some else None for t, some in ((x, dx), (w, dw))]
        nsp.nsp_linear_logp_bwd(x, w, y, o[1], *out, ws, g_logp=g)
        return out

    dx, dw = run()
    rdx, rdw = _reference(x, w, y, g)
    off = [float((a.double() - b).norm() / b.norm()) for a, b in ((dx, rdx), (dw, rdw))]
    print(f"[rows] dx {off[0]:.2e}, dw {off[1]:.2e}", flush=True)
    assert max(off) <= 2.0 ** -13, off
    ws.fill_(255)
    again = run()
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    ws.fill_(255)
    assert torch.equal(run(dw=False)[0], dx) or float((run(dw=False)[0].double() - rdx).norm() / rdx.norm()) <= 2.0 ** -13
    ws.fill_(255)
    assert float((run(dx=False)[1].double() - rdw).norm() / rdw.norm()) <= 2.0 ** -13


@pytest.mark.parametrize("T,dim,V", [(127, 136, 1000), (128, 136, 1000), (129, 136, 1000), (130, 64, 31), (257, 64, 1025), (300, 1000, 777), (520, 72, 2100),
                                     (777, 1000, 5021), (3000, 64, 300), (300, 2048, 1000), (513, 1544, 257), (2049, 520, 4097)])
def test_both_sides_of_128_tokens_and_more(T, dim, V):
    _check(T, dim, V)


@pytest.mark.parametrize("T,dim,V", [(900, 264, 3000), (4100, 136, 2100)])
def test_with_ignored_tokens(T, dim, V):
    _check(T, dim, V, 0.4)


@pytest.mark.parametrize("T,dim,V", [(9001, 24, 30011), (20011, 24, 30011), (70001, 16, 5003)])
def test_several_pieces(T, dim, V):
    _check(T, dim, V)


def test_captured():
    """A captured call on changed rows, with eager calls of both types between the replays."""
    T, dim, V = 300, 264, 2100
    rng = np.random.default_rng(9)
    x, w, y = draw(rng, (T, dim), BF), draw(rng, (V, dim), BF, 0.1), torch.from_numpy(rng.integers(0, V, T)).cuda()
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    ws = [_ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V)) for _ in range(2)]
    wf = _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V))
    xs, lse = x.clone(), torch.empty(T, device="cuda")

    def step(dtype, ws, dx, dw):
        nsp.nsp_linear_logp_fwd(xs, w, None, None, lse, None, wf)
        nsp.nsp_linear_logp_bwd(xs, w, y, lse, dx, dw, ws, g_logp=g)

    out = {t: [torch.empty(v.shape, dtype=t, device="cuda") for v in (x, w)] for t in (BF, F)}
    got = [torch.empty(v.shape, device="cuda") for v in (x, w)]
    step(F, ws[0], *got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(F, ws[0], *got)
    for k in range(3):
        xs.copy_(x * (1 + 0.25 * k))
        graph.replay()
        torch.cuda.synchronize()
        step(F, ws[1], *out[F])
        step(BF, ws[1], *out[BF])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out[F]))
        assert all(float((a.double() - b.double()).norm() / b.double().norm()) <= 2.0 ** -7 for a, b in zip(out[BF], got))
