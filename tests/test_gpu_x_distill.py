"""Distillation from a teacher's top alternatives against the float64 definition.

Tolerances: lse as for the token log probabilities,
    tl = (S + 24) 2^-24 + 2^-21 (max|z| + ln V + 12),  S = vocab / 256 + 24;
    q     2^-21 (2 + |t| + |c|) of itself (its exponent's product with log2(e) and
          the two sums before it)
    loss  sum of q's error times |t - c - logp| and q times (tl + 2^-22 (|z| + |lse| + |t| + |c| + 1)),
          and (top + 8) 2^-24 of the terms' sizes
    dz    half a step, 2^-21 (1 + |z| + |lse|) + 2^-21 (2 + max|t| + |c|) + (top + 8) 2^-24 of
          p S, and q's error and (top + 8) 2^-24 of its weight where an alternative lies."""
import math

import numpy as np
import pytest
import torch

from oracle import rows as R
from oracle import vocab as O
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, half_step, strided, untouched, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _inputs(T, V, K, dtype, seed, twice=True):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.standard_normal((T, V)) * 3).astype(np.float32)).to(dtype).cuda()
    index = rng.integers(-1, V + 1, (T, K))              # none on both sides, and the same ones again
    t = (rng.standard_normal((T, K)) * 2 - 3).astype(np.float32)
    t[rng.random((T, K)) < 0.1] = -INF
    return rng, z, torch.from_numpy(index).cuda(), torch.from_numpy(t).cuda()


def _forward(z, index, t, kind, scale=1.0):
    T, V = z.shape
    loss, lse = torch.full((T,), -7.0, device="cuda"), torch.full((T,), -7.0, device="cuda")
    ws = torch.full((nsp.nsp_distill_fwd_workspace(T, V),), 255, dtype=torch.uint8, device="cuda")
    nsp.nsp_distill_fwd(z, index, t, loss, lse, ws, kind=kind, scale=scale)
    return loss, lse


def _sizes(z, index, t, kind, scale):
    z64, i, t64 = as64(z), index.cpu().numpy(), as64(t)
    q, d, there = O.weights(i, t64, z.shape[1], kind == 1)
    tt = np.where(there, t64, 0.0)
    return z64, i, t64, q, d, there, np.abs(tt) + np.abs(np.where(there, tt - d, 0.0)).max(1, keepdims=True)


def _check_fwd(z, index, t, loss, lse, kind, scale):
    z64, i, t64, q, d, there, size = _sizes(z, index, t, kind, scale)
    want, want_lse = O.distill(z64, i, t64, kind == 1, scale)
    V, K = z.shape[1], index.shape[1]
    big = np.where(np.isfinite(z64), np.abs(z64), 0.0).max(1) * scale
    tl = (V / 256 + 48) * 2.0 ** -24 + 2.0 ** -21 * (big + math.log(V) + 12)
    within("lse", as64(lse), want_lse, tl)
    zk = np.take_along_axis(z64, np.clip(i, 0, V - 1), 1) * scale
    lp = np.where(there & np.isfinite(zk), zk - np.where(np.isfinite(want_lse), want_lse, 0.0)[:, None], 0.0)
    qq = np.where(there, q, 0.0)
    term = np.abs(d - lp)
    tol = (qq * 2.0 ** -21 * (2 + size) * term + qq * (tl[:, None] + 2.0 ** -22 * (big[:, None] + np.abs(lp) + big[:, None] + size + 1))
           + (K + 8) * 2.0 ** -24 * qq * term).sum(1)
    within("loss", as64(loss), want, np.where(np.isfinite(tol), tol, 0.0) + 2.0 ** -126)


def _check_bwd(z, index, t, lse, g, dz, kind, scale):
    z64, i, t64, q, d, there, size = _sizes(z, index, t, kind, scale)
    l64, g64 = as64(lse), as64(g)
    T, V = z.shape
    K = index.shape[1]
    want = O.distill_backward(z64, i, t64, l64, g64, kind == 1, scale)
    with np.errstate(invalid="ignore"):
        p = np.exp(z64 * scale - l64[:, None])
    p = np.where(np.isfinite(p), p, 0.0)
    zs = np.where(np.isfinite(z64), np.abs(z64 * scale), 0.0)
    far = np.where(np.isfinite(l64), np.abs(l64), 0.0)[:, None]
    qq = np.where(there & np.isfinite(q), q, 0.0)
    weight = 2.0 ** -21 * (2 + size.max(1, keepdims=True)) + (K + 8) * 2.0 ** -24
    tol = (2.0 ** -21 * (1 + zs + far) + weight) * p * qq.sum(1, keepdims=True)
    for r in range(T):
        np.add.at(tol[r], i[r, there[r]], (weight[r] + 2.0 ** -23) * qq[r, there[r]])
    tol = tol * np.abs(g64)[:, None] * scale * 1.01 + half_step(dz.dtype) * np.abs(want)
    within("dlogits", as64(dz), want, tol + np.where(want == 0, 0.0, 2.0 ** -120))


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 2, 3), (3, 7, 2), (5, 65, 64), (2, 2049, 65), (8, 4099, 20), (1, 131072, 256), (300, 1000, 5),
                                   (1030, 5000, 8), (40, 50021, 64)])
def test_against_the_definition(T, V, K, dtype, kind):
    rng, z, index, t = _inputs(T, V, K, dtype, T + V + K)
    for scale in (1.0, 0.6):
        loss, lse = _forward(z, index, t, kind, scale)
        _check_fwd(z, index, t, loss, lse, kind, scale)
        g = torch.from_numpy((rng.standard_normal(T) * (rng.random(T) < 0.8)).astype(np.float32)).cuda()
        dz = torch.full_like(z, NAN)
        nsp.nsp_distill_bwd(z, index, t, lse, g, dz, kind=kind, scale=scale)
        torch.cuda.synchronize()
        _check_bwd(z, index, t, lse, g, dz, kind, scale)


def test_gradient_against_differences():
    """Central differences of the forward in float32, steps of 2^-5: the third-order
    term is below step^2 / 6 of S <= 1.6, values round at 2^-20 of their size."""
    _, z, index, t = _inputs(4, 37, 6, F, 3)
    for kind in (0, 1):
        _, lse = _forward(z, index, t, kind)
        dz, h = torch.empty_like(z), 2.0 ** -5
        nsp.nsp_distill_bwd(z, index, t, lse, torch.ones(4, device="cuda"), dz, kind=kind)
        for v in range(37):
            up, down = z.clone(), z.clone()
            up[:, v] += h
            down[:, v] -= h
            d = (as64(_forward(up, index, t, kind)[0]) - as64(_forward(down, index, t, kind)[0])) / (as64(up)[:, v] - as64(down)[:, v])
            assert np.abs(d - as64(dz)[:, v]).max() <= 2.0 ** -11 + 2.0 ** -20 * 16 / h


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [9, 4099, 70000])
def test_masked_lost_and_empty_rows(V, dtype):
    rng, z, index, t = _inputs(14, V, 4, dtype, V)
    z[torch.from_numpy(rng.random((14, V)) < 0.3).cuda()] = -INF
    index.clamp_(0, V - 1)
    t.clamp_(min=-5.0)
    z[0] = -INF                                          # nothing but masked logits
    z[1] = torch.finfo(dtype).min
    z[2, V // 2] = NAN
    z[3, V // 3] = INF
    index[4] = -1                                        # no alternatives
    t[5] = -INF
    t[6, 1] = NAN
    t[7, 2] = INF
    z[8, index[8, 0]] = -INF                             # a masked alternative
    z[9, index[9]] = 1.0
    index[10] = index[10, 0]                             # one token four times
    z[10, index[10]] = 0.5
    t[11] = torch.tensor([-200.0, -1.0, -150.0, -2.0])   # weights that are zero in float32, of masked logits too
    z[11, index[11, 1]], z[11, index[11, 3]] = 2.0, 1.0
    z[12, index[12]] = 3.0
    t[12] = torch.finfo(F).min
    z[13, index[13]] = 0.0
    for kind in (0, 1):
        loss, lse = _forward(z, index, t, kind, 1.25)
        # (weights that float32 holds no number for are zeros)
        t64 = t.clone()
        t64[11][t64[11] < -100] = -INF
        _check_fwd(z, index, t64, loss, lse, kind, 1.25)
        g = torch.from_numpy(rng.standard_normal(14).astype(np.float32)).cuda()
        dz = torch.full_like(z, NAN)
        nsp.nsp_distill_bwd(z, index, t, lse, g, dz, kind=kind, scale=1.25)
        torch.cuda.synchronize()
        _check_bwd(z, index, t64, lse, g, dz, kind, 1.25)


@pytest.mark.parametrize("dtype", [BF, F])
def test_strided_rows_and_in_place(dtype):
    rng, z, index, t = _inputs(30, 4099, 12, dtype, 8)
    g = torch.from_numpy(rng.standard_normal(30).astype(np.float32)).cuda()
    loss, lse = _forward(z, index, t, 1)
    want = torch.empty_like(z)
    nsp.nsp_distill_bwd(z, index, t, lse, g, want, kind=1)
    zs, buf, out = strided(z, 3, 7)
    l2, s2 = _forward(zs, index, t, 1)
    # (the vectors of another alignment are the same; so are their sums)
    assert torch.equal(loss, l2) and torch.equal(lse, s2)
    dz, bd, outd = strided(torch.zeros_like(z), 5, 2)
    nsp.nsp_distill_bwd(zs, index, t, lse, g, dz, kind=1)
    nsp.nsp_distill_bwd(zs, index, t, lse, g, zs, kind=1)          # in place
    torch.cuda.synchronize()
    assert torch.equal(dz, want) and torch.equal(zs, want) and untouched(bd, outd) and untouched(buf, out)


def test_with_a_teacher_of_this_library():
    """The alternatives of nsp_token_logp_fwd of the teacher's logits, fewer than asked for in places."""
    rng = np.random.default_rng(4)
    T, V, K = 20, 3000, 16
    teacher = torch.from_numpy((rng.standard_normal((T, V)) * 3).astype(np.float32)).cuda()
    teacher[3, 5:] = -INF
    f = {n: torch.empty(T, device="cuda") for n in ("lse", "loss", "s_lse")}
    top, at = torch.empty((T, K), device="cuda"), torch.empty((T, K), dtype=torch.int64, device="cuda")
    nsp.nsp_token_logp_fwd(teacher, None, None, f["lse"], None, top, at,
                           torch.empty(nsp.nsp_token_logp_workspace(T, V, K), dtype=torch.uint8, device="cuda"))
    assert (at[3, 5:] == -1).all()
    student = teacher.clone()
    loss, lse = _forward(student, at, top, nsp.NSP_DISTILL_GIVEN)
    # the teacher itself: no divergence but the roundings of its lse
    assert float(loss.abs().max()) <= 2.0 ** -18
    _check_fwd(student, at, top, loss, lse, 0, 1.0)


@pytest.mark.parametrize("T,V", [(8, 131072), (600, 3001)])
def test_repeats_streams_and_graphs(T, V):
    rng, z, index, t = _inputs(T, V, 20, BF, 2)
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    zs, loss, lse, dz = z.clone(), torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(z)
    ws = torch.empty(nsp.nsp_distill_fwd_workspace(T, V), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nsp.nsp_distill_fwd(zs, index, t, loss, lse, ws)
        nsp.nsp_distill_bwd(zs, index, t, lse, g, dz)
    for k in range(3):
        zs.copy_(z * (1 + 0.5 * k))
        graph.replay()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):            # (its buffers are filled on that stream too)
            l2, s2 = _forward(zs, index, t, 0)
        side.synchronize()
        d2 = torch.empty_like(z)
        nsp.nsp_distill_bwd(zs, index, t, s2, g, d2)
        assert torch.equal(loss, l2) and torch.equal(lse, s2) and torch.equal(dz, d2)


def test_no_tokens():
    z, i, f = torch.empty((0, 9), device="cuda"), torch.empty((0, 2), dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    nsp.nsp_distill_fwd(z, i, torch.empty((0, 2), device="cuda"), f, f)
    nsp.nsp_distill_bwd(z, i, torch.empty((0, 2), device="cuda"), f, f, z)
