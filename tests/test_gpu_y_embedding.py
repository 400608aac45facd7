"""The embedding and its gradient against the float64 definition.

Tolerances: forward, the product's rounding (2^-24) and half a step of the type.
Gradient: with n rows of an id, an addition for each in float32 and the scale's
product, (n + 8) 2^-24 of the sum of the rows' sizes, and half a step of the type."""
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


def _ids(rng, T, V, much=True):
    """Ids out of the vocabulary on both sides among them; one id of many tokens."""
    ids = rng.integers(-2, V + 2, T)
    if much:
        ids[rng.random(T) < 0.4] = V // 2
    return torch.from_numpy(ids).cuda()


def _bwd(ids, dy, V, dtype, scale=1.0, dw=None):
    T, dim = dy.shape
    dw = torch.full((V, dim), NAN, dtype=dtype, device="cuda") if dw is None else dw
    ws = torch.full((nsp.nsp_embedding_bwd_workspace(T, dim, V),), 255, dtype=torch.uint8, device="cuda")
    nsp.nsp_embedding_bwd(ids, dy, dw, ws, scale=scale)
    return dw


def _check_bwd(ids, dy, V, dw, scale):
    i, d64 = ids.cpu().numpy(), as64(dy)
    there = (i >= 0) & (i < V)
    size, n = np.zeros((V, dy.shape[1])), np.bincount(i[there], minlength=V)
    np.add.at(size, i[there], np.abs(d64[there]))
    want = np.zeros_like(size)
    np.add.at(want, i[there], d64[there])
    want *= scale
    tol = abs(scale) * (n[:, None] + 8) * 2.0 ** -24 * size + half_step(dw.dtype) * np.abs(want)
    within("dw", as64(dw), want, tol + np.where(size == 0, 0.0, 2.0 ** -126))


TYPES = [(BF, BF), (BF, F), (F, BF), (F, F)]


@pytest.mark.parametrize("wt,dt", TYPES)
@pytest.mark.parametrize("T,dim,V", [(1, 1, 1), (1, 8, 3), (3, 3, 2), (5, 7, 10), (24, 512, 1000), (100, 4099, 50), (2049, 80, 300), (70, 1111, 5)])
def test_rows(T, dim, V, wt, dt):
    rng = np.random.default_rng(T * dim + V)
    ids, w = _ids(rng, T, V), draw(rng, (V, dim), wt)
    for scale in (1.0, -33.0):
        y = torch.full((T, dim), NAN, dtype=dt, device="cuda")
        nsp.nsp_embedding_fwd(ids, w, y, scale=scale)
        want = O.embedding(ids.cpu().numpy(), as64(w), scale)
        within("y", as64(y), want, (2.0 ** -24 + half_step(dt)) * np.abs(want))


@pytest.mark.parametrize("wt,dt", TYPES)
@pytest.mark.parametrize("T,dim,V", [(1, 1, 1), (1, 8, 3), (3, 3, 2), (7, 9, 10), (8, 16, 1), (9, 16, 1), (24, 512, 1000), (100, 1111, 50), (2049, 80, 300),
                                     (4096, 33, 70000), (4097, 33, 70000), (9000, 24, 1023), (9000, 24, 1024), (20000, 8, 3), (300000, 5, 40),
                                     (16384, 16, 600), (16385, 16, 600), (17000, 12, 511), (17000, 12, 512), (30000, 9, 270000), (600001, 3, 50)])
def test_gradient(T, dim, V, wt, dt):
    rng = np.random.default_rng(T * dim + V + 1)
    ids, dy = _ids(rng, T, V), draw(rng, (T, dim), dt)
    _check_bwd(ids, dy, V, _bwd(ids, dy, V, wt, 0.7), 0.7)


@pytest.mark.parametrize("T", [32, 64, 5000, 17000])
def test_long_runs_and_their_borders(T):
    """Ids whose tokens begin and end at the borders of chunks, and one of them all."""
    rng = np.random.default_rng(T)
    dy = draw(rng, (T, 40), BF)
    for lengths in ([T], [8] * (T // 8), [1, 7, 8, 9, 15, 16, 17, 24, 32], [T // 2, T - T // 2 - 1, 1], [T - 1, 1], [1, T - 1]):
        ids = np.repeat(np.arange(len(lengths)), lengths)[:T]
        ids = np.concatenate([ids, np.full(T - len(ids), len(lengths))])
        V = int(ids.max()) + 2
        rng.shuffle(ids)
        t = torch.from_numpy(ids).cuda()
        _check_bwd(t, dy, V, _bwd(t, dy, V, F), 1.0)
    none = torch.full((T,), -1, device="cuda")
    assert not _bwd(none, dy, 7, BF).any()


def test_sums_in_order():
    """Whole numbers that leave no roundings: one token more or less would show."""
    for T, V in ((3000, 7), (50000, 11), (70000, 40000)):
        rng = np.random.default_rng(T)
        ids = torch.from_numpy(rng.integers(0, V, T)).cuda()
        dy = torch.from_numpy(rng.integers(-8, 9, (T, 12)).astype(np.float32)).cuda()
        want = np.zeros((V, 12))
        np.add.at(want, ids.cpu().numpy(), as64(dy))
        assert np.array_equal(as64(_bwd(ids, dy, V, F)), want)


def test_padding_rows_are_not_read():
    rng = np.random.default_rng(6)
    ids, dy = _ids(rng, 500, 60), draw(rng, (500, 72), BF)
    off = (ids < 0) | (ids >= 60)
    want = _bwd(ids, dy, 60, F)
    dy[off] = NAN
    assert torch.equal(_bwd(ids, dy, 60, F), want)


@pytest.mark.parametrize("wt,dt", TYPES)
def test_views_with_strides(wt, dt):
    rng = np.random.default_rng(7)
    ids, w, dy = _ids(rng, 600, 50), draw(rng, (50, 77), wt), draw(rng, (600, 77), dt)
    ws, _, _ = strided(w, 3, 5)
    y, buf, out = strided(torch.zeros((600, 77), dtype=dt, device="cuda"), 1, 2)
    y2 = torch.empty((600, 77), dtype=dt, device="cuda")
    nsp.nsp_embedding_fwd(ids, ws, y, scale=2.0)
    nsp.nsp_embedding_fwd(ids, w, y2, scale=2.0)
    dys, _, _ = strided(dy, 1, 4)
    dw, bw, ow = strided(torch.zeros((50, 77), dtype=wt, device="cuda"), 3, 1)
    _bwd(ids, dys, 50, wt, 1.0, dw)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and untouched(buf, out) and torch.equal(dw, _bwd(ids, dy, 50, wt)) and untouched(bw, ow)
    # one row of gradients for all tokens
    one = dy[:1].expand(600, 77)
    assert torch.equal(_bwd(ids, one, 50, wt), _bwd(ids, one.contiguous(), 50, wt))


def test_no_tokens():
    dw = torch.full((9, 10), NAN, dtype=BF, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    nsp.nsp_embedding_bwd(none, torch.empty((0, 10), device="cuda"), dw, None)
    nsp.nsp_embedding_fwd(none, dw, torch.empty((0, 10), device="cuda"))
    torch.cuda.synchronize()
    assert not dw.any()


@pytest.mark.parametrize("T", [24, 9000, 20000])
def test_repeats_streams_and_graphs(T):
    rng = np.random.default_rng(11)
    V = 700
    ids, dy = _ids(rng, T, V), draw(rng, (T, 264), BF)
    want = _bwd(ids, dy, V, F)
    assert torch.equal(want, _bwd(ids, dy, V, F))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                # (its buffers are filled on that stream too)
        got = _bwd(ids, dy, V, F)
    side.synchronize()
    assert torch.equal(want, got)
    i2, dw = ids.clone(), torch.empty_like(want)
    ws = torch.empty(nsp.nsp_embedding_bwd_workspace(T, 264, V), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nsp.nsp_embedding_bwd(i2, dy, dw, ws)
    for k in range(3):
        i2.copy_((ids * (k + 1)) % V)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, _bwd(i2, dy, V, F))
