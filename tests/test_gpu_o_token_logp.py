"""Token log probabilities against the float64 definition.

Tolerances.  A lane adds at most S = vocab / 256 + 24 terms of a row one after
another (a part of a row: fewer), each term's exponent within 2^-23 (|z| + |m|
+ |d|) and the reference moves; so
    lse      (S + 24) 2^-24 + 2^-21 (max|z| + ln V + 12)
    entropy  (S + 64) 2^-22 (ln V + 12)    (u / s and ln s cancel at most to
             terms of 16 powers of two and ln V)
    logp     that of lse and 2^-23 (|z| + |lse|)
    dz       half a step, and 2^-21 (1 + |z| + |lse|) of p times the sizes of
             its coefficients, and 2^-23 of the target's own."""
import math

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import F32, as64, half_step, strided, untouched, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _logits(rng, T, V, dtype, masked=0.0, spread=3.0):
    z = (rng.standard_normal((T, V)) * spread).astype(np.float32)
    if masked:
        z[rng.random((T, V)) < masked] = -np.inf
    return torch.from_numpy(z).to(dtype).cuda()


def _forward(z, y, top=0, scale=1.0, stream=None):
    T, V = z.shape
    f32 = dict(dtype=F, device="cuda")
    o = {n: torch.full((T,), -7.0, **f32) for n in ("logp", "lse", "entropy")}
    o["top_logp"] = torch.full((T, top), -7.0, **f32)
    o["top_index"] = torch.full((T, top), -7, dtype=torch.int64, device="cuda")
    ws = torch.full((nsp.nsp_token_logp_workspace(T, V, top),), 255, dtype=torch.uint8, device="cuda")
    nsp.nsp_token_logp_fwd(z, y, o["logp"], o["lse"], o["entropy"], o["top_logp"] if top else None, o["top_index"] if top else None, ws,
                           scale=scale, stream=stream)
    return o


def _check_fwd(z, y, o, scale, top):
    z64, V = as64(z), z.shape[1]
    want = R.token_logp(z64, y.cpu().numpy(), scale, top)
    S = V / 256 + 24
    big = np.where(np.isfinite(z64), np.abs(z64), 0.0).max(1) * scale
    tl = (S + 24) * F32 + 2.0 ** -21 * (big + math.log(V) + 12)
    within("lse", as64(o["lse"]), want["lse"], tl)
    within("entropy", as64(o["entropy"]), want["entropy"], (S + 64) * 2.0 ** -22 * (math.log(V) + 12))
    lse = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0.0)
    tp = tl + 2.0 ** -23 * (big + lse)
    within("logp", as64(o["logp"]), want["logp"], tp)
    if top:
        assert np.array_equal(o["top_index"].cpu().numpy(), want["top_index"])
        within("top_logp", as64(o["top_logp"]), want["top_logp"], tp[:, None])


def _check_bwd(z, y, lse, ent, g, dz, scale):
    z64, l64, e64 = as64(z), as64(lse), as64(ent)
    gl, gs, ge = (None if t is None else as64(t) for t in g)
    t = None if y is None else y.cpu().numpy()
    want = R.token_logp_backward(z64, t, l64, e64, gl, gs, ge, scale)
    size = sum(0.0 if v is None else np.abs(v) for v in (gl, gs))
    zs = z64 * scale
    with np.errstate(invalid="ignore"):
        d = zs - l64[:, None]
        p = np.exp(d)
        a = np.where(np.isfinite(zs), np.abs(zs), 0.0) + np.where(np.isfinite(l64), np.abs(l64), 0.0)[:, None]
        live = np.isfinite(d)
        c = np.zeros_like(p) + (size[:, None] if np.ndim(size) else size)
        if ge is not None:
            c += np.abs(ge)[:, None] * (np.where(live, np.abs(d), 0.0) + np.abs(e64)[:, None] + 1)
        tol = half_step(dz.dtype) * np.abs(want) + 2.0 ** -21 * (1 + a) * np.where(live, p, 0.0) * scale * c
    if gl is not None:
        for r, v in enumerate(t):
            if 0 <= v < z.shape[1]:
                tol[r, v] += 2.0 ** -23 * abs(gl[r]) * scale
    within("dlogits", as64(dz), want, tol + np.where(want == 0, 0.0, 2.0 ** -120))     # (what is below 2^-126 may be flushed)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,V,top", [
    (1, 1, 1), (1, 2, 5), (3, 7, 0), (2, 64, 64), (5, 65, 3), (1, 2047, 8), (1, 2049, 8), (8, 4099, 1), (2, 32000, 20), (1, 131072, 8),
    (1, 160001, 64), (300, 1000, 5), (2049, 515, 2), (1030, 5000, 0), (40, 50021, 7)])
def test_against_the_definition(T, V, top, dtype):
    rng = np.random.default_rng(T + V)
    z = _logits(rng, T, V, dtype)
    y = torch.from_numpy(rng.integers(-1, V + 1, T)).cuda()                # ignored ones on both sides
    for scale in (1.0, 0.6):
        _check_fwd(z, y, _forward(z, y, top, scale), scale, top)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 7), (5, 2049), (2, 50021), (700, 1000), (4, 131072)])
def test_gradient(T, V, dtype):
    rng = np.random.default_rng(T * V)
    z = _logits(rng, T, V, dtype)
    y = torch.from_numpy(rng.integers(-1, V + 1, T)).cuda()
    o = _forward(z, y, 0, 0.8)
    g = [torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda() for _ in range(3)]
    for use in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1), (0, 0, 0)):
        gl, gs, ge = (t if u else None for t, u in zip(g, use))
        dz = torch.full_like(z, float("nan"))
        nsp.nsp_token_logp_bwd(z, y if use[0] else None, o["lse"], dz, g_logp=gl, g_entropy=ge, entropy=o["entropy"] if use[2] else None,
                               g_lse=gs, scale=0.8)
        torch.cuda.synchronize()
        _check_bwd(z, y if use[0] else None, o["lse"], o["entropy"], (gl, gs, ge), dz, 0.8)


def test_gradient_against_differences():
    """Central differences of the forward itself, in float32: steps of 2^-5,
    whose third-order term is below 2^-12 of a coefficient of at most 4, and
    whose values round at 2^-21 of their size."""
    rng = np.random.default_rng(5)
    z, y = _logits(rng, 4, 37, F, spread=1.0), torch.tensor([3, 36, 0, -1], device="cuda")
    w = [1.0, 0.5, -0.7]
    o = _forward(z, y)
    g = [torch.full((4,), v, device="cuda") for v in w]
    dz = torch.empty_like(z)
    nsp.nsp_token_logp_bwd(z, y, o["lse"], dz, g_logp=g[0], g_entropy=g[2], entropy=o["entropy"], g_lse=g[1])

    def f(x):
        r = _forward(x, y)
        return w[0] * as64(r["logp"]) + w[1] * as64(r["lse"]) + w[2] * as64(r["entropy"])
    h = 2.0 ** -5
    for v in range(37):
        up, down = z.clone(), z.clone()
        up[:, v] += h
        down[:, v] -= h
        d = (f(up) - f(down)) / (as64(up)[:, v] - as64(down)[:, v])
        assert np.abs(d - as64(dz)[:, v]).max() <= 2.0 ** -10 + 2.0 ** -19 * 8 / h


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [9, 4099, 70000])
def test_masked_vocabularies_and_odd_rows(V, dtype):
    rng = np.random.default_rng(V)
    z = _logits(rng, 12, V, dtype, masked=0.5)
    low = torch.finfo(dtype).min
    z[0] = -INF                                     # nothing left
    z[1] = -INF
    z[1, V - 1] = 2.5                               # one left, the last
    z[2] = low                                      # nothing left, masked by the type's lowest value
    z[3, :] = low
    z[3, V // 2] = 0.0                              # masked by the lowest value
    z[4] = 0.0                                      # all alike
    z[5] = -0.0
    z[5, ::2] = 0.0                                 # both zeros are one value
    z[6, 0] = float("nan")
    z[7, V // 3] = INF
    z[8, :] = torch.arange(V, device="cuda").to(dtype)          # ever larger (in bf16 with ties)
    z[9, :] = -torch.arange(V, device="cuda").to(dtype)
    z[10, : V // 2] = -INF                          # the first half masked
    y = torch.tensor([0, V - 1, 1, V // 2, 2, 3, 4, 5, V - 1, 0, V - 1, -1], device="cuda")
    for top in (0, 1, 6, 64):
        o = _forward(z, y, top)
        torch.cuda.synchronize()
        _check_fwd(z, y, o, 1.0, top)
    g = [torch.from_numpy(rng.standard_normal(12).astype(np.float32)).cuda() for _ in range(3)]
    rows = [r for r in range(12) if r not in (6, 7)]
    for gl, gs, ge in ((g[0], None, None), g):
        dz = torch.full_like(z, float("nan"))
        nsp.nsp_token_logp_bwd(z, y, o["lse"], dz, g_logp=gl, g_entropy=ge, entropy=o["entropy"] if ge is not None else None, g_lse=gs)
        torch.cuda.synchronize()
        assert not dz[0].any() and not dz[2].any() and bool(dz[6].isnan().any()) and bool(dz[7].isnan().any())
        sub = torch.tensor(rows, device="cuda")
        _check_bwd(z[sub], y[sub], o["lse"][sub], o["entropy"][sub], tuple(None if t is None else t[sub] for t in (gl, gs, ge)), dz[sub], 1.0)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V,pad", [(1000, 1), (4096, 8), (5003, 13)])
def test_padded_rows_and_in_place(V, pad, dtype):
    """Rows further apart than the vocabulary is wide, at any alignment: what
    lies between is neither read nor written."""
    rng = np.random.default_rng(V + pad)
    z = _logits(rng, 17, V, dtype)
    y = torch.from_numpy(rng.integers(0, V, 17)).cuda()
    zv, zb, zm = strided(z, 3, pad)
    o, p = _forward(z, y, 4), _forward(zv, y, 4)
    torch.cuda.synchronize()
    assert all(torch.equal(o[n], p[n]) for n in o)
    gl = torch.ones(17, device="cuda")
    dz = torch.empty_like(z)
    nsp.nsp_token_logp_bwd(z, y, o["lse"], dz, g_logp=gl)
    dv, db, dm = strided(torch.zeros_like(z), 1, pad + 2)
    nsp.nsp_token_logp_bwd(zv, y, o["lse"], dv, g_logp=gl)
    torch.cuda.synchronize()
    assert torch.equal(dv, dz) and untouched(db, dm) and torch.equal(zv, z)
    nsp.nsp_token_logp_bwd(zv, y, o["lse"], zv, g_logp=gl)
    torch.cuda.synchronize()
    assert torch.equal(zv, dz) and untouched(zb, zm)


def test_broadcast_rows_and_no_rows():
    rng = np.random.default_rng(1)
    z = _logits(rng, 1, 3001, BF).expand(5, 3001)
    y = torch.arange(5, device="cuda")
    _check_fwd(z, y, _forward(z, y, 3), 1.0, 3)
    e = torch.empty(0, 50, dtype=BF, device="cuda")
    f = torch.empty(0, dtype=F, device="cuda")
    nsp.nsp_token_logp_fwd(e, torch.empty(0, dtype=torch.int64, device="cuda"), f, f)
    nsp.nsp_token_logp_bwd(e, None, f, e)


def test_outputs_left_out():
    rng = np.random.default_rng(2)
    z = _logits(rng, 6, 9000, F)
    y = torch.arange(6, device="cuda")
    o = _forward(z, y)
    lse = torch.empty(6, device="cuda")
    ws = torch.empty(nsp.nsp_token_logp_workspace(6, 9000), dtype=torch.uint8, device="cuda")
    nsp.nsp_token_logp_fwd(z, None, None, lse, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(lse, o["lse"])


def test_offsets_past_32_bits():
    """Rows whose elements lie past 2^31 (one tensor of 2^32 bytes and more)."""
    T, V = 9, (1 << 28) + 3
    z = torch.zeros(T, V, dtype=BF, device="cuda")
    z[:, 12345] = 30.0
    z[T - 1, V - 1] = 31.0
    y = torch.full((T,), V - 1, device="cuda")
    o = _forward(z, y, 2)
    torch.cuda.synchronize()
    want = 30.0 + math.log1p((V - 1) * math.exp(-30.0))
    tol = (V / 256 / 64 + 48) * F32 * 31 + 2.0 ** -21 * 64
    lse = as64(o["lse"])
    assert np.abs(lse[:-1] - want).max() <= tol
    assert o["top_index"][0].tolist() == [12345, 0] and o["top_index"][T - 1].tolist() == [V - 1, 12345]
    assert abs(float(o["logp"][T - 1]) - (31.0 - lse[-1])) <= 2.0 ** -18
    nsp.nsp_token_logp_bwd(z, y, o["lse"], z, g_logp=torch.ones(T, device="cuda"))
    torch.cuda.synchronize()
    p = math.exp(31.0 - lse[-1])
    assert abs(float(z[T - 1, V - 1]) - (1 - p)) <= half_step(BF) * (1 - p) + 2.0 ** -15
    assert abs(float(z[0, 12345]) + math.exp(30.0 - want)) <= half_step(BF) + 2.0 ** -15
    del z
    torch.cuda.empty_cache()


def test_repeatable_on_a_side_stream_and_replayed():
    rng = np.random.default_rng(3)
    z, y = _logits(rng, 5, 40000, BF), torch.from_numpy(rng.integers(0, 40000, 5)).cuda()
    o = _forward(z, y, 8)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    p = _forward(z, y, 8, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o[n], p[n]) for n in o)
    outs, graphs = [], []
    for _ in range(2):                              # each with a workspace of its own
        q = {n: torch.zeros_like(t) for n, t in o.items()}
        q["dz"] = torch.zeros_like(z)
        ws = torch.empty(nsp.nsp_token_logp_workspace(5, 40000, 8), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nsp.nsp_token_logp_fwd(z, y, q["logp"], q["lse"], q["entropy"], q["top_logp"], q["top_index"], ws)
            nsp.nsp_token_logp_bwd(z, y, q["lse"], q["dz"], g_logp=q["logp"], g_entropy=q["lse"], entropy=q["entropy"])
        outs.append((q, ws))
        graphs.append(g)
    for _ in range(3):
        z.copy_(_logits(rng, 5, 40000, BF))
        for g in graphs:
            g.replay()
        o = _forward(z, y, 8)
        torch.cuda.synchronize()
        _check_fwd(z, y, o, 1.0, 8)
        for q, _ in outs:
            assert all(torch.equal(o[n], q[n]) for n in o)
            _check_bwd(z, y, q["lse"], q["entropy"], (q["logp"], None, q["lse"]), q["dz"], 1.0)
