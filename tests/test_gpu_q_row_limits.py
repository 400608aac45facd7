"""The row operators past the sizes that one launch or 32 bits hold: more rows
than workgroups (each takes several), rows whose elements lie past 2^31, values
at the ends of float32.  Results are compared with the same rows in a small
call (bit for bit: a row's result depends on that row alone) or with float64."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _e(*shape, dtype=F):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _randn(*shape, dtype=F, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _some(T):
    """Rows at the ends, where a workgroup's second turn begins, and between."""
    r = [0, 1, 63, 64, T // 3, T - 2, T - 1] + [k for k in ((1 << 20) * 4, (1 << 22), (1 << 22) + 1) if k < T]
    return torch.tensor(sorted(set(r)), device="cuda")


def test_more_tokens_than_waves():
    T = (1 << 22) + 5000
    x, pos = _randn(T, 1, 8, dtype=BF), torch.arange(T, device="cuda") % 100003
    freqs = torch.from_numpy(nsp.nsp_rotary_frequencies(8, 1e4)[0]).cuda()
    y, s = _e(T, 1, 8, dtype=BF), _some(T)
    nsp.nsp_rotary_fwd(pos, freqs, x, y)
    z = _e(len(s), 1, 8, dtype=BF)
    nsp.nsp_rotary_fwd(pos[s], freqs, x[s], z)
    torch.cuda.synchronize()
    assert torch.equal(y[s], z)
    back = _e(T, 1, 8, dtype=BF)
    nsp.nsp_rotary_bwd(pos, freqs, y, back)                    # every row turned back: two roundings of bf16
    torch.cuda.synchronize()
    assert float((back.float() - x.float()).abs().max()) <= 2.0 ** -7 * float(x.float().abs().max()) * 2 ** 0.5


def test_more_rows_than_workgroups():
    T = (1 << 22) + 5000
    z, y = _randn(T, 12, dtype=BF, seed=2), torch.arange(T, device="cuda") % 12
    s = _some(T)

    def calls(z, y):
        n = z.shape[0]
        o = dict(logp=_e(n), lse=_e(n), ent=_e(n), tl=_e(n, 3), ti=_e(n, 3, dtype=torch.int64), dz=_e(n, 12, dtype=BF))
        nsp.nsp_token_logp_fwd(z, y, o["logp"], o["lse"], o["ent"], o["tl"], o["ti"])
        nsp.nsp_token_logp_bwd(z, y, o["lse"], o["dz"], g_logp=o["logp"], g_entropy=o["logp"], entropy=o["ent"])
        return o

    big, small = calls(z, y), calls(z[s], y[s])
    torch.cuda.synchronize()
    assert all(torch.equal(big[n][s], small[n]) for n in big)
    want = R.token_logp(as64(z[s]), y[s].cpu().numpy(), 1.0, 3)
    assert np.array_equal(small["ti"].cpu().numpy(), want["top_index"])
    # every row's gradient of logp alone sums to nothing: p sums to one
    dz = _e(T, 12, dtype=BF)
    nsp.nsp_token_logp_bwd(z, y, big["lse"], dz, g_logp=torch.ones(T, device="cuda"))
    assert float(dz.float().sum(1).abs().max()) <= 12 * 2.0 ** -9 + 2.0 ** -9     # (12 roundings of numbers below 1)


def test_many_rows_of_a_norm():
    T = 3000001
    x, g, w = _randn(T, 24, dtype=BF, seed=3), _randn(T, 24, dtype=BF, seed=4), _randn(24, dtype=BF, seed=5)
    y, mean, rstd, dx = _e(T, 24, dtype=BF), _e(T), _e(T), _e(T, 24, dtype=BF)
    dw, db = _e(24, dtype=F), _e(24, dtype=F)
    wf = w.float()
    nsp.nsp_norm_fwd(x, wf, None, y, mean, rstd)
    nsp.nsp_norm_bwd(x, wf, g, mean, rstd, dx, dw, db, _e(nsp.nsp_norm_bwd_workspace(T, 1, 24), dtype=torch.uint8))
    s = _some(T)
    y2, dx2 = _e(len(s), 24, dtype=BF), _e(len(s), 24, dtype=BF)
    nsp.nsp_norm_fwd(x[s], wf, None, y2)
    nsp.nsp_norm_bwd(x[s], wf, g[s], mean[s], rstd[s], dx2, None, None, None)
    torch.cuda.synchronize()
    assert torch.equal(y[s], y2) and torch.equal(dx[s], dx2)
    x64, g64 = x.double(), g.double()
    t = g64 * (x64 - mean.double()[:, None]) * rstd.double()[:, None]
    u = (128 + T / 256) * 2.0 ** -24                           # (the sums' bound: rows of a workgroup, its groups, strands)
    assert bool(((dw - t.sum(0)).abs() <= u * t.abs().sum(0)).all()) and bool(((db - g64.sum(0)).abs() <= u * g64.abs().sum(0)).all())


def test_rows_past_32_bits():
    """Three tokens 2^30 + 8 elements apart."""
    step, D = (1 << 30) + 8, 128
    buf = torch.zeros(2 * step + 2 * D, dtype=BF, device="cuda")
    view = torch.as_strided(buf, (3, 2, D), (step, D, 1))
    x = _randn(3, 2, D, dtype=BF, seed=6)
    view.copy_(x)
    pos, freqs = torch.tensor([5, 6, 7], device="cuda"), torch.from_numpy(nsp.nsp_rotary_frequencies(D, 1e4)[0]).cuda()
    a, b = _e(3, 2, D, dtype=BF), _e(3, 2, D, dtype=BF)
    nsp.nsp_rotary_fwd(pos, freqs, x, a)
    nsp.nsp_rotary_fwd(pos, freqs, view, b)
    assert torch.equal(a, b)
    mean, rstd, w = _e(6), _e(6), _randn(D, seed=7)
    nsp.nsp_norm_fwd(x, w, None, a, mean, rstd)
    nsp.nsp_norm_fwd(view, w, None, b, mean, rstd)
    assert torch.equal(a, b)
    dw, dw2 = _e(D), _e(D)
    nsp.nsp_norm_bwd(x, w, a, mean, rstd, b, dw, None, None)
    nsp.nsp_norm_bwd(view, w, a, mean, rstd, view, dw2, None, None)          # in place, far apart
    torch.cuda.synchronize()
    assert torch.equal(view, b) and torch.equal(dw, dw2)
    del buf, view
    torch.cuda.empty_cache()


def test_ends_of_float32():
    """Logits as large as 1e37 and scales from 2^-20 to 2^20: no overflow where
    the results are finite."""
    for scale in (2.0 ** -20, 1.0, 2.0 ** 20):
        z = _randn(4, 5000, seed=8) / scale
        z[1, 7] = 30.0 / scale
        y, o = torch.tensor([0, 7, 4999, 3], device="cuda"), [_e(4) for _ in range(3)]
        ws = _e(nsp.nsp_token_logp_workspace(4, 5000), dtype=torch.uint8)
        nsp.nsp_token_logp_fwd(z, y, *o, workspace=ws, scale=scale)
        torch.cuda.synchronize()
        want = R.token_logp(as64(z), y.cpu().numpy(), scale)
        for t, n in zip(o, ("logp", "lse", "entropy")):
            assert np.abs(as64(t) - want[n]).max() <= 2.0 ** -18 * (1 + np.abs(want[n]).max()), (scale, n)
    z = torch.full((2, 3000), -1e37, device="cuda")
    z[0, 10] = 1e37
    o = [_e(2) for _ in range(3)]
    ws = _e(nsp.nsp_token_logp_workspace(2, 3000), dtype=torch.uint8)
    nsp.nsp_token_logp_fwd(z, torch.tensor([10, 0], device="cuda"), *o, workspace=ws)
    torch.cuda.synchronize()
    logp, lse, ent = (as64(t) for t in o)
    assert logp[0] == 0 and ent[0] == 0 and abs(lse[0] / 1e37 - 1) <= 2.0 ** -22
    # a row of equal logits: ln V each, however large they are
    assert abs(logp[1] + np.log(3000)) <= 2.0 ** -18 * 8 and abs(ent[1] - np.log(3000)) <= 2.0 ** -18 * 8
    # neighbouring floats there are as far apart as a softmax can tell: one of them takes it all
    big = torch.tensor([[1e30] * 3, [-1e30] * 3, [3e9] * 3], device="cuda")
    big[:, 1] = torch.nextafter(big[:, 1], torch.tensor(float("inf"), device="cuda"))
    o, tl, ti = [_e(3) for _ in range(3)], _e(3, 2), _e(3, 2, dtype=torch.int64)
    nsp.nsp_token_logp_fwd(big, torch.ones(3, dtype=torch.int64, device="cuda"), *o, tl, ti)
    torch.cuda.synchronize()
    assert bool((o[0] == 0).all()) and bool((o[2] == 0).all()) and ti.cpu().tolist() == [[1, 0]] * 3 and bool((tl[:, 0] == 0).all())
    # and whatever lse is rounded to, a probability is at most 1
    dz = _e(3, 3)
    nsp.nsp_token_logp_bwd(big, torch.ones(3, dtype=torch.int64, device="cuda"), o[1], dz, g_logp=torch.ones(3, device="cuda"))
    torch.cuda.synchronize()
    assert bool(dz.isfinite().all()) and float(dz.abs().max()) <= 1.0
