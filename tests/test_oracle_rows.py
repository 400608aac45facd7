"""Pins of the row operators' oracle (oracle/rows.py): finite differences,
closed forms, invariants, and torch's float64 functions."""
import numpy as np
import pytest
import torch

from oracle import rows as R


def _diff(f, x, g, h=1e-6):
    """Central differences of <f(x), g>."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        out[i] = ((f(a) - f(b)) * g).sum() / (2 * h)
    return out


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rot", [2, 6, 8])
def test_rotary(pairs, rot):
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    pos, freqs = np.array([0, 1, 2, 1000, -3]), 1.0 / 10.0 ** (np.arange(rot // 2))
    y = R.rotary(x, pos, freqs, pairs)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., rot:], x[..., rot:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))            # lengths are kept
    # scores depend on the distance alone
    q, k = R.rotary(x, pos + 7, freqs, pairs), R.rotary(g, pos - 4, freqs, pairs)
    q2, k2 = R.rotary(x, pos + 107, freqs, pairs), R.rotary(g, pos + 96, freqs, pairs)
    assert np.allclose((q * k).sum(-1), (q2 * k2).sum(-1))
    # the quarter turn of a pair by hand
    z = np.zeros((1, 1, 8))
    z[0, 0, 0] = 1.0
    t = R.rotary(z, [1], [np.pi / 2] + [0.0] * (rot // 2 - 1), pairs, scale=3.0)
    at = 1 if pairs else rot // 2
    assert t[0, 0, at] == pytest.approx(3.0) and abs(t[0, 0, 0]) < 1e-15
    assert np.allclose(R.rotary(g, pos, freqs, pairs, 1.3, backward=True), _diff(lambda v: R.rotary(v, pos, freqs, pairs, 1.3), x, g))


@pytest.mark.parametrize("rms", [False, True])
def test_norm(rms):
    rng = np.random.default_rng(2)
    x, dy, w, b = rng.standard_normal((4, 2, 7)) + 0.5, rng.standard_normal((4, 2, 7)), rng.standard_normal(7), rng.standard_normal(7)
    y, mean, rstd = R.norm(x, w, b, 1e-3, rms)
    t = torch.from_numpy(x)
    ref = (t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-3) * torch.from_numpy(w) + torch.from_numpy(b) if rms else
           torch.nn.functional.layer_norm(t, (7,), torch.from_numpy(w), torch.from_numpy(b), 1e-3))
    assert np.allclose(y, ref.numpy())
    dx, dw, db = R.norm_backward(x, w, dy, mean, rstd, rms)
    assert np.allclose(dx, _diff(lambda v: R.norm(v, w, b, 1e-3, rms)[0], x, dy), atol=1e-7)
    assert np.allclose(dw, _diff(lambda v: R.norm(x, v, b, 1e-3, rms)[0], w, dy), atol=1e-7)
    assert np.allclose(db, _diff(lambda v: R.norm(x, w, v, 1e-3, rms)[0], b, dy), atol=1e-7)
    assert np.allclose(R.norm(x, None, None, 1e-3, rms)[0] * w + b, y)


def test_token_logp():
    rng = np.random.default_rng(3)
    z, y = rng.standard_normal((6, 9)) * 3, np.array([0, 8, 4, -1, 9, 2])
    z[5, [1, 3]] = -np.inf
    o = R.token_logp(z, y, 0.7, 4)
    lp = torch.log_softmax(torch.from_numpy(z * 0.7), 1).numpy()
    for t in range(6):
        assert o["logp"][t] == pytest.approx(lp[t, y[t]] if 0 <= y[t] < 9 else 0.0)
    live = np.where(np.isinf(lp), 0.0, lp)
    assert np.allclose(o["entropy"], -(np.exp(lp) * live).sum(1)) and np.allclose(o["lse"], torch.logsumexp(torch.from_numpy(z * 0.7), 1).numpy())
    assert np.array_equal(o["top_index"], np.argsort(-z, 1, kind="stable")[:, :4])
    g = {n: rng.standard_normal(6) for n in ("logp", "lse", "entropy")}
    z = rng.standard_normal((6, 9))
    o = R.token_logp(z, y, 0.7)
    dz = R.token_logp_backward(z, y, o["lse"], o["entropy"], g["logp"], g["lse"], g["entropy"], 0.7)
    want = sum(_diff(lambda v, n=n: R.token_logp(v, y, 0.7)[n], z, g[n]) for n in g)
    assert np.allclose(dz, want, atol=1e-7)


def test_token_logp_of_odd_rows():
    inf, nan = np.inf, np.nan
    z = np.array([[1.0, 1.0, 0.0, 1.0], [-inf] * 4, [0.0, nan, 2.0, 1.0], [0.0, inf, 1.0, -inf], [-inf, -3e38, 5.0, -inf], [-0.0, 0.0, -1.0, 0.0]])
    o = R.token_logp(z, [0, 1, 2, 3, 0, 1], 1.0, 3)
    assert o["top_index"].tolist() == [[0, 1, 3], [-1, -1, -1], [2, 3, 0], [1, 2, 0], [2, -1, -1], [0, 1, 3]]
    assert o["lse"][1] == -inf and o["entropy"][1] == 0 and o["logp"][1] == -inf
    assert np.isnan(o["lse"][2:4]).all() and o["lse"][4] == 5 and o["entropy"][4] == 0 and o["logp"][4] == -inf
    low = R.token_logp(np.full((1, 4), -3.4e38), [2], 1.0, 2)
    assert low["lse"][0] == -inf and low["top_index"][0].tolist() == [-1, -1]
    assert not R.token_logp_backward(z, [0] * 6, o["lse"], o["entropy"], np.ones(6))[1].any()
