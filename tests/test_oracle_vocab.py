"""The oracle of the vocabulary's operators against torch's own formulas and
automatic differentiation in float64, on the CPU."""
import numpy as np
import torch

from oracle import vocab as O


def _t(x, grad=False):
    return torch.from_numpy(np.asarray(x, np.float64)).requires_grad_(grad)


def test_linear_logp_and_its_gradient():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((6, 5)), rng.standard_normal((9, 5))
    y = np.array([3, -1, 8, 0, 9, 2])
    g = rng.standard_normal((3, 6))
    tx, tw = _t(x, True), _t(w, True)
    lp = torch.log_softmax(1.3 * tx @ tw.t(), 1)
    given = torch.from_numpy((y >= 0) & (y < 9))
    logp = torch.where(given, lp.gather(1, torch.from_numpy(y).clamp(0, 8)[:, None])[:, 0], torch.zeros(6, dtype=torch.float64))
    lse = torch.logsumexp(1.3 * tx @ tw.t(), 1)
    ent = -(lp.exp() * lp).sum(1)
    ((logp * _t(g[0])).sum() + (lse * _t(g[1])).sum() + (ent * _t(g[2])).sum()).backward()
    got = O.linear_logp(x, w, y, 1.3)
    for n, v in (("logp", logp), ("lse", lse), ("entropy", ent)):
        assert np.abs(got[n] - v.detach().numpy()).max() < 1e-12
    dx, dw, _ = O.linear_logp_backward(x, w, y, got["lse"], got["entropy"], *g, scale=1.3)
    assert np.abs(dx - tx.grad.numpy()).max() < 1e-12 and np.abs(dw - tw.grad.numpy()).max() < 1e-12


def test_tokens_without_a_gradient_take_no_part():
    x, w = np.ones((3, 2)), np.ones((4, 2))
    x[1] = np.nan
    lse = np.array([2.0 + np.log(4.0)] * 3)
    dx, dw, _ = O.linear_logp_backward(x, w, np.array([1, -1, 2]), lse, np.zeros(3), np.ones(3))
    assert np.isfinite(dx).all() and np.isfinite(dw).all() and not dx[1].any()


def test_distillation_and_its_gradient():
    rng = np.random.default_rng(2)
    z, index, t = rng.standard_normal((5, 11)) * 2, rng.integers(-1, 12, (5, 4)), rng.standard_normal((5, 4)) - 2
    index[0] = [3, 3, 5, 3]                                # the same token more than once
    index[1] = -1
    t[2, 1] = -np.inf
    for normalized in (False, True):
        tz = _t(z, True)
        lp = torch.log_softmax(0.7 * tz, 1)
        loss = torch.zeros(5, dtype=torch.float64)
        for r in range(5):
            ks = [k for k in range(4) if 0 <= index[r, k] < 11 and t[r, k] > -np.inf]
            if ks:
                v = _t(t[r, ks])
                v = v - torch.logsumexp(v, 0) if normalized else v
                loss[r] = (v.exp() * (v - lp[r, index[r, ks]])).sum()
        got, lse = O.distill(z, index, t, normalized, 0.7)
        assert np.abs(got - loss.detach().numpy()).max() < 1e-12
        assert np.abs(lse - torch.logsumexp(0.7 * tz, 1).detach().numpy()).max() < 1e-12
        g = rng.standard_normal(5)
        (loss * _t(g)).sum().backward()
        assert np.abs(O.distill_backward(z, index, t, lse, g, normalized, 0.7) - tz.grad.numpy()).max() < 1e-12


def test_distillation_of_masked_and_lost_rows():
    z = np.array([[0.0, -np.inf, 1.0], [0.0, -np.inf, 1.0], [-np.inf] * 3, [np.nan, 0.0, 0.0], [0.0, 0.0, 0.0]])
    index = np.array([[1], [0], [0], [1], [1]])
    t = np.array([[-1.0], [-1.0], [-1.0], [-1.0], [np.nan]])
    loss, lse = O.distill(z, index, t)
    assert loss[0] == np.inf and np.isfinite(loss[1]) and loss[2] == np.inf and np.isnan(loss[3]) and np.isnan(loss[4])
    d = O.distill_backward(z, index, t, lse, np.ones(5))
    assert d[0, 1] == -np.exp(-1.0) and not d[2].any() and np.isnan(d[3]).all() and np.isnan(d[4]).all()


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(3)
    w, ids = rng.standard_normal((7, 3)), np.array([0, 6, 6, 2, 6, 0])
    tw = _t(w, True)
    y = 1.5 * tw[torch.from_numpy(ids)]
    dy = rng.standard_normal((6, 3))
    (y * _t(dy)).sum().backward()
    assert np.abs(O.embedding(ids, w, 1.5) - y.detach().numpy()).max() < 1e-15
    assert np.abs(O.embedding_backward(ids, dy, 7, 1.5) - tw.grad.numpy()).max() < 1e-14
    out = np.array([-1, 7, 1])
    assert not O.embedding(out, w)[:2].any() and not O.embedding_backward(out, dy[:3], 7)[[0, 2, 3, 4, 5, 6]].any()
