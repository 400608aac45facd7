"""Pins of the row operators' oracle: a masked target's log probability is the
limit of ever smaller logits, whichever masked value stands there."""
import numpy as np

from oracle import rows as R


def test_a_masked_target_is_a_limit():
    z = np.array([[0.0, 1.0, v] for v in (-1e3, -2.0 ** 125, -2.0 ** 126, -3.4e38, -np.inf)])
    for scale in (2.0 ** -60, 0.25, 1.0):
        logp = R.token_logp(z, [2] * 5, scale)["logp"]
        assert np.all(np.diff(logp[:3]) < 0) and np.all(logp[2:] == -np.inf) and np.all(np.isfinite(logp[:2]))
    z[3, 0] = np.nan
    assert np.isnan(R.token_logp(z, [2] * 5)["logp"][3])
