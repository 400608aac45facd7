"""The distillation's gradient of rows that a workgroup passes over in several turns (more
than 16 alternatives in bf16 two of 16 KB, more than 128 four), over the logits
themselves: bit for bit what a call into another buffer gives, whose values are held to the
definition elsewhere; odd lengths, a row's last turn short, alternatives in every
turn and at its borders."""
import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, strided, untouched

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,V,K", [(1, 70001, 20), (3, 33000, 17), (5, 40000, 129), (2, 131072, 256), (30, 16385, 64), (24, 50021, 33), (7, 9001, 256)])
def test_in_place(T, V, K, dtype):
    rng = np.random.default_rng(T + V + K)
    z = torch.from_numpy((rng.standard_normal((T, V)) * 3).astype(np.float32)).to(dtype).cuda()
    index = rng.integers(0, V, (T, K))
    turn = 256 * (8 if dtype == BF else 4) * 4
    edges = [v for k in range(1, 9) for v in (k * turn - 1, k * turn) if v < V][:K - 1]
    index[:, :len(edges)] = edges
    index[:, -1] = V - 1
    index = torch.from_numpy(index).cuda()
    t = torch.from_numpy((rng.standard_normal((T, K)) - 5).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    lse = torch.logsumexp(z.double(), 1).float()
    for kind in (nsp.NSP_DISTILL_GIVEN, nsp.NSP_DISTILL_NORMALIZED):
        want = torch.full_like(z, float("nan"))
        nsp.nsp_distill_bwd(z, index, t, lse, g, want, kind=kind)
        # every row's gradient sums to g (S - S), up to the roundings of its elements
        assert bool((want.double().sum(1).abs() <= 2.0 ** -7 * want.double().abs().sum(1) + 1e-6).all())
        zs, buf, out = strided(z, 5, 3)
        again = z.clone()
        nsp.nsp_distill_bwd(zs, index, t, lse, g, zs, kind=kind)
        nsp.nsp_distill_bwd(again, index, t, lse, g, again, kind=kind)
        torch.cuda.synchronize()
        assert torch.equal(zs, want) and torch.equal(again, want) and untouched(buf, out)
        # the weights of alternatives at the borders of the turns
        q = as64(t)
        q = np.exp(q - (np.log(np.exp(q).sum(1, keepdims=True)) if kind else 0.0))
        i = index.cpu().numpy()
        for r in range(T):
            at = np.unique(i[r])
            have = np.array([q[r, i[r] == v].sum() for v in at])
            zz = as64(z)[r, at]
            full = as64(g)[r] * (np.exp(zz - as64(lse)[r]) * q[r].sum() - have)
            assert np.abs(as64(want)[r, at] - full).max() <= (2.0 ** -7 if dtype == BF else 2.0 ** -14) * (np.abs(as64(g)[r]) * (have + q[r].sum() * np.exp(zz - as64(lse)[r]))).max()
