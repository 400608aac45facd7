"""Backwards of many rows at the widths that no vectors a lane fit: less than a
vector, more than 16384.  Their dw and db are held to the bound of all others,
128 + rows / 256 roundings of the terms' sizes."""
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from norm_exact import LAYER, RMS, Exact
from rows_util import F32

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("n,dtype", [(1, BF), (7, BF), (1, F), (3, F)])
def test_small_terms_behind_large_ones(n, dtype):
    """128 rows of 2^24, then ones: a sum of one strand would stand still."""
    rows = 1 << 20
    dy = torch.ones(rows, n, dtype=dtype, device="cuda")
    dy[:128] = 2.0 ** 24
    x, rstd, dx = torch.ones_like(dy), torch.ones(rows, device="cuda"), torch.empty_like(dy)
    dw, db = (torch.zeros(n, device="cuda") for _ in range(2))
    ws = torch.empty(nsp.nsp_norm_bwd_workspace(rows, 1, n), dtype=torch.uint8, device="cuda")
    nsp.nsp_norm_bwd(x, torch.ones(n, device="cuda"), dy, None, rstd, dx, dw, db, ws, kind=RMS)
    torch.cuda.synchronize()
    want = 128 * 2.0 ** 24 + rows - 128
    tol = (128 + rows / 256) * F32 * want
    assert float((dw.double() - want).abs().max()) <= tol and float((db.double() - want).abs().max()) <= tol, (dw - want, tol)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("rows,n,dtype", [(37, 7, BF), (4096, 5, BF), (4097, 7, BF), (30011, 1, BF), (300007, 3, F), (20003, 2, F),
                                          (4096, 20000, BF), (5003, 16392, BF), (4099, 16385, F)])
def test_every_row_counts(rows, n, dtype, kind):
    e = Exact(rows, n, dtype, kind).run()
    torch.cuda.synchronize()
    e.check()
    dx, dw, db = e.dx.clone(), e.dw.clone(), e.db.clone()
    e.run(dx=e.dy)                                    # in place: dw and db are of what dy was
    torch.cuda.synchronize()
    assert torch.equal(e.dy, dx) and torch.equal(e.dw, dw) and torch.equal(e.db, db)


def test_the_bias_alone():
    e = Exact(9001, 6, BF, RMS)
    nsp.nsp_norm_bwd(e.x, e.w, e.dy, None, e.rstd, e.dx, None, e.db, e.ws, kind=RMS)
    torch.cuda.synchronize()
    e.dw = (e.dy.double() * e.x.double() * e.rstd.double()[:, None]).sum(0)
    e.check()
