"""Gradients from hidden rows while another stream writes the workspace, which the call
needs for itself (two calls at a time need two): the gradients are then anything, but
nothing outside dx's and dw's rows and the workspace is written, whatever number of rows,
places and order of tokens lie there.  Afterwards a call alone gives what it gave before."""
import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import draw, strided, untouched
from test_gpu_zc_embedding_workspace_written import bands_whole, guarded, noises

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


# (two rows a token; sums of the logits in parts; places by every workgroup and by one)
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,dim,V", [(40, 264, 3000), (100, 2048, 300), (300, 2048, 1000), (900, 136, 2100), (2000, 136, 2100), (5000, 72, 700)])
def test_nothing_else_is_touched(T, dim, V, dtype):
    rng = np.random.default_rng(T)
    x, w = draw(rng, (T, dim), BF), draw(rng, (V, dim), BF, 0.1)
    y = torch.from_numpy(rng.integers(-1, V, T)).cuda()
    g = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    lse = torch.empty(T, device="cuda")
    nsp.nsp_linear_logp_fwd(x, w, None, None, lse, None, torch.empty(nsp.nsp_linear_logp_fwd_workspace(T, dim, V), dtype=torch.uint8, device="cuda"))
    dx, bx, outx = strided(torch.zeros((T, dim), dtype=dtype, device="cuda"), 8, 8)
    dw, bw, outw = strided(torch.zeros((V, dim), dtype=dtype, device="cuda"), 16, 8)
    buf, ws = guarded(nsp.nsp_linear_logp_bwd_workspace(T, dim, V))

    def run():
        nsp.nsp_linear_logp_bwd(x, w, y, lse, dx, dw, ws, g_logp=g)

    def whole():
        return untouched(bx, outx) and untouched(bw, outw) and bands_whole(buf)

    run()
    want = dx.clone(), dw.clone()
    side, some = torch.cuda.Stream(), noises(ws.numel())
    torch.cuda.synchronize()
    for i in range(30):
        with torch.cuda.stream(side):
            ws.copy_(some[i % len(some)])
        run()
        with torch.cuda.stream(side):                  # (the number of rows, their order and places lie first)
            ws[:1 << 16].copy_(some[(i + 1) % len(some)][:1 << 16])
    torch.cuda.synchronize()
    assert whole()
    run()
    torch.cuda.synchronize()
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and whole()
