"""The embedding's gradient while another stream writes the workspace, which the call
needs for itself (two calls at a time need two): its sums are then anything, but
nothing outside dw's rows and the workspace is written and no row outside dy is read,
whatever the counts, ids and places in the workspace are.  Afterwards a call alone gives what
it gave before."""
import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import draw, strided, untouched

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def guarded(n):
    """n bytes between two bands of 0xA5: (buffer, bytes)."""
    buf = torch.full((n + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    return buf, buf[GUARD:GUARD + n]


def bands_whole(buf):
    return bool((buf[:GUARD] == 0xA5).all()) and bool((buf[-GUARD:] == 0xA5).all())


def noises(n):
    """What may come to lie in it: all ones, zeros, any bits, small whole numbers, numbers next to 2^31."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    words = -(-n // 4)
    low = [(-(1 << 31), (1 << 31) - 1), (0, 600), ((1 << 31) - 600, (1 << 31) - 1)]
    out = [torch.full((n,), 255, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")]
    return out + [torch.randint(a, b, (words,), generator=g, device="cuda", dtype=torch.int32).view(torch.uint8)[:n] for a, b in low]


@pytest.mark.parametrize("T,dim,V", [(9000, 40, 700), (17000, 40, 700), (20000, 3, 70000), (60000, 264, 300), (600001, 8, 5000)])
def test_nothing_else_is_touched(T, dim, V):
    rng = np.random.default_rng(T)
    ids = torch.from_numpy(rng.integers(-1, V + 1, T)).cuda()
    dy = draw(rng, (T, dim), torch.bfloat16)
    dw, band, outside = strided(torch.zeros((V, dim), device="cuda"), 16, 8)
    buf, ws = guarded(nsp.nsp_embedding_bwd_workspace(T, dim, V))
    nsp.nsp_embedding_bwd(ids, dy, dw, ws)
    want = dw.clone()
    side, some = torch.cuda.Stream(), noises(ws.numel())
    torch.cuda.synchronize()
    for i in range(40):
        with torch.cuda.stream(side):
            ws.copy_(some[i % len(some)])
        nsp.nsp_embedding_bwd(ids, dy, dw, ws)
        with torch.cuda.stream(side):
            ws.copy_(some[(i + 1) % len(some)])
    torch.cuda.synchronize()
    assert untouched(band, outside) and bands_whole(buf)
    nsp.nsp_embedding_bwd(ids, dy, dw, ws)
    torch.cuda.synchronize()
    assert torch.equal(dw, want) and untouched(band, outside) and bands_whole(buf)
