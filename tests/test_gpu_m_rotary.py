"""Rotary positions against the float64 definition.

Tolerance: half a step of the type, and of each product's factor 2^-21: the
angle's fraction of a half turn is rounded once (2^-25 pi), sincospi is within
2 units of the last place (2^-23), the amplitude's product, the two products
and their difference round 2^-24 each; the angle itself, in 64 bits, is within
2^-50 of its size."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp

from gpu_util import require_gpu
from rows_util import as64, draw, half_step, strided, untouched, within

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _check(name, x, y, pos, freqs, pairs, scale, backward):
    x64, r = as64(x), 2 * len(freqs)
    want = R.rotary(x64, pos, freqs, pairs, scale, backward)
    first, second = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    both = np.abs(x64[..., first]) + np.abs(x64[..., second])
    angle = np.abs(np.asarray(pos, np.float64))[:, None, None] * freqs
    tol = half_step(x.dtype) * np.abs(want)
    for part in (first, second):
        tol[..., part] += both * abs(scale) * (2.0 ** -21 + angle * 2.0 ** -50)
    tol[..., r:] = 0.0
    within(name, as64(y), want, tol)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T,hq,hk,D,rot", [
    (1, 1, 0, 2, 2), (1, 32, 4, 128, 128), (3, 4, 1, 128, 128), (37, 8, 2, 64, 32), (5, 3, 1, 80, 20), (7, 2, 2, 7, 6), (4, 1, 3, 33, 30),
    (513, 5, 1, 96, 96), (2, 2, 1, 256, 256), (3, 2, 1, 256, 130), (19, 16, 16, 128, 64)])
def test_against_the_definition(T, hq, hk, D, rot, dtype, pairs, backward):
    rng = np.random.default_rng(T * 1000 + D)
    pos = rng.integers(0, 400000, T)
    pos[0] = 0 if T > 1 else 393215
    freqs = 1e6 ** (-np.arange(0, rot, 2) / rot)
    q, k = draw(rng, (T, hq, D), dtype), draw(rng, (T, max(1, hk), D), dtype)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    call = nsp.nsp_rotary_bwd if backward else nsp.nsp_rotary_fwd
    args = (q, qo, k, ko) if hk else (q, qo)
    call(torch.from_numpy(pos).cuda(), torch.from_numpy(freqs).cuda(), *args, scale=1.25, layout=int(pairs))
    torch.cuda.synchronize()
    _check("q", q, qo, pos, freqs, pairs, 1.25, backward)
    if hk:
        _check("k", k, ko, pos, freqs, pairs, 1.25, backward)
    else:
        assert bool(ko.isnan().all())


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("lead,gap,token_gap", [(0, 0, 0), (1, 3, 5), (4, 8, 16)])
def test_strided_views_and_in_place(lead, gap, token_gap, dtype, pairs):
    """Any element alignment; what lies between the rows stays as it is; the
    unrotated rest is kept in place; a broadcast input."""
    rng = np.random.default_rng(7)
    T, D = 6, 48
    pos, freqs = np.array([0, 5, 1 << 24, -9, 77, 131071]), 1e4 ** (-np.arange(0, 36, 2) / 36)
    p, f = torch.from_numpy(pos).cuda(), torch.from_numpy(freqs).cuda()
    q, k = draw(rng, (T, 4, D), dtype), draw(rng, (T, 2, D), dtype)
    qv, qb, qm = strided(q, lead, gap, token_gap)
    kv, kb, km = strided(k, lead, gap, token_gap)
    qo, qob, qom = strided(torch.zeros_like(q), lead + 1, gap, token_gap)
    nsp.nsp_rotary_fwd(p, f, qv, qo, kv, kv, layout=int(pairs))              # q apart, k in place
    torch.cuda.synchronize()
    _check("q", q, qo, pos, freqs, pairs, 1.0, False)
    _check("k in place", k, kv, pos, freqs, pairs, 1.0, False)
    assert torch.equal(qv, q) and untouched(qb, qm) and untouched(kb, km) and untouched(qob, qom)
    one = q[:1].expand(T, 4, D)                                              # every token the same row
    out = torch.empty_like(q)
    nsp.nsp_rotary_fwd(p, f, one, out, layout=int(pairs))
    torch.cuda.synchronize()
    _check("broadcast", one, out, pos, freqs, pairs, 1.0, False)


def test_heads_before_tokens():
    """[heads, tokens, dim] memory, seen as [tokens, heads, dim]."""
    rng = np.random.default_rng(8)
    x = draw(rng, (3, 50, 64), BF)
    pos, freqs = np.arange(50), 1e4 ** (-np.arange(0, 64, 2) / 64)
    y = torch.empty_like(x)
    nsp.nsp_rotary_fwd(torch.from_numpy(pos).cuda(), torch.from_numpy(freqs).cuda(), x.transpose(0, 1), y.transpose(0, 1))
    torch.cuda.synchronize()
    _check("q", x.transpose(0, 1), y.transpose(0, 1), pos, freqs, False, 1.0, False)


def test_gradient_is_the_inverse_turn_and_the_transpose():
    rng = np.random.default_rng(9)
    pos, freqs = torch.randint(0, 300000, (200,), device="cuda"), torch.from_numpy(nsp.nsp_rotary_frequencies(128, 1e6)[0]).cuda()
    x, g = draw(rng, (200, 4, 128), F), draw(rng, (200, 4, 128), F)
    y, dx, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    nsp.nsp_rotary_fwd(pos, freqs, x, y, scale=2.0)
    nsp.nsp_rotary_bwd(pos, freqs, g, dx, scale=2.0)
    nsp.nsp_rotary_bwd(pos, freqs, y, back, scale=0.5)
    torch.cuda.synchronize()
    # <R x, g> = <x, R' g>, each pair's within 2^-20 of its products' size
    a, b = (as64(y) * as64(g)).sum(), (as64(x) * as64(dx)).sum()
    assert abs(a - b) <= 2.0 ** -19 * 2 * (np.abs(as64(x)).sum() * 4)
    assert np.abs(as64(back) - as64(x)).max() <= 2.0 ** -19 * 2 * np.abs(as64(x)).max()


def test_no_tokens_many_tokens_and_determinism():
    freqs = torch.from_numpy(nsp.nsp_rotary_frequencies(64, 1e4)[0]).cuda()
    e = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    nsp.nsp_rotary_fwd(torch.empty(0, dtype=torch.int64, device="cuda"), freqs, e, e)
    rng = np.random.default_rng(10)
    T = 70001                                                               # several tokens a workgroup, the last one short
    pos = np.concatenate([np.arange(40000), np.arange(T - 40000)])
    x = draw(rng, (T, 1, 64), BF)
    y, z = torch.empty_like(x), torch.empty_like(x)
    for out in (y, z):
        nsp.nsp_rotary_fwd(torch.from_numpy(pos).cuda(), freqs, x, out)
    torch.cuda.synchronize()
    assert torch.equal(y.view(torch.int16), z.view(torch.int16))
    _check("long", x, y, pos, as64(freqs), False, 1.0, False)


def test_on_another_stream_and_replayed():
    """A side stream, and a graph whose replays read what the buffers hold then."""
    rng = np.random.default_rng(11)
    freqs = torch.from_numpy(nsp.nsp_rotary_frequencies(128, 1e4)[0]).cuda()
    x, pos = draw(rng, (33, 3, 128), BF), torch.arange(33, device="cuda")
    y = torch.zeros_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    nsp.nsp_rotary_fwd(pos, freqs, x, y, stream=s)
    s.synchronize()
    _check("side stream", x, y, pos.cpu().numpy(), as64(freqs), False, 1.0, False)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nsp.nsp_rotary_fwd(pos, freqs, x, y)
    for k in range(3):
        x.copy_(draw(rng, x.shape, BF))
        pos.add_(1000)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        _check(f"replay {k}", x, y, pos.cpu().numpy(), as64(freqs), False, 1.0, False)
