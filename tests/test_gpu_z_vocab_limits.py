"""The vocabulary's operators past the sizes that one launch, one piece or 32 bits hold:
more tokens than a panel of statistics, more rows than workgroups, rows whose
elements lie past 2^31, the largest vocabularies.  Results are compared with the
same rows in a small call, with whole numbers that leave no roundings, or with
float64 on the GPU (a relative 2-norm within the roundings of the gradient of the
logits and of the result, 2^-8 each)."""
import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
BF, F, I64 = torch.bfloat16, torch.float32, torch.int64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _e(*shape, dtype=F):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _randn(*shape, dtype=F, seed=1, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _ids(T, V, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(0, V, (T,), generator=g, device="cuda")


def _ws(n):
    return _e(n, dtype=torch.uint8) if n else None


def _linear(x, w, y, entropy=True):
    T, (V, dim) = x.shape[0], w.shape
    o = {"logp": _e(T), "lse": _e(T), "entropy": _e(T) if entropy else None}
    nsp.nsp_linear_logp_fwd(x, w, y, o["logp"], o["lse"], o["entropy"], _ws(nsp.nsp_linear_logp_fwd_workspace(T, dim, V)))
    return o


def _linear_bwd(x, w, y, lse, g, dtype=BF):
    T, (V, dim) = x.shape[0], w.shape
    dx, dw = _e(T, dim, dtype=dtype), _e(V, dim, dtype=dtype)
    nsp.nsp_linear_logp_bwd(x, w, y, lse, dx, dw, _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V)), g_logp=g)
    return dx, dw


def _reference(x, w, y, g):
    """logp, lse, dx, dw in float64, some tokens at a time."""
    x, w = x.double(), w.double()
    out = [], [], []
    dw = torch.zeros_like(w)
    step = max(1, (1 << 26) // len(w))
    for a in range(0, len(x), step):
        xx, gg, yy = x[a:a + step], g[a:a + step].double()[:, None], y[a:a + step, None]
        z = xx @ w.t()
        lse = torch.logsumexp(z, 1, keepdim=True)
        da = -gg * (z - lse).exp()
        da.scatter_add_(1, yy, gg)
        for o, v in zip(out, (z.gather(1, yy)[:, 0] - lse[:, 0], lse[:, 0], da @ w)):
            o.append(v)
        dw += da.t() @ xx
    return (*map(torch.cat, out), dw)


def _near(a, b, tol):
    assert float((a.double() - b).norm() / b.norm()) <= tol


@pytest.mark.parametrize("T,dim,V", [(70001, 16, 700), (300001, 8, 40)])
def test_more_tokens_than_a_panel(T, dim, V):
    """Panels of the forward; tokens whose places one workgroup finds, whose rows many
    gather in turns.  logp: 2^-20 (1 + |logp| + |lse|) holds dim + V / 16 additions of steps of 2^-24."""
    x, w, y, g = _randn(T, dim, dtype=BF), _randn(V, dim, dtype=BF, seed=2, scale=0.5), _ids(T, V), _randn(T, seed=3)
    o = _linear(x, w, y)
    logp, lse, rdx, rdw = _reference(x, w, y, g)
    tol = 2.0 ** -20 * (1 + logp.abs() + lse.abs()) * (dim + V / 16) / 16
    assert bool(((o["logp"].double() - logp).abs() <= tol).all()) and bool(((o["lse"].double() - lse).abs() <= tol).all())
    dx, dw = _linear_bwd(x, w, y, o["lse"], g)
    _near(dx, rdx, 2.0 ** -7)
    _near(dw, rdw, 2.0 ** -7)


def test_largest_vocabulary():
    """2^24 rows: fewer tokens a panel, tiles near what a launch holds."""
    V, dim, T = 1 << 24, 8, 4100
    w, x, y = _randn(V, dim, dtype=BF, seed=2, scale=0.5), _randn(T, dim, dtype=BF), _ids(T, V)
    o = _linear(x, w, y)
    few = torch.tensor([0, 1, 4094, 4095, 4096, T - 1], device="cuda")
    z = x[few].double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    # 64 additions of a tile, 2^16 tiles in strands of 1024: 1100 steps of 2^-24; logits and exponents 2^-21 (|z| + 17)
    assert float((o["lse"][few].double() - lse).abs().max()) <= 1100 * 2.0 ** -24 + 2.0 ** -21 * (float(z.abs().max()) + 17)
    logp = z.gather(1, y[few, None])[:, 0] - lse
    assert float((o["logp"][few].double() - logp).abs().max()) <= 1100 * 2.0 ** -24 + 2.0 ** -20 * (float(z.abs().max()) + 17)
    assert bool(o["entropy"].isfinite().all())


def test_linear_rows_past_32_bits():
    """Views whose strides put the last rows past 2^31 elements, and hidden rows of more than 2^31 bytes."""
    T, V, dim, far = 2100, 2200, 64, 1 << 20
    x, w, y, g = _randn(T, dim, dtype=BF), _randn(V, dim, dtype=BF, seed=2, scale=0.3), _ids(T, V), _randn(T, seed=3)
    o = _linear(x, w, y)
    want = _linear_bwd(x, w, y, o["lse"], g)
    xf, wf, df = (torch.as_strided(_e((n - 1) * far + dim, dtype=BF), (n, dim), (far, 1)) for n in (T, V, V))
    assert (T - 1) * far > 1 << 31
    xf.copy_(x)
    wf.copy_(w)
    o2 = _linear(xf, wf, y)
    assert all(torch.equal(o[n], o2[n]) for n in o)
    dx = _e(T, dim, dtype=BF)
    nsp.nsp_linear_logp_bwd(xf, wf, y, o["lse"], dx, df, _ws(nsp.nsp_linear_logp_bwd_workspace(T, dim, V)), g_logp=g)
    assert torch.equal(dx, want[0]) and torch.equal(df, want[1])


def test_linear_many_wide_rows():
    T, V, dim = 70001, 48, 16384
    x, w, y, g = _randn(T, dim, dtype=BF), _randn(V, dim, dtype=BF, seed=2, scale=2.0 ** -7), _ids(T, V), _randn(T, seed=3)
    assert 2 * T * dim > 1 << 31
    o = _linear(x, w, y)
    dx, dw = _linear_bwd(x, w, y, o["lse"], g, F)
    few = torch.tensor([0, 1, 32767, 32768, 65535, 65536, T - 1], device="cuda")
    _, lse, rdx, _ = _reference(x[few], w, y[few], g[few])
    assert float((o["lse"][few].double() - lse).abs().max()) <= 2.0 ** -12    # sums of 16384 terms around 1, 2^-24 each
    _near(dx[few], rdx, 2.0 ** -8)
    rdw = torch.zeros(V, dim, dtype=torch.float64, device="cuda")
    for a in range(0, T, 8192):
        rdw += _reference(x[a:a + 8192], w, y[a:a + 8192], g[a:a + 8192])[3]
    _near(dw, rdw, 2.0 ** -8)


def test_distillation_of_more_parts_than_workgroups():
    T, V, K = (1 << 22) + 4099, 24, 3
    z, index, t = _randn(T, V, dtype=BF), _ids(T * K, V).view(T, K), _randn(T, K, seed=4).sub_(3)
    loss, lse, dz, g = _e(T), _e(T), _e(T, V, dtype=BF), _randn(T, seed=5)
    nsp.nsp_distill_fwd(z, index, t, loss, lse, _ws(nsp.nsp_distill_fwd_workspace(T, V)))
    nsp.nsp_distill_bwd(z, index, t, lse, g, dz)
    s = torch.tensor([0, 1, T // 3, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, T - 1], device="cuda")
    n = len(s)
    l2, s2, d2 = _e(n), _e(n), _e(n, V, dtype=BF)
    nsp.nsp_distill_fwd(z[s], index[s], t[s], l2, s2, _ws(nsp.nsp_distill_fwd_workspace(n, V)))
    nsp.nsp_distill_bwd(z[s], index[s], t[s], s2, g[s], d2)
    assert torch.equal(loss[s], l2) and torch.equal(lse[s], s2) and torch.equal(dz[s], d2)
    # every row's gradient: p and q are one's parts, so its sum is S - S, up to the roundings of 24 elements
    q = t.double().exp().sum(1)
    assert bool((dz.double().sum(1).abs() <= V * 2.0 ** -8 * 2 * q * g.double().abs()).all())


def test_distillation_rows_past_32_bits():
    T, V, K = 33, 70001, 20
    z, index, t = _randn(T, V, dtype=BF), _ids(T * K, V).view(T, K), _randn(T, K, seed=4).sub_(3)
    far = 1 << 27
    zf, df = (torch.as_strided(_e((T - 1) * far + V, dtype=BF), (T, V), (far, 1)) for _ in range(2))
    zf.copy_(z)
    out = []
    for a, d in ((z, _e(T, V, dtype=BF)), (zf, df)):
        loss, lse = _e(T), _e(T)
        nsp.nsp_distill_fwd(a, index, t, loss, lse, _ws(nsp.nsp_distill_fwd_workspace(T, V)))
        nsp.nsp_distill_bwd(a, index, t, lse, torch.ones_like(loss), d)
        out.append((loss, lse, d))
    assert (T - 1) * far > 1 << 31 and all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("T,dim", [((1 << 24) + 77, 8), ((1 << 20) * 4 + 4099, 1040), ((1 << 21) + 77, 1100)])
def test_embedding_of_many_tokens(T, dim):
    V = 1009
    w, ids = _randn(V, dim, dtype=BF), _ids(T, V)
    y = _e(T, dim, dtype=BF)
    nsp.nsp_embedding_fwd(ids, w, y)
    for a in range(0, T, 1 << 21):
        assert torch.equal(y[a:a + (1 << 21)], w[ids[a:a + (1 << 21)]])


def _whole(T, dim, seed=3):
    """Whole numbers -1 .. 2, as bf16."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(-1, 3, (T, dim), generator=g, device="cuda", dtype=torch.int8).to(BF)


def _count(ids, dy, V):
    """Sums of whole numbers, exact: by differences of running sums over the sorted ids
    (no atomic: those of torch on one frequent row take minutes)."""
    keys, order = ids.sort(stable=True)
    ends = torch.searchsorted(keys, torch.arange(V + 1, device="cuda"))
    want = torch.empty(V, dy.shape[1], dtype=torch.int64, device="cuda")
    for c in range(0, dy.shape[1], 256):
        run = torch.zeros(len(ids) + 1, min(256, dy.shape[1] - c), dtype=torch.int64, device="cuda")
        torch.cumsum(dy[order, c:c + 256].to(torch.int64), 0, out=run[1:])
        want[:, c:c + 256] = run[ends[1:]] - run[ends[:-1]]
    assert int(want.abs().max()) < 2 ** 24
    return want.double()


@pytest.mark.parametrize("T,dim,V", [(1 << 26, 1, 70001), ((1 << 24) + 5, 8, 300), ((1 << 22) + 4099, 33, (1 << 18) + 3), (540001, 4104, 5003)])
def test_embedding_gradient_of_many_tokens(T, dim, V):
    """Thousands of blocks of the sort, ids of many chunks, gradients past 2^31 elements."""
    ids, dy = _ids(T, V), _whole(T, dim)
    ids[::7] = V // 2                           # a frequent one
    dw = _e(V, dim)
    nsp.nsp_embedding_bwd(ids, dy, dw, _ws(nsp.nsp_embedding_bwd_workspace(T, dim, V)))
    torch.cuda.synchronize()
    print("[limits] gradient is there", flush=True)
    assert torch.equal(dw.double(), _count(ids, dy, V))


@pytest.mark.parametrize("T", [300, 9000, 20000])
def test_largest_table(T):
    """2^30 rows: four digits of the sort, more rows than a launch has threads for."""
    V = 1 << 30
    ids, dy = _ids(T, V), _whole(T, 1)
    ids[:3] = torch.tensor([0, V - 1, V], device="cuda")
    ids[T // 2:] = ids[:T - T // 2]             # twice each, about
    dw = torch.full((V, 1), float("nan"), dtype=BF, device="cuda")
    nsp.nsp_embedding_bwd(ids, dy, dw, _ws(nsp.nsp_embedding_bwd_workspace(T, 1, V)))
    there = ids < V
    at, slot = ids[there].unique(return_inverse=True)
    want = torch.zeros(len(at), dtype=torch.float64, device="cuda").index_add_(0, slot, dy[there][:, 0].double())
    assert torch.equal(dw[at][:, 0].double(), want)
    dw[at] = 0
    assert not dw.any()                         # (a NaN counts as something)
    y = _e(T, 1, dtype=BF)
    dw[at] = 3
    nsp.nsp_embedding_fwd(ids, dw, y)
    assert torch.equal(y[:, 0].float(), 3 * there.float())


@pytest.mark.parametrize("T", [300, 20000])
def test_table_with_far_rows(T):
    V, dim, far = 5000, 24, 1 << 20
    assert (V - 1) * far > 1 << 32
    w, ids, dy = _randn(V, dim, dtype=BF), _ids(T, V), _whole(T, dim)
    ids[0] = V - 1
    wf = torch.as_strided(_e((V - 1) * far + dim, dtype=BF), (V, dim), (far, 1))
    wf.copy_(w)
    y, y2 = _e(T, dim), _e(T, dim)
    nsp.nsp_embedding_fwd(ids, w, y)
    nsp.nsp_embedding_fwd(ids, wf, y2)
    assert torch.equal(y, y2)
    ws = _ws(nsp.nsp_embedding_bwd_workspace(T, dim, V))
    nsp.nsp_embedding_bwd(ids, dy, wf, ws)
    assert torch.equal(wf.double(), _count(ids, dy, V))


@pytest.mark.parametrize("wt,dt", [(BF, BF), (F, F), (BF, F), (F, BF)])
@pytest.mark.parametrize("T,dim", [(511, 40), (1024, 33), (1025, 33), (2047, 7), (2048, 72), (2049, 72), (1024, 1032), (1040, 1032), (2000, 300)])
def test_embedding_gradient_with_and_without_a_sort(T, dim, wt, dt):
    """Sizes around those from which tokens are sorted: sums of whole numbers, exact in float32 (and, below 256, in bf16)."""
    V = 77
    ids, dy = _ids(T, V + 2) - 1, _whole(T, dim).to(dt)         # ids out of the vocabulary on both sides
    ids[T // 3:T // 2] = 5
    there = (ids >= 0) & (ids < V)
    want = _count(torch.where(there, ids, V), dy, V + 1)[:V]
    dw = torch.full((V, dim), float("nan"), dtype=wt, device="cuda")
    nsp.nsp_embedding_bwd(ids, dy, dw, _ws(nsp.nsp_embedding_bwd_workspace(T, dim, V)))
    assert torch.equal(dw, want.to(wt))
    # one id of all; none at all; rows apart, what lies between them left as it was
    for one in (3, -1):
        ids.fill_(one)
        wide = torch.full((V, dim + 3), 7.0, dtype=wt, device="cuda")
        nsp.nsp_embedding_bwd(ids, dy, wide[:, :dim], _ws(nsp.nsp_embedding_bwd_workspace(T, dim, V)))
        want = torch.zeros(V, dim, dtype=torch.float64, device="cuda")
        if one >= 0:
            want[one] = dy.double().sum(0)
        assert torch.equal(wide[:, :dim], want.to(wt)) and bool((wide[:, dim:] == 7).all())


@pytest.mark.parametrize("T,dim", [(1, 1 << 20), (2, 1 << 20), (20, 70001), (32, 40000), (33, 40000)])
def test_embedding_of_widest_rows(T, dim):
    """Few tokens of wide rows: with and without a sort, one chunk and two."""
    V = 5
    ids, dy, w = _ids(T, V), _whole(T, dim).float(), _whole(V, dim)
    ids[T // 2:] = 3
    dw = torch.full((V, dim), float("nan"), device="cuda")
    nsp.nsp_embedding_bwd(ids, dy, dw, _ws(nsp.nsp_embedding_bwd_workspace(T, dim, V)))
    assert torch.equal(dw.double(), _count(ids, dy, V))
    y = _e(T, dim)
    nsp.nsp_embedding_fwd(ids, w, y, scale=2.0)
    assert torch.equal(y, 2 * w[ids].float())
