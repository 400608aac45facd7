"""Refusals of the row operators, their workspace sizes and the rotary
frequencies: host code, checked without a GPU (nothing is launched on any of
the error paths, and the addresses are never used)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

FAKE = 0x10000
EINVAL, EUNSUPPORTED, EWORKSPACE = nsp.NSP_EINVAL, nsp.NSP_EUNSUPPORTED, nsp.NSP_EWORKSPACE


def _rows(data=FAKE, ts=0, hs=0):
    return bytes(nsp.CRows(data, ts, hs))


def _call(name, args):
    lib = nsp.load_library()
    st = getattr(lib, name)(*args.values())
    return st, lib.nsp_last_error().decode()


def _rotary(**kw):
    a = dict(layout=0, dtype=0, T=4, D=64, rot=64, freqs=FAKE, scale=1.0, pos=FAKE, hq=2, q=_rows(FAKE, 128, 64), qo=_rows(2 * FAKE, 128, 64),
             hk=1, k=_rows(3 * FAKE, 64, 64), ko=_rows(4 * FAKE, 64, 64), stream=None)
    a.update(kw)
    return a


def _norm_fwd(**kw):
    a = dict(kind=0, dtype=0, wdtype=0, T=4, H=2, n=64, x=_rows(FAKE, 128, 64), w=FAKE, b=FAKE, eps=1e-5, y=_rows(2 * FAKE, 128, 64), mean=FAKE,
             rstd=FAKE, stream=None)
    a.update(kw)
    return a


def _norm_bwd(**kw):
    a = dict(kind=0, dtype=0, wdtype=0, T=4, H=2, n=64, x=_rows(FAKE, 128, 64), w=FAKE, dy=_rows(2 * FAKE, 128, 64), mean=FAKE, rstd=FAKE,
             dx=_rows(3 * FAKE, 128, 64), dw=FAKE, db=FAKE, ws=FAKE, ws_bytes=1 << 20, stream=None)
    a.update(kw)
    return a


def _logp_fwd(**kw):
    a = dict(dtype=0, T=4, V=5000, z=FAKE, stride=5000, y=FAKE, scale=1.0, logp=FAKE, lse=FAKE, ent=FAKE, top=2, tl=FAKE, ti=FAKE, ws=FAKE,
             ws_bytes=4 << 20, stream=None)
    a.update(kw)
    return a


def _logp_bwd(**kw):
    a = dict(dtype=0, T=4, V=5000, z=FAKE, stride=5000, y=FAKE, scale=1.0, lse=FAKE, ent=FAKE, gl=FAKE, gs=FAKE, ge=FAKE, dz=4 * FAKE,
             dstride=5000, stream=None)
    a.update(kw)
    return a


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("call", ["nsp_rotary_fwd", "nsp_rotary_bwd"])
@pytest.mark.parametrize("kw,status,word", [
    (dict(layout=2), EINVAL, "layout"), (dict(dtype=2), EINVAL, "dtype"), (dict(T=-1), EINVAL, "n_tokens"), (dict(T=1 << 31), EINVAL, "n_tokens"),
    (dict(T=(1 << 31) - 1), EINVAL, "rows"), (dict(D=0, rot=2), EINVAL, "head_dim"), (dict(D=257, rot=2), EUNSUPPORTED, "head_dim"),
    (dict(rot=0), EINVAL, "rot_dim"), (dict(rot=63), EINVAL, "rot_dim"), (dict(rot=66), EINVAL, "rot_dim"), (dict(scale=INF), EINVAL, "scale"),
    (dict(scale=NAN), EINVAL, "scale"), (dict(freqs=None), EINVAL, "freqs"), (dict(freqs=FAKE + 4), EINVAL, "freqs"),
    (dict(pos=None), EINVAL, "positions"), (dict(pos=FAKE + 4), EINVAL, "positions"), (dict(hq=0), EINVAL, "q_heads"),
    (dict(hk=-1), EINVAL, "k_heads"), (dict(hk=0), EINVAL, "NULL"), (dict(q=None), EINVAL, "q"), (dict(ko=None), EINVAL, "k"),
    (dict(q=_rows(None, 128, 64)), EINVAL, "NULL"), (dict(q=_rows(FAKE + 1, 128, 64)), EINVAL, "aligned"),
    (dict(dtype=1, q=_rows(FAKE + 2, 128, 64)), EINVAL, "aligned"), (dict(q=_rows(FAKE, -1, 64)), EINVAL, "strides"),
    (dict(q=_rows(FAKE, 1 << 41, 64)), EINVAL, "strides"), (dict(qo=_rows(2 * FAKE, 128, 63)), EINVAL, "overlap"),
    (dict(qo=_rows(2 * FAKE, 127, 64)), EINVAL, "overlap"), (dict(qo=_rows(2 * FAKE, 0, 64)), EINVAL, "overlap"),
    (dict(qo=_rows(2 * FAKE, 64, 64)), EINVAL, "overlap"), (dict(qo=_rows(FAKE + 2, 128, 64)), EINVAL, "same view"),
    (dict(qo=_rows(FAKE, 64, 256)), EINVAL, "same view"), (dict(ko=_rows(3 * FAKE + 64, 64, 64)), EINVAL, "same view"),
])
def test_rotary_refusals(call, kw, status, word):
    st, msg = _call(call, _rotary(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", [
    (dict(kind=2), EINVAL, "kind"), (dict(dtype=3), EINVAL, "dtype"), (dict(wdtype=3), EINVAL, "w_dtype"), (dict(T=-1), EINVAL, "n_tokens"),
    (dict(T=1 << 30, H=4), EINVAL, "rows"), (dict(H=0), EINVAL, "n_heads"), (dict(n=0), EINVAL, "n = 0"), (dict(n=65537), EUNSUPPORTED, "65537"),
    (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=NAN), EINVAL, "eps"), (dict(eps=INF), EINVAL, "eps"), (dict(x=None), EINVAL, "x is NULL"),
    (dict(y=None), EINVAL, "y is NULL"), (dict(y=_rows(2 * FAKE, 64, 64)), EINVAL, "overlap"), (dict(y=_rows(FAKE + 128, 128, 64)), EINVAL, "same view"),
    (dict(w=FAKE + 1), EINVAL, "w is"), (dict(wdtype=1, b=FAKE + 2), EINVAL, "b is"), (dict(mean=FAKE + 2), EINVAL, "mean"),
    (dict(rstd=FAKE + 2), EINVAL, "rstd"),
])
def test_norm_refusals(kw, status, word):
    st, msg = _call("nsp_norm_fwd", _norm_fwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", [
    (dict(kind=-1), EINVAL, "kind"), (dict(dtype=3), EINVAL, "dtype"), (dict(n=65537), EUNSUPPORTED, "n ="), (dict(dy=None), EINVAL, "dy"),
    (dict(dx=None), EINVAL, "dx"), (dict(dx=_rows(3 * FAKE, 0, 64)), EINVAL, "overlap"), (dict(dx=_rows(2 * FAKE, 128, 65)), EINVAL, "overlap"),
    (dict(dx=_rows(2 * FAKE + 4, 128, 64)), EINVAL, "same view"), (dict(dx=_rows(FAKE + 4, 128, 64)), EINVAL, "same view"),
    (dict(mean=None), EINVAL, "mean"), (dict(rstd=None), EINVAL, "rstd"), (dict(dw=FAKE + 1), EINVAL, "dw"), (dict(db=FAKE + 1), EINVAL, "db"),
    (dict(T=200, ws=None), EWORKSPACE, "workspace"), (dict(T=200, ws=FAKE + 128), EINVAL, "workspace"),
    (dict(T=200, ws_bytes=10), EWORKSPACE, "workspace"),
])
def test_norm_backward_refusals(kw, status, word):
    st, msg = _call("nsp_norm_bwd", _norm_bwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(T=-1), EINVAL, "n_tokens"), (dict(V=0), EINVAL, "vocab"), (dict(V=(1 << 30) + 1), EUNSUPPORTED, "vocab"),
    (dict(scale=0.0), EINVAL, "scale"), (dict(scale=-1.0), EINVAL, "scale"), (dict(scale=NAN), EINVAL, "scale"), (dict(scale=1e30), EINVAL, "scale"),
    (dict(z=None), EINVAL, "logits"), (dict(z=FAKE + 1), EINVAL, "logits"), (dict(stride=-1), EINVAL, "stride"), (dict(lse=None), EINVAL, "lse"),
    (dict(y=None), EINVAL, "targets"), (dict(y=FAKE + 4), EINVAL, "targets"), (dict(top=-1), EINVAL, "top"), (dict(top=65), EUNSUPPORTED, "top"),
    (dict(tl=None), EINVAL, "top_logp"), (dict(ti=None), EINVAL, "top_index"), (dict(ti=FAKE + 4), EINVAL, "top_index"),
    (dict(ws=None), EWORKSPACE, "workspace"), (dict(ws_bytes=1), EWORKSPACE, "workspace"), (dict(ws=FAKE + 16), EINVAL, "workspace"),
])
def test_token_logp_refusals(kw, status, word):
    st, msg = _call("nsp_token_logp_fwd", _logp_fwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=2), EINVAL, "dtype"), (dict(V=-5), EINVAL, "vocab"), (dict(scale=0.0), EINVAL, "scale"), (dict(lse=None), EINVAL, "lse"),
    (dict(ent=None), EINVAL, "entropy"), (dict(y=None), EINVAL, "targets"), (dict(gl=FAKE + 1), EINVAL, "g_logp"),
    (dict(gs=FAKE + 1), EINVAL, "g_lse"), (dict(ge=FAKE + 1), EINVAL, "g_entropy"), (dict(dz=None), EINVAL, "dlogits"),
    (dict(dstride=4999), EINVAL, "overlap"), (dict(dz=FAKE + 2), EINVAL, "same view"), (dict(dz=FAKE, dstride=6000), EINVAL, "same view"),
])
def test_token_logp_backward_refusals(kw, status, word):
    st, msg = _call("nsp_token_logp_bwd", _logp_bwd(**kw))
    assert st == status and word in msg, msg


def test_calls_without_tokens_need_no_data():
    none = _rows(None, 0, 0)
    for name, a in (("nsp_rotary_fwd", _rotary(T=0, q=none, qo=none, k=none, ko=none, pos=None, freqs=None)),
                    ("nsp_norm_fwd", _norm_fwd(T=0, x=none, y=none, mean=None, rstd=None)),
                    ("nsp_norm_bwd", _norm_bwd(T=0, x=none, dy=none, dx=none, mean=None, rstd=None, dw=None, db=None, ws=None, ws_bytes=0)),
                    ("nsp_token_logp_fwd", _logp_fwd(T=0, z=None, y=None, lse=None, logp=None, tl=None, ti=None, ws=None, ws_bytes=0)),
                    ("nsp_token_logp_bwd", _logp_bwd(T=0, z=None, y=None, lse=None, ent=None, dz=None))):
        assert _call(name, a) == (nsp.NSP_OK, ""), name


def test_workspace_sizes():
    rng = np.random.default_rng(0)
    for _ in range(300):
        T, H, n = int(math.exp(rng.uniform(0, 14))), int(rng.integers(1, 40)), int(math.exp(rng.uniform(0, math.log(65536))))
        w = nsp.nsp_norm_bwd_workspace(T, H, n)
        assert 0 <= w <= 8192 * n + 1024 and w % 256 == 0
        V, top = int(math.exp(rng.uniform(0, 14))), int(rng.integers(0, 65))
        w = nsp.nsp_token_logp_workspace(T, V, top)
        assert 0 <= w <= 4 << 20 and w % 256 == 0
    assert nsp.nsp_norm_bwd_workspace(0, 4, 128) == 0 and nsp.nsp_norm_bwd_workspace(4, 4, 0) == 0 and nsp.nsp_norm_bwd_workspace(-1, 1, 8) == 0
    assert nsp.nsp_token_logp_workspace(1 << 20, 50000, 64) == 0 and nsp.nsp_token_logp_workspace(8, 0, 0) == 0
    assert nsp.nsp_token_logp_workspace(8, 50000, 65) == 0


def test_frequencies():
    """Each scaling by its definition; the interpolated by-parts and the base
    rule at the ends of their ranges."""
    r = 128
    f, s = nsp.nsp_rotary_frequencies(r, 1e6)
    i = np.arange(0, r, 2)
    assert np.allclose(f, 1e6 ** (-i / r), rtol=1e-14, atol=0) and s == 1.0
    g, s = nsp.nsp_rotary_frequencies(r, 1e6, nsp.NSP_ROTARY_LINEAR, 4.0)
    assert np.allclose(g, f / 4, rtol=1e-14, atol=0) and s == 1.0
    g, s = nsp.nsp_rotary_frequencies(r, 1e6, nsp.NSP_ROTARY_BASE, 8.0)
    assert g[0] == f[0] and g[-1] == pytest.approx(f[-1] / 8, rel=1e-12) and s == 1.0
    g, s = nsp.nsp_rotary_frequencies(r, 1e6, nsp.NSP_ROTARY_PARTS, 12.0, 32768, 1.0, 32.0)
    turns = 32768 * f / (2 * math.pi)
    assert np.array_equal(g[turns >= 32], f[turns >= 32]) and np.allclose(g[turns <= 1], f[turns <= 1] / 12, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 32)
    k = (turns[mid] - 1) / 31
    assert mid.any() and np.allclose(g[mid], f[mid] * (k + (1 - k) / 12), rtol=1e-13, atol=0)
    assert s == pytest.approx(0.1 * math.log(12) + 1, rel=2.0 ** -23)
    assert np.array_equal(nsp.nsp_rotary_frequencies(2, 1e4)[0], [1.0])


@pytest.mark.parametrize("a", [
    (0, 1e4), (3, 1e4), (1026, 1e4), (64, 0.0), (64, INF), (64, NAN), (64, 1e4, 4), (64, 1e4, 1, 0.5), (64, 1e4, 1, NAN), (2, 1e4, 2, 2.0),
    (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, 100.0, 3.0, 3.0), (64, 1e4, 3, 2.0, 100.0, -1.0, 3.0), (64, 1e4, 3, 2.0, 100.0, 1.0, INF)])
def test_frequency_refusals(a):
    with pytest.raises(nsp.NspError) as e:
        nsp.nsp_rotary_frequencies(*a)
    assert e.value.status == EINVAL


BF, F = torch.bfloat16, torch.float32


def _t(*shape, dtype=F):
    return torch.zeros(shape, dtype=dtype)


def _refuse(error, match, call, *a, **kw):
    with pytest.raises(error, match=match):
        call(*a, **kw)


def test_the_binding_refuses_what_it_cannot_describe():
    """Types, shapes, strides and places are checked before an address is
    taken; tensors on the host pass all of it but the last."""
    x, w, r = _t(4, 2, 64, dtype=BF), _t(64), _t(8)
    nf, nb, rf, lf, lb = nsp.nsp_norm_fwd, nsp.nsp_norm_bwd, nsp.nsp_rotary_fwd, nsp.nsp_token_logp_fwd, nsp.nsp_token_logp_bwd
    _refuse(TypeError, "on the GPU", nf, x, w, None, x, r, r)
    _refuse(TypeError, "x: a tensor", nf, None, w, None, x)
    _refuse(TypeError, "x: a tensor", nf, 3, w, None, x)
    _refuse(TypeError, r"x: \[tokens, n\]", nf, w, w, None, w)
    _refuse(TypeError, r"x: \[tokens, n\]", nf, _t(2, 2, 2, 2), w, None, x)
    _refuse(TypeError, "y: torch.bfloat16", nf, x, w, None, x.float())
    _refuse(TypeError, "y: .*is needed", nf, x, w, None, x[:3])
    _refuse(TypeError, "y: .*is needed", nf, x, w, None, x.view(8, 64))
    _refuse(ValueError, "y: .*contiguous", nf, x, w, None, _t(4, 64, 2, dtype=BF).transpose(1, 2))
    _refuse(TypeError, "weight: 64 contiguous", nf, x, _t(63), None, x)
    _refuse(TypeError, "weight: 64 contiguous", nf, x, _t(128)[::2], None, x)
    _refuse(TypeError, "bias: 64 contiguous elements of torch.float32", nf, x, w, w.to(BF), x)
    _refuse(TypeError, "weight: unsupported dtype", nf, x, w.half(), None, x)
    _refuse(TypeError, "x: unsupported dtype", nf, x.half(), None, None, x.half())
    _refuse(TypeError, "mean: 8 contiguous", nf, x, w, None, x, _t(7))
    _refuse(TypeError, "rstd: 8 contiguous", nf, x, w, None, x, None, _t(8, dtype=torch.float64))
    _refuse(TypeError, "misses 'y'", nf, x, w, None)
    _refuse(TypeError, "unexpected argument 'epsilon'", nf, x, w, None, x, epsilon=1.0)
    _refuse(TypeError, "'x' twice", nf, x, w, None, x, x=x)
    _refuse(TypeError, "at most", nf, *([x] * 10))
    _refuse(TypeError, None, nf, x, w, None, x, eps="a")
    _refuse(TypeError, "on the GPU", nb, x, w, x, r, r, x, w, None, _t(16, dtype=torch.uint8))
    _refuse(TypeError, "dy: .*is needed", nb, x, w, x[:, :1], r, r, x, w, None, None)
    _refuse(TypeError, "dbias: 64 contiguous", nb, x, w, x, r, r, x, w, _t(65), None)
    _refuse(TypeError, "workspace: contiguous", nb, x, w, x, r, r, x, w, None, _t(16)[::2])
    pos, fr = torch.zeros(4, dtype=torch.int64), _t(32, dtype=torch.float64)
    _refuse(TypeError, "on the GPU", rf, pos, fr, x, x, x, x)
    _refuse(TypeError, "q: .*head_dim", rf, pos, fr, x[0], x[0])
    _refuse(TypeError, "positions: 4 contiguous elements of torch.int64", rf, pos.int(), fr, x, x)
    _refuse(TypeError, "positions: 4", rf, pos[:3], fr, x, x)
    _refuse(TypeError, "freqs: .*float64", rf, pos, fr.float(), x, x)
    _refuse(TypeError, "k and k_out: both", rf, pos, fr, x, x, x)
    _refuse(TypeError, "k: .*is needed", rf, pos, fr, x, x, x[:3], x[:3])
    _refuse(TypeError, "k_out: .*is needed", rf, pos, fr, x, x, x, x[:, :1])
    _refuse(TypeError, "dk: .*is needed", nsp.nsp_rotary_bwd, pos, fr, x, x, x, x.float())
    z, y, v = _t(4, 90), torch.zeros(4, dtype=torch.int64), _t(4)
    _refuse(TypeError, "on the GPU", lf, z, y, v, v, v, _t(4, 3), torch.zeros(4, 3, dtype=torch.int64), None, scale=2)
    _refuse(TypeError, "tokens, vocab", lf, x, y, v, v)
    _refuse(TypeError, "lse: a tensor", lf, z, y, v, None)
    _refuse(TypeError, "targets: 4", lf, z, y.int(), v, v)
    _refuse(ValueError, "logits: .*contiguous", lf, _t(90, 4).t(), y, v, v)
    _refuse(TypeError, "top_logp and top_index", lf, z, y, v, v, v, _t(4, 3))
    _refuse(TypeError, "top_index: 12", lf, z, y, v, v, v, _t(4, 3), torch.zeros(4, 2, dtype=torch.int64))
    _refuse(TypeError, r"top_logp: \[tokens, top\]", lf, z, y, v, v, v, _t(3, 4), torch.zeros(4, 3, dtype=torch.int64))
    _refuse(TypeError, "dlogits: .*is needed", lb, z, y, v, z[:, :80])
    _refuse(TypeError, "g_logp: 4", lb, z, y, v, z, g_logp=_t(5))
    _refuse(TypeError, "on the GPU", lb, z, y, v, z, g_logp=v, g_entropy=v, entropy=v, g_lse=v, stream=0)
    m = torch.zeros(4, 90, device="meta")
    _refuse(TypeError, "on the GPU", lb, m, None, torch.zeros(4, device="meta"), m)


def test_calls_leave_no_references():
    """Refused calls neither keep nor lose references to what they were given."""
    import sys
    x, w = _t(4, 2, 64, dtype=BF), _t(64)
    before = [sys.getrefcount(t) for t in (x, w, BF, F)]
    for _ in range(1000):
        for a in ((x, w, None, x), (x, w, None, w), (x, x, None, x), (x, None, w, x, w)):
            with pytest.raises((TypeError, ValueError)):
                nsp.nsp_norm_fwd(*a)
    after = [sys.getrefcount(t) for t in (x, w, BF, F)]
    assert all(abs(a - b) < 100 for a, b in zip(after, before)), (before, after)
