"""Refusals of the vocabulary's operators, their workspace sizes and their
binding: host code, checked without a GPU (nothing is launched on any of the error
paths, and the addresses are never used)."""
import math
import sys

import numpy as np
import pytest
import torch

from paper_2609_22755_amd import nsp

FAKE, FAR = 0x10000, 1 << 44
EINVAL, EUNSUPPORTED, EWORKSPACE = nsp.NSP_EINVAL, nsp.NSP_EUNSUPPORTED, nsp.NSP_EWORKSPACE
BF, F = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _rows(data=FAKE, ts=64, hs=0):
    return bytes(nsp.CRows(data, ts, hs))


def _call(name, args):
    lib = nsp.load_library()
    st = getattr(lib, name)(*args.values())
    return st, lib.nsp_last_error().decode()


def _linear_fwd(**kw):
    a = dict(T=4, dim=64, V=500, x=_rows(FAKE), w=_rows(FAR), y=FAKE, scale=1.0, logp=FAKE, lse=FAKE, ent=FAKE, ws=FAKE, ws_bytes=1 << 40,
             stream=None)
    a.update(kw)
    return a


def _linear_bwd(**kw):
    a = dict(gdtype=0, T=4, dim=64, V=500, x=_rows(FAKE), w=_rows(FAR), y=FAKE, scale=1.0, lse=FAKE, ent=FAKE, gl=FAKE, gs=FAKE, ge=FAKE,
             dx=_rows(2 * FAR), dw=_rows(3 * FAR), ws=FAKE, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return a


def _distill_fwd(**kw):
    a = dict(dtype=0, T=4, V=5000, z=FAKE, stride=5000, top=3, index=FAKE, t=FAKE, kind=0, scale=1.0, loss=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 20,
             stream=None)
    a.update(kw)
    return a


def _distill_bwd(**kw):
    a = dict(dtype=0, T=4, V=5000, z=FAKE, stride=5000, top=3, index=FAKE, t=FAKE, kind=0, scale=1.0, lse=FAKE, g=FAKE, dz=FAR, dstride=5000,
             stream=None)
    a.update(kw)
    return a


def _embed_fwd(**kw):
    a = dict(wdtype=0, dtype=0, T=4, dim=64, V=500, ids=FAKE, w=_rows(FAR), scale=1.0, y=_rows(FAKE), stream=None)
    a.update(kw)
    return a


def _embed_bwd(**kw):
    a = dict(wdtype=0, dtype=0, T=4, dim=64, V=500, ids=FAKE, dy=_rows(FAKE), scale=1.0, dw=_rows(FAR), ws=FAKE, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return a


LINEAR = [
    (dict(T=-1), EINVAL, "n_tokens"), (dict(T=1 << 31), EINVAL, "n_tokens"), (dict(T=(1 << 22) + 1), EUNSUPPORTED, "n_tokens"),
    (dict(dim=0), EINVAL, "dim"), (dict(dim=60), EUNSUPPORTED, "dim"), (dict(dim=65544), EUNSUPPORTED, "dim"), (dict(V=0), EINVAL, "vocab"),
    (dict(V=(1 << 24) + 1), EUNSUPPORTED, "vocab"), (dict(scale=0.0), EINVAL, "scale"), (dict(scale=NAN), EINVAL, "scale"),
    (dict(scale=1e30), EINVAL, "scale"), (dict(x=None), EINVAL, "x is NULL"), (dict(x=_rows(None)), EINVAL, "x is NULL"),
    (dict(x=_rows(FAKE + 8)), EINVAL, "16-byte"), (dict(x=_rows(FAKE, 68)), EINVAL, "16 bytes"), (dict(x=_rows(FAKE, -64)), EINVAL, "strides"),
    (dict(x=_rows(FAKE, (1 << 20) + 8)), EUNSUPPORTED, "stride"), (dict(w=None), EINVAL, "w is NULL"), (dict(w=_rows(FAR + 2)), EINVAL, "16-byte"),
    (dict(w=_rows(FAR, 65)), EINVAL, "16 bytes"), (dict(w=_rows(FAR, 1 << 21)), EUNSUPPORTED, "stride"), (dict(y=None), EINVAL, "targets"),
    (dict(y=FAKE + 4), EINVAL, "targets"), (dict(lse=None), EINVAL, "lse"), (dict(lse=FAKE + 2), EINVAL, "lse"), (dict(ent=FAKE + 1), EINVAL, "entropy"),
    (dict(ws=None), EWORKSPACE, "workspace"), (dict(ws_bytes=100), EWORKSPACE, "workspace"), (dict(ws=FAKE + 128), EINVAL, "workspace"),
]


@pytest.mark.parametrize("kw,status,word", LINEAR + [(dict(logp=FAKE + 1), EINVAL, "logp")])
def test_linear_refusals(kw, status, word):
    st, msg = _call("nsp_linear_logp_fwd", _linear_fwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", LINEAR + [
    (dict(gdtype=2), EINVAL, "grad_dtype"), (dict(ent=None), EINVAL, "entropy"), (dict(gl=FAKE + 1), EINVAL, "g_logp"), (dict(gs=FAKE + 2), EINVAL, "g_lse"),
    (dict(ge=FAKE + 3), EINVAL, "g_entropy"), (dict(dx=_rows(None)), EINVAL, "dx"), (dict(dx=_rows(2 * FAR, 56)), EINVAL, "overlap"),
    (dict(dx=_rows(2 * FAR, 0)), EINVAL, "overlap"), (dict(dx=_rows(2 * FAR + 8)), EINVAL, "16-byte"), (dict(dx=_rows(2 * FAR, 68)), EINVAL, "16 bytes"),
    (dict(dw=_rows(3 * FAR, 63)), EINVAL, "overlap"), (dict(dx=_rows(FAKE)), EINVAL, "dx overlaps x"), (dict(dx=_rows(FAKE + 64 * 2 * 3)), EINVAL, "dx overlaps x"),
    (dict(dw=_rows(FAKE)), EINVAL, "dw overlaps x"), (dict(dw=_rows(FAR)), EINVAL, "dw overlaps w"), (dict(dx=_rows(FAR + 128)), EINVAL, "dx overlaps w"),
    (dict(dw=_rows(2 * FAR + 256)), EINVAL, "dw overlaps dx"),
])
def test_linear_backward_refusals(kw, status, word):
    st, msg = _call("nsp_linear_logp_bwd", _linear_bwd(**kw))
    assert st == status and word in msg, msg


DISTILL = [
    (dict(dtype=2), EINVAL, "dtype"), (dict(T=-1), EINVAL, "n_tokens"), (dict(V=0), EINVAL, "vocab"), (dict(V=(1 << 30) + 1), EUNSUPPORTED, "vocab"),
    (dict(scale=0.0), EINVAL, "scale"), (dict(scale=-1.0), EINVAL, "scale"), (dict(z=None), EINVAL, "logits"), (dict(z=FAKE + 1), EINVAL, "logits"),
    (dict(stride=-1), EINVAL, "stride"), (dict(top=0), EINVAL, "top"), (dict(top=257), EUNSUPPORTED, "top"), (dict(kind=2), EINVAL, "kind"),
    (dict(index=None), EINVAL, "index"), (dict(index=FAKE + 4), EINVAL, "index"), (dict(t=None), EINVAL, "teacher"), (dict(t=FAKE + 2), EINVAL, "teacher"),
    (dict(lse=None), EINVAL, "lse"),
]


@pytest.mark.parametrize("kw,status,word", DISTILL + [
    (dict(loss=FAKE + 2), EINVAL, "loss"), (dict(ws=None), EWORKSPACE, "workspace"), (dict(ws_bytes=1), EWORKSPACE, "workspace"),
    (dict(ws=FAKE + 16), EINVAL, "workspace")])
def test_distill_refusals(kw, status, word):
    st, msg = _call("nsp_distill_fwd", _distill_fwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", DISTILL + [
    (dict(g=None), EINVAL, "g_loss"), (dict(dz=None), EINVAL, "dlogits"), (dict(dstride=4999), EINVAL, "overlap"), (dict(dz=FAKE + 2), EINVAL, "same view"),
    (dict(dz=FAKE, dstride=6000), EINVAL, "same view")])
def test_distill_backward_refusals(kw, status, word):
    st, msg = _call("nsp_distill_bwd", _distill_bwd(**kw))
    assert st == status and word in msg, msg


EMBED = [
    (dict(wdtype=2), EINVAL, "w_dtype"), (dict(dtype=-1), EINVAL, "dtype"), (dict(T=-1), EINVAL, "n_tokens"), (dict(T=(1 << 26) + 1), EUNSUPPORTED, "n_tokens"),
    (dict(dim=0), EINVAL, "dim"), (dict(dim=(1 << 20) + 1), EUNSUPPORTED, "dim"), (dict(V=0), EINVAL, "vocab"), (dict(V=(1 << 30) + 1), EUNSUPPORTED, "vocab"),
    (dict(scale=INF), EINVAL, "scale"), (dict(scale=NAN), EINVAL, "scale"), (dict(ids=None), EINVAL, "tokens"), (dict(ids=FAKE + 4), EINVAL, "tokens"),
]


@pytest.mark.parametrize("kw,status,word", EMBED + [
    (dict(w=None), EINVAL, "w is NULL"), (dict(w=_rows(FAR + 1)), EINVAL, "w is"), (dict(w=_rows(FAR, -1)), EINVAL, "strides"), (dict(y=None), EINVAL, "y"),
    (dict(y=_rows(FAKE, 63)), EINVAL, "overlap"), (dict(y=_rows(FAR + 64)), EINVAL, "y overlaps w"), (dict(dtype=1, y=_rows(FAKE + 2)), EINVAL, "y is")])
def test_embedding_refusals(kw, status, word):
    st, msg = _call("nsp_embedding_fwd", _embed_fwd(**kw))
    assert st == status and word in msg, msg


@pytest.mark.parametrize("kw,status,word", EMBED + [
    (dict(dy=None), EINVAL, "dy"), (dict(dy=_rows(FAKE + 1)), EINVAL, "dy is"), (dict(dw=None), EINVAL, "dw"), (dict(dw=_rows(FAR, 60)), EINVAL, "overlap"),
    (dict(dw=_rows(FAKE + 2)), EINVAL, "dw overlaps dy"), (dict(ws=None), EWORKSPACE, "workspace"), (dict(ws_bytes=1), EWORKSPACE, "workspace"),
    (dict(ws=FAKE + 64), EINVAL, "workspace")])
def test_embedding_backward_refusals(kw, status, word):
    st, msg = _call("nsp_embedding_bwd", _embed_bwd(**kw))
    assert st == status and word in msg, msg


def test_calls_without_tokens_need_no_data():
    none = _rows(None, 0)
    for name, a in (("nsp_linear_logp_fwd", _linear_fwd(T=0, x=none, w=none, y=None, logp=None, lse=None, ent=None, ws=None, ws_bytes=0)),
                    ("nsp_linear_logp_bwd", _linear_bwd(T=0, x=none, w=none, y=None, lse=None, ent=None, gl=None, gs=None, ge=None, dx=none, dw=None,
                                                        ws=None, ws_bytes=0)),
                    ("nsp_linear_logp_bwd", _linear_bwd(dx=None, dw=None, ws=None, ws_bytes=0)),      # neither gradient: nothing to do
                    ("nsp_distill_fwd", _distill_fwd(T=0, z=None, index=None, t=None, loss=None, lse=None, ws=None, ws_bytes=0)),
                    ("nsp_distill_bwd", _distill_bwd(T=0, z=None, index=None, t=None, lse=None, g=None, dz=None)),
                    ("nsp_embedding_fwd", _embed_fwd(T=0, ids=None, w=none, y=none))):
        assert _call(name, a) == (nsp.NSP_OK, ""), name


def test_workspace_sizes():
    """Whole 256 bytes; what the documentation says of them; 0 for invalid sizes."""
    rng = np.random.default_rng(0)
    spread = lambda hi: int(math.exp(rng.uniform(0, math.log(hi))))       # noqa: E731
    for _ in range(300):
        T, dim, V = spread(1 << 22), 8 * spread(8192), spread(1 << 20)
        f, b = nsp.nsp_linear_logp_fwd_workspace(T, dim, V), nsp.nsp_linear_logp_bwd_workspace(T, dim, V)
        assert f % 256 == 0 and b % 256 == 0
        rows = min(T + 256, 32768)
        assert 0 < f <= 16 * rows * (V // 256 + 1) + 4 * rows + 512 + 256 * 256 * 256 * 4
        pieces = max(1 << 29, 8192 * (T + 256)) + 512 * (T + 256)
        sums = 4 * (T + 256) * dim + 256 * 256 * 256 * 4
        assert 0 < b <= 2 * (T + 256) * (dim + 64) + 28 * (T + 256) + pieces + 2 * sums + (1 << 20), (T, dim, V, b)
        d = nsp.nsp_distill_fwd_workspace(T, V)
        assert 0 <= d <= 520 << 10 and d % 256 == 0
        T, dim, V = spread(1 << 22), spread(1 << 14), spread(1 << 20)
        e = nsp.nsp_embedding_bwd_workspace(T, dim, V)
        assert e % 256 == 0 and 0 < e <= 16 * T + V + dim * T + 8 * dim + (2 << 20) + T
    for args in ((0, 64, 100), (-1, 64, 100), (4, 60, 100), (4, 64, 0), ((1 << 22) + 1, 64, 100), (4, 1 << 17, 100), (4, 64, 1 << 25)):
        assert nsp.nsp_linear_logp_fwd_workspace(*args) == 0 and nsp.nsp_linear_logp_bwd_workspace(*args) == 0, args
    assert nsp.nsp_distill_fwd_workspace(1 << 20, 50000) == 0 and nsp.nsp_distill_fwd_workspace(8, 0) == 0 and nsp.nsp_distill_fwd_workspace(-1, 9) == 0
    for args in ((0, 64, 100), (-1, 64, 100), (4, 0, 100), (4, 64, 0), ((1 << 26) + 1, 64, 100)):
        assert nsp.nsp_embedding_bwd_workspace(*args) == 0, args


def _t(*shape, dtype=F):
    return torch.zeros(shape, dtype=dtype)


def _refuse(error, match, call, *a, **kw):
    with pytest.raises(error, match=match):
        call(*a, **kw)


def test_the_binding_refuses_what_it_cannot_describe():
    """Types, shapes, strides and places are checked before an address is taken;
    tensors on the host pass all of it but the last."""
    x, w, y, v = _t(4, 64, dtype=BF), _t(90, 64, dtype=BF), torch.zeros(4, dtype=torch.int64), _t(4)
    ff, fb = nsp.nsp_linear_logp_fwd, nsp.nsp_linear_logp_bwd
    _refuse(TypeError, "on the GPU", ff, x, w, y, v, v, v, _t(16, dtype=torch.uint8), scale=2)
    _refuse(TypeError, "x: .*bfloat16", ff, x.float(), w, y, v, v)
    _refuse(TypeError, "weight: .*bfloat16", ff, x, w.float(), y, v, v)
    _refuse(TypeError, r"x: \[tokens, dim\]", ff, w[0], w, y, v, v)
    _refuse(TypeError, r"weight: \[vocab, 64\]", ff, x, w[:, :60], y, v, v)
    _refuse(ValueError, "weight: .*contiguous", ff, x, _t(64, 90, dtype=BF).t(), y, v, v)
    _refuse(TypeError, "targets: 4", ff, x, w, y.int(), v, v)
    _refuse(TypeError, "lse: a tensor", ff, x, w, y, v, None)
    _refuse(TypeError, "entropy: 4", ff, x, w, y, v, v, _t(5))
    _refuse(TypeError, "misses 'lse'", ff, x, w, y, v)
    _refuse(TypeError, "on the GPU", fb, x, w, y, v, x, w, None, g_logp=v, g_entropy=v, entropy=v, g_lse=v, scale=1.0, stream=0)
    _refuse(TypeError, "dweight: torch.bfloat16", fb, x, w, y, v, x, w.float(), None)
    _refuse(TypeError, "dx: .*is needed", fb, x, w, y, v, x[:3], None, None)
    _refuse(TypeError, "dx: unsupported dtype", fb, x, w, y, v, x.half(), None, None)
    _refuse(TypeError, "g_lse: 4", fb, x, w, y, v, x, w, None, g_lse=_t(3))
    z, i, t = _t(4, 90), torch.zeros(4, 3, dtype=torch.int64), _t(4, 3)
    df, db = nsp.nsp_distill_fwd, nsp.nsp_distill_bwd
    _refuse(TypeError, "on the GPU", df, z, i, t, v, v)
    _refuse(TypeError, r"index: \[tokens, top\]", df, z, i[0], t, v, v)
    _refuse(TypeError, r"index: \[4, top\]", df, z, i[:3], t, v, v)
    _refuse(TypeError, "index: 12 contiguous elements of torch.int64", df, z, i.int(), t, v, v)
    _refuse(TypeError, "teacher_logp: 12", df, z, i, t[:, :2], v, v)
    _refuse(TypeError, "teacher_logp: a tensor", df, z, i, None, v, v)
    _refuse(TypeError, "logits: unsupported dtype", df, z.half(), i, t, v, v)
    _refuse(ValueError, "kind", df, z, i, t, v, v, kind=1 << 32)
    _refuse(TypeError, "g_loss: a tensor", db, z, i, t, v, None, z)
    _refuse(TypeError, "dlogits: .*is needed", db, z, i, t, v, v, z[:, :80])
    _refuse(TypeError, "on the GPU", db, z, i, t, v, v, z, kind=1, scale=0.5, stream=0)
    ef, eb = nsp.nsp_embedding_fwd, nsp.nsp_embedding_bwd
    _refuse(TypeError, "on the GPU", ef, y, w, _t(4, 64), 2.0)
    _refuse(TypeError, "tokens: 4", ef, y[:3], w, x)
    _refuse(TypeError, "tokens: a tensor", ef, None, w, x)
    _refuse(TypeError, r"weight: \[vocab, 60\]", ef, y, w, x[:, :60])
    _refuse(TypeError, r"y: \[tokens, dim\]", ef, y, w, x[0])
    _refuse(TypeError, "weight: unsupported dtype", ef, y, w.half(), x)
    _refuse(TypeError, "on the GPU", eb, y, x, w, None)
    _refuse(TypeError, r"dweight: \[vocab, 64\]", eb, y, x, w[:, :32], None)
    _refuse(TypeError, "workspace: contiguous", eb, y, x, w, _t(16)[::2])


def test_calls_leave_no_references():
    x, w, y, v = _t(4, 64, dtype=BF), _t(90, 64, dtype=BF), torch.zeros(4, dtype=torch.int64), _t(4)
    before = [sys.getrefcount(t) for t in (x, w, y, v, BF)]
    for _ in range(1000):
        for call, a in ((nsp.nsp_linear_logp_fwd, (x, w, y, v, v)), (nsp.nsp_linear_logp_bwd, (x, w, y, v, x, x, None)),
                        (nsp.nsp_embedding_bwd, (y, x, w, None)), (nsp.nsp_distill_fwd, (x, y, v, v, v))):
            with pytest.raises((TypeError, ValueError)):
                call(*a)
    after = [sys.getrefcount(t) for t in (x, w, y, v, BF)]
    assert all(abs(a - b) < 100 for a, b in zip(after, before)), (before, after)
