"""The row operators as a packed step uses them, around the attention.

Training: norm, projection, norm of the heads where they lie in its output,
rotation by the packed positions, Ulysses pack, attention, unpack, output
projection, norm, logits, token log probabilities with their entropy, and all
of it backward; against the same step in float64 with automatic
differentiation.  Serving: the last token of every sequence, one row each.

Tolerance of the whole step, relative 2-norm: q, k, v, O and dO are rounded to
bf16 (2^-8 each at most: 5 x 0.4%), the attention may be off by its own 0.5%
forward and 1% backward, and the row operators' float32 roundings are far below:
3.5% in all, 4% allowed.  Rows of the loss depend on O alone: 2.5%."""
import math

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2609_22755_amd import nsp
from paper_2609_22755_amd.workloads import small_worklist

from gpu_util import require_gpu
from rows_util import as64

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
HQ, HK, D, HIDDEN, V, EPS = 8, 2, 64, 96, 517, 1e-5
LENGTHS = [70, 1, 130, 33]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _weights(rng):
    w = {"in": (HIDDEN, (HQ + 2 * HK) * D), "out": (HQ * D, HIDDEN), "head": (HIDDEN, V)}
    w = {k: (rng.standard_normal(s) / math.sqrt(s[0])).astype(np.float32) for k, s in w.items()}
    for k, n in (("n1", HIDDEN), ("nq", D), ("nk", D), ("n2", HIDDEN)):
        w[k] = (1 + 0.2 * rng.standard_normal(n)).astype(np.float32)
    w["b2"] = (0.1 * rng.standard_normal(HIDDEN)).astype(np.float32)
    return w


def _reference(x, w, pos, freqs, scale, targets, g_logp, g_ent):
    """The step in float64 on the CPU; gradients of x and of every weight."""
    t = {k: torch.from_numpy(v).double().requires_grad_(True) for k, v in w.items()}
    x = torch.from_numpy(x).double().requires_grad_(True)

    def rms(v, g):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * g

    T = x.shape[0]
    qkv = (rms(x, t["n1"]) @ t["in"]).view(T, HQ + 2 * HK, D)
    q, k, v = rms(qkv[:, :HQ], t["nq"]), rms(qkv[:, HQ:HQ + HK], t["nk"]), qkv[:, HQ + HK:]
    a = torch.from_numpy(pos).double()[:, None, None] * torch.from_numpy(freqs)
    c, s = scale * a.cos(), scale * a.sin()

    def turn(z):
        z1, z2 = z[..., :D // 2], z[..., D // 2:]
        return torch.cat((z1 * c - z2 * s, z2 * c + z1 * s), -1)

    q, k = turn(q), turn(k)
    outs, at = [], 0
    for n in LENGTHS:
        qi, ki, vi = q[at:at + n].transpose(0, 1), k[at:at + n].transpose(0, 1), v[at:at + n].transpose(0, 1)
        ki, vi = ki.repeat_interleave(HQ // HK, 0), vi.repeat_interleave(HQ // HK, 0)
        z = (qi @ ki.transpose(1, 2)) / math.sqrt(D)
        z = z.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
        outs.append((z.softmax(-1) @ vi).transpose(0, 1))
        at += n
    y = x + torch.cat(outs).reshape(T, HQ * D) @ t["out"]
    h = torch.nn.functional.layer_norm(y, (HIDDEN,), t["n2"], t["b2"], EPS)
    lp = torch.log_softmax(h @ t["head"], -1)
    tg = torch.from_numpy(targets)
    logp = torch.where(tg >= 0, lp.gather(1, tg.clamp_min(0)[:, None])[:, 0], torch.zeros(T, dtype=torch.float64))
    ent = -(lp.exp() * lp).sum(-1)
    ((logp * g_logp).sum() + (ent * g_ent).sum()).backward()
    return logp.detach(), ent.detach(), x.grad, {k: v.grad for k, v in t.items()}


def test_training_step():
    rng = np.random.default_rng(31)
    wl = small_worklist(LENGTHS, HQ, HK, D)
    T = int(wl.lengths.sum())
    w, x = _weights(rng), rng.standard_normal((T, HIDDEN)).astype(np.float32)
    pos = wl.positions()
    assert np.array_equal(pos, np.concatenate([np.arange(n) for n in LENGTHS]))
    freqs, amp = nsp.nsp_rotary_frequencies(D, 1e4, nsp.NSP_ROTARY_PARTS, 4.0, 64.0, 1.0, 8.0)
    targets = rng.integers(0, V, T)
    targets[np.cumsum(LENGTHS) - 1] = -1                       # the last token of a sequence has none
    g_logp, g_ent = torch.full((T,), -1.0 / T, dtype=torch.float64), torch.full((T,), 0.02 / T, dtype=torch.float64)
    ref_logp, ref_ent, ref_dx, ref_dw = _reference(x, w, pos, freqs, amp, targets, g_logp, g_ent)

    def e(*shape, dtype=F):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def ws(tokens, heads, n):
        return e(nsp.nsp_norm_bwd_workspace(tokens, heads, n), dtype=torch.uint8)

    W = {k: torch.from_numpy(v).cuda() for k, v in w.items()}
    X, P, FR = torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda(), torch.from_numpy(freqs).cuda()
    Y = torch.from_numpy(targets).cuda()
    sc = 1.0 / math.sqrt(D)
    # ---- forward
    h1, r1 = e(T, HIDDEN), e(T)
    nsp.nsp_norm_fwd(X, W["n1"], None, h1, None, r1, eps=EPS, kind=nsp.NSP_NORM_RMS)
    qkv = (h1 @ W["in"]).to(BF).view(T, HQ + 2 * HK, D)
    qv, kv = qkv[:, :HQ], qkv[:, HQ:HQ + HK]
    q, k, rq, rk = e(T, HQ, D, dtype=BF), e(T, HK, D, dtype=BF), e(T * HQ), e(T * HK)
    nsp.nsp_norm_fwd(qv, W["nq"], None, q, None, rq, eps=EPS, kind=nsp.NSP_NORM_RMS)
    nsp.nsp_norm_fwd(kv, W["nk"], None, k, None, rk, eps=EPS, kind=nsp.NSP_NORM_RMS)
    nsp.nsp_rotary_fwd(P, FR, q, q, k, k, scale=amp)           # in place
    head = {n: e(wl.q_elems() if n in ("q", "do") else wl.kv_elems(), dtype=BF) for n in ("q", "k", "v", "do")}
    for n, t in (("q", q), ("k", k), ("v", qkv[:, HQ + HK:].contiguous())):
        nsp.nsp_ulysses_pack(wl, nsp.NSP_KIND_Q if n == "q" else nsp.NSP_KIND_KV, t, head[n])
    buf = nsp.alloc_like_worklist(wl)
    nsp.nsp_varlen_attn_fwd(wl, head["q"], head["k"], head["v"], buf["o"], buf["lse"], sc)
    o = e(T, HQ * D, dtype=BF)
    nsp.nsp_ulysses_unpack(wl, nsp.NSP_KIND_Q, nsp.NSP_UNPACK_SELECT, buf["o"], o)
    y = X + o.float() @ W["out"]
    h2, m2, r2 = e(T, HIDDEN), e(T), e(T)
    nsp.nsp_norm_fwd(y, W["n2"], W["b2"], h2, m2, r2, eps=EPS)
    logits = h2 @ W["head"]
    logp, lse, ent = e(T), e(T), e(T)
    lws = e(nsp.nsp_token_logp_workspace(T, V), dtype=torch.uint8)
    nsp.nsp_token_logp_fwd(logits, Y, logp, lse, ent, workspace=lws)
    # ---- backward
    dz = logits                                                # in place
    nsp.nsp_token_logp_bwd(logits, Y, lse, dz, g_logp=g_logp.float().cuda(), g_entropy=g_ent.float().cuda(), entropy=ent)
    G = {"head": h2.t() @ dz}
    dh2 = dz @ W["head"].t()
    dy = e(T, HIDDEN)
    G["n2"], G["b2"] = e(HIDDEN), e(HIDDEN)
    nsp.nsp_norm_bwd(y, W["n2"], dh2, m2, r2, dy, G["n2"], G["b2"], ws(T, 1, HIDDEN))
    G["out"] = o.float().t() @ dy
    do = (dy @ W["out"].t()).to(BF)
    nsp.nsp_ulysses_pack(wl, nsp.NSP_KIND_Q, do, head["do"])
    nsp.nsp_varlen_attn_bwd(wl, head["q"], head["k"], head["v"], buf["o"], head["do"], buf["lse"], buf["dq"], buf["dk"], buf["dv"], buf["ws"], sc)
    dq, dk, dv = e(T, HQ, D, dtype=BF), e(T, HK, D, dtype=BF), e(T, HK, D, dtype=BF)
    nsp.nsp_ulysses_unpack(wl, nsp.NSP_KIND_Q, nsp.NSP_UNPACK_SELECT, buf["dq"], dq)
    nsp.nsp_ulysses_unpack(wl, nsp.NSP_KIND_KV, nsp.NSP_UNPACK_SUM, buf["dk"], dk)
    nsp.nsp_ulysses_unpack(wl, nsp.NSP_KIND_KV, nsp.NSP_UNPACK_SUM, buf["dv"], dv)
    nsp.nsp_rotary_bwd(P, FR, dq, dq, dk, dk, scale=amp)       # in place
    dqkv = e(T, HQ + 2 * HK, D, dtype=BF)
    G["nq"], G["nk"] = e(D), e(D)
    nsp.nsp_norm_bwd(qv, W["nq"], dq, None, rq, dqkv[:, :HQ], G["nq"], None, ws(T, HQ, D), kind=nsp.NSP_NORM_RMS)
    nsp.nsp_norm_bwd(kv, W["nk"], dk, None, rk, dqkv[:, HQ:HQ + HK], G["nk"], None, ws(T, HK, D), kind=nsp.NSP_NORM_RMS)
    dqkv[:, HQ + HK:] = dv
    d = dqkv.view(T, -1).float()
    G["in"] = h1.t() @ d
    dx, G["n1"] = e(T, HIDDEN), e(HIDDEN)
    nsp.nsp_norm_bwd(X, W["n1"], d @ W["in"].t(), None, r1, dx, G["n1"], None, ws(T, 1, HIDDEN), kind=nsp.NSP_NORM_RMS)
    dx += dy
    torch.cuda.synchronize()

    def off(a, b):
        b = b.numpy() if isinstance(b, torch.Tensor) else b
        return float(np.linalg.norm(as64(a) - b) / np.linalg.norm(b))

    errs = {"logp": off(logp, ref_logp), "entropy": off(ent, ref_ent)}
    grads = {"dx": off(dx, ref_dx), **{k: off(G[k], ref_dw[k]) for k in G}}
    print("[step] " + ", ".join(f"{k} {v:.2e}" for k, v in {**errs, **grads}.items()), flush=True)
    assert all(v <= 2.5e-2 for v in errs.values()) and all(v <= 4e-2 for v in grads.values()), (errs, grads)


def test_serving_step_of_single_tokens():
    """Three sequences' next tokens, far apart: the same rows as in one long
    packed call, bit for bit where no sum depends on the number of rows."""
    rng = np.random.default_rng(32)
    T, pos = 3, torch.tensor([393215, 0, 77], device="cuda")
    freqs = torch.from_numpy(nsp.nsp_rotary_frequencies(128, 1e6)[0]).cuda()
    qkv = torch.from_numpy(rng.standard_normal((T, 40, 128)).astype(np.float32)).to(BF).cuda()
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(128)).astype(np.float32)).cuda()

    def heads(x, p):
        q, k = torch.empty(len(p), 32, 128, dtype=BF, device="cuda"), torch.empty(len(p), 4, 128, dtype=BF, device="cuda")
        nsp.nsp_norm_fwd(x[:, :32], w, None, q, kind=nsp.NSP_NORM_RMS)
        nsp.nsp_norm_fwd(x[:, 32:36], w, None, k, kind=nsp.NSP_NORM_RMS)
        nsp.nsp_rotary_fwd(p, freqs, q, q, k, k)
        return q, k

    one = heads(qkv, pos)
    many = heads(qkv.repeat(700, 1, 1), pos.repeat(700))
    logits = torch.from_numpy((3 * rng.standard_normal((T, 32000))).astype(np.float32)).to(BF).cuda()
    lse, lp, ti = torch.empty(T, device="cuda"), torch.empty(T, 5, device="cuda"), torch.empty(T, 5, dtype=torch.int64, device="cuda")
    ws = torch.empty(nsp.nsp_token_logp_workspace(T, 32000, 5), dtype=torch.uint8, device="cuda")
    nsp.nsp_token_logp_fwd(logits, None, None, lse, None, lp, ti, ws, scale=1.5)
    torch.cuda.synchronize()
    for a, b in zip(one, many):
        assert all(torch.equal(a, b[i * T:(i + 1) * T]) for i in (0, 350, 699))
    want = R.token_logp(as64(logits), [-1] * T, 1.5, 5)
    assert np.array_equal(ti.cpu().numpy(), want["top_index"])


def test_two_streams_at_once():
    """The same calls on two streams at a time, each with its own outputs and
    workspace, give what one alone gives."""
    rng = np.random.default_rng(33)
    x, g = (torch.from_numpy(rng.standard_normal((20000, 256)).astype(np.float32)).to(BF).cuda() for _ in range(2))
    z = torch.from_numpy(rng.standard_normal((30, 60000)).astype(np.float32)).cuda()
    y = torch.from_numpy(rng.integers(0, 60000, 30)).cuda()

    def outputs():
        f = dict(device="cuda")
        return dict(y=torch.empty_like(x), mean=torch.empty(20000, **f), rstd=torch.empty(20000, **f), dx=torch.empty_like(x),
                    dw=torch.empty(256, dtype=BF, **f), db=torch.empty(256, dtype=BF, **f),
                    ws=torch.empty(nsp.nsp_norm_bwd_workspace(20000, 1, 256), dtype=torch.uint8, **f), logp=torch.empty(30, **f),
                    lse=torch.empty(30, **f), tl=torch.empty(30, 9, **f), ti=torch.empty(30, 9, dtype=torch.int64, **f),
                    ws2=torch.empty(nsp.nsp_token_logp_workspace(30, 60000, 9), dtype=torch.uint8, **f))

    def calls(o, stream=None):
        nsp.nsp_norm_fwd(x, None, None, o["y"], o["mean"], o["rstd"], stream=stream)
        nsp.nsp_norm_bwd(x, None, g, o["mean"], o["rstd"], o["dx"], o["dw"], o["db"], o["ws"], stream=stream)
        nsp.nsp_token_logp_fwd(z, y, o["logp"], o["lse"], None, o["tl"], o["ti"], o["ws2"], stream=stream)

    sets, streams = [outputs() for _ in range(3)], [torch.cuda.Stream() for _ in range(2)]
    calls(sets[0])
    torch.cuda.synchronize()
    for _ in range(5):
        for o, s in zip(sets[1:], streams):
            calls(o, s)
    torch.cuda.synchronize()
    for o in sets[1:]:
        assert all(torch.equal(o[n], sets[0][n]) for n in o if not n.startswith("ws"))


def test_kernel_times_are_reported():
    x = torch.randn(100, 64, device="cuda")
    nsp.nsp_timing_reset()
    nsp.nsp_timing_enable(True)
    nsp.nsp_norm_fwd(x, None, None, torch.empty_like(x))
    lse = torch.empty(100, device="cuda")
    nsp.nsp_token_logp_fwd(x, None, None, lse)
    nsp.nsp_timing_enable(False)
    got = {n: nsp.nsp_timing_query(n) for n in nsp.ROW_KERNELS}
    nsp.nsp_timing_reset()
    assert got["norm_fwd"][0] == 1 and got["token_logp_fwd"][0] == 1 and got["norm_fwd"][1] > 0
    assert got["rotary"][0] == got["norm_bwd"][0] == got["token_logp_bwd"][0] == 0
