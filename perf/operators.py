"""The row operators of a packed training or serving step around the
attention: rotary positions, norms of rows and the log probabilities of given
tokens, forward and backward, as the public entry points offer them and in
their plain form.

A case is one call:
  rotary  fwd / bwd   queries and keys [T, heads, dim] of one step, the
                      positions restarting at every packed sequence
                      (`batch` "packed") or one token a sequence ("decode");
                      `fused`: they are views of one projection's output
                      [T, hq + 2 hkv, dim] (bwd: the gradients are written
                      into such a tensor)
  norm    fwd / bwd   rows of n values: [T, n], or with `heads` the rows of
                      each head in such a projection's output
  logp    fwd / bwd   [T, vocab] logits in rows of `pad` more elements than
                      the vocabulary has; `top` alternatives; `masked`: the
                      share of the vocabulary that is masked by -inf;
                      a tenth of the targets is ignored (prompt, padding)
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LONGEST = 393216                      # tokens of the longest sequence of the workloads
LARGEST = {"rotary": 262144 * 36 * 128, "norm": 65536 * 8192, "logp": 8192 * 131072}   # elements


def _rotary(name, T, hq, hkv, dim, op="fwd", rot=None, layout="half", dtype="bf16", scaling="none", batch="packed", fused=True):
    return {"name": name, "kind": "rotary", "op": op, "T": T, "hq": hq, "hkv": hkv, "dim": dim, "rot": rot or dim, "layout": layout,
            "dtype": dtype, "scaling": scaling, "batch": batch, "fused": fused}


def _norm(name, T, n, op="fwd", center=False, heads=0, dtype="bf16", wtype="bf16"):
    return {"name": name, "kind": "norm", "op": op, "T": T, "n": n, "center": center, "heads": heads, "dtype": dtype, "wtype": wtype}


def _logp(name, T, vocab, op="fwd", top=0, dtype="bf16", scale=1.0, masked=0.0, pad=0):
    return {"name": name, "kind": "logp", "op": op, "T": T, "vocab": vocab, "top": top, "dtype": dtype, "scale": scale, "masked": masked,
            "pad": pad}


def listed():
    return [
        # a serving step: one new token of 24 sequences, far into long contexts
        _rotary("rotary_decode", 24, 32, 4, 128, scaling="parts", batch="decode"),
        # a small model with half of each head rotated, neighbours paired, in
        # float32, an odd number of tokens: the gradient
        _rotary("rotary_part_bwd_f32", 5003, 8, 2, 64, op="bwd", rot=32, layout="pairs", dtype="f32", scaling="linear", fused=False),
        # an ordinary share of short packed sequences, views of the projection
        _rotary("rotary_short", 65536, 32, 4, 128),
        # the largest: the long-tail share's tokens, the gradient
        _rotary("rotary_long_bwd", 262144, 32, 4, 128, op="bwd", scaling="parts"),
        # a serving step's hidden rows
        _norm("norm_decode", 24, 4096),
        # the norm of every query head of a share, in the projection's output
        _norm("norm_heads_bwd", 65536, 128, op="bwd", heads=32),
        # odd rows of an odd width, with mean and bias, in float32
        _norm("norm_odd_bwd_f32", 4999, 1111, op="bwd", center=True, dtype="f32", wtype="f32"),
        # the largest: wide hidden rows of a training step
        _norm("norm_wide_bwd", 65536, 8192, op="bwd", center=True),
        # a serving step: the sampled tokens with eight alternatives
        _logp("logp_decode_top8", 8, 131072, top=8, scale=1.25),
        # scoring of a ragged batch over an odd, partly masked vocabulary in
        # float32, with twenty alternatives
        _logp("logp_odd_top20_f32", 777, 50021, top=20, dtype="f32", masked=0.1),
        # the loss of a training step, forward, in rows padded to whole tiles
        _logp("logp_train", 4096, 151643, pad=293),
        # the largest: its gradient
        _logp("logp_train_bwd", 8192, 131072, op="bwd"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind, op = rng.choice(["rotary", "norm", "logp"]), rng.choice(["fwd", "bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    wide = 2 if dtype == "f32" else 1
    if kind == "rotary":
        hq, hkv, dim = rng.choice([(32, 4, 128), (32, 4, 128), (32, 8, 128), (16, 16, 128), (4, 1, 128), (8, 2, 64), (24, 8, 96), (12, 3, 80)])
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        c = _rotary("", _spread(rng, 1, LARGEST["rotary"] // (wide * (hq + hkv) * dim)), hq, hkv, dim, op, rot, rng.choice(["half", "half", "pairs"]),
                    dtype, rng.choice(["none", "linear", "parts"]), rng.choice(["packed", "packed", "decode"]), rng.random() < 0.6)
    elif kind == "norm":
        heads = rng.choice([0, 0, rng.choice([2, 4, 8, 32])])
        n = rng.choice([32, 64, 80, 128, 192]) if heads else _spread(rng, 16, 16384)
        if not heads and rng.random() < 0.6:
            n = max(16, n // 64 * 64)
        c = _norm("", _spread(rng, 1, min(262144, LARGEST["norm"] // (wide * n * max(1, heads + 2)))), n, op, rng.random() < 0.5, heads, dtype,
                  "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]))
    else:
        V, top = _spread(rng, 1000, 160000), 0 if op == "bwd" else rng.choice([0, 0, 1, 5, 8, 20, 64])
        wide *= 4 if top else 1       # alternatives are asked for in scoring and serving
        c = _logp("", _spread(rng, 1, min(16384, LARGEST["logp"] // (wide * V))), V, op, top, dtype, rng.choice([1.0, 1.0, 0.7, 1.25]), rng.choice([0.0, 0.0, 0.3]), rng.choice([0, 0, 5, 64]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

def _random(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dtype)


def _freqs(c):
    """The angle of one position, in radians, of every pair of a head."""
    f = 1e6 ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"])
    if c["scaling"] == "linear":      # the positions of a context four times as long
        f = f / 4.0
    elif c["scaling"] == "parts":     # only the slow pairs, from a context of 32768
        turns = 32768.0 * f / (2.0 * math.pi)
        fast = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (fast + (1.0 - fast) / 12.0)
    return f


def _amplitude(c):
    return 0.1 * math.log(12.0) + 1.0 if c["scaling"] == "parts" else 1.0


def _positions(c, seed):
    rng = np.random.default_rng(seed)
    if c["batch"] == "decode":
        return rng.integers(0, LONGEST, c["T"]).astype(np.int64)
    parts, left = [], c["T"]
    while left > 0:
        n = min(left, max(1, int(4096 * math.exp(rng.normal(0.0, 1.3)))))
        if len(parts) > 2000:
            n = left
        parts.append(np.arange(n, dtype=np.int64))
        left -= n
    return np.concatenate(parts)


def prepare(case, seed):
    c, g = case, _random(seed)
    T, dt = c["T"], TYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] == "rotary":
        hq, hkv, D = c["hq"], c["hkv"], c["dim"]
        s["freqs"] = torch.from_numpy(_freqs(c)).to(DEV)
        s["positions"] = torch.from_numpy(_positions(c, seed)).to(DEV)
        s["scale"] = _amplitude(c)
        whole = _normal(g, (T, hq + 2 * hkv, D), dt) if c["fused"] and c["op"] == "fwd" else torch.empty((T, hq + 2 * hkv, D), dtype=dt, device=DEV)
        parts = (whole[:, :hq], whole[:, hq:hq + hkv])

        def apart(make):
            return make((T, hq, D)), make((T, hkv, D))

        if c["fused"]:
            other = apart(lambda sh: torch.empty(sh, dtype=dt, device=DEV)) if c["op"] == "fwd" else apart(lambda sh: _normal(g, sh, dt))
            (s["q"], s["k"]), (s["q_out"], s["k_out"]) = (parts, other) if c["op"] == "fwd" else (other, parts)
        else:
            s["q"], s["k"] = apart(lambda sh: _normal(g, sh, dt))
            s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    elif c["kind"] == "norm":
        n, h, wt = c["n"], c["heads"], TYPES[c["wtype"]]
        # hidden rows: a spread and a middle of their own, a few wide channels
        shape = (T, h + 2, n) if h else (T, n)
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
        x *= 0.5 + 3.0 * torch.rand(shape[:-1] + (1,), generator=g, device=DEV)
        x += 0.5 * torch.randn(shape[:-1] + (1,), generator=g, device=DEV)
        x[..., ::97] *= 4.0
        x = x.to(dt)
        s["x"] = x[:, :h] if h else x
        s["w"] = (1.0 + _normal(g, (n,), torch.float32, 0.2)).to(wt)
        s["b"] = _normal(g, (n,), wt, 0.2) if c["center"] else None
        s["eps"] = 1e-6
        rows = T * max(1, h)
        out = tuple(s["x"].shape)
        if c["op"] == "fwd":
            s["y"] = torch.empty(out, dtype=dt, device=DEV)
            s["mean"] = torch.empty(rows, dtype=torch.float32, device=DEV) if c["center"] else None
            s["rstd"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        else:
            x64 = s["x"].double()
            mean = x64.mean(-1, keepdim=True) if c["center"] else 0.0
            var = (x64 - mean).square().mean(-1)
            s["mean"] = mean.float().reshape(-1) if c["center"] else None
            s["rstd"] = (var + s["eps"]).rsqrt().float().reshape(-1)
            del x64, var
            s["dy"] = _normal(g, out, dt)
            s["dx"] = torch.empty(out, dtype=dt, device=DEV)
            s["dw"] = torch.empty(n, dtype=wt, device=DEV)
            s["db"] = torch.empty(n, dtype=wt, device=DEV) if c["center"] else None
            # the most that any number of rows of this width asks for
            s["ws"] = torch.empty(8192 * n + 1024, dtype=torch.uint8, device=DEV)
    else:
        V = c["vocab"]
        z = torch.empty((T, V + c["pad"]), dtype=dt, device=DEV)
        for a in range(0, T, 1024):   # a model's logits: a middle, a spread, a few likely tokens
            e = min(T, a + 1024)
            y = torch.randn((e - a, V), generator=g, device=DEV, dtype=torch.float32)
            y = y * 2.5 - 1.0
            likely = torch.randint(0, V, (e - a, 4), generator=g, device=DEV)
            y.scatter_add_(1, likely, 6.0 + 5.0 * torch.rand((e - a, 4), generator=g, device=DEV))
            z[a:e, :V] = y.to(dt)
        del y
        if c["masked"]:
            gone = torch.rand(V, generator=g, device=DEV) < c["masked"]
            gone[0] = False
            z[:, :V].masked_fill_(gone[None, :], -math.inf)
        s["logits"] = z[:, :V]
        y = torch.randint(0, V, (T,), generator=g, device=DEV)
        if c["masked"]:
            y = torch.where(gone[y], torch.zeros_like(y), y)
        off = torch.rand(T, generator=g, device=DEV) < 0.1
        s["targets"] = torch.where(off, torch.full_like(y, -1), y)
        k = c["top"]
        f32 = {"dtype": torch.float32, "device": DEV}
        if c["op"] == "fwd":
            for name in ("logp", "lse", "entropy"):
                s[name] = torch.empty(T, **f32)
            s["top_logp"] = torch.empty((T, k), **f32) if k else None
            s["top_index"] = torch.empty((T, k), dtype=torch.int64, device=DEV) if k else None
            s["ws"] = torch.empty(4 << 20, dtype=torch.uint8, device=DEV)   # serves every number of rows
        else:
            s["lse"], s["entropy"] = torch.empty(T, **f32), torch.empty(T, **f32)
            for a in range(0, T, 1024):
                lp = s["logits"][a:a + 1024].double() * c["scale"]
                lse = torch.logsumexp(lp, 1)
                lp -= lse[:, None]
                s["lse"][a:a + 1024] = lse
                s["entropy"][a:a + 1024] = -(lp.exp() * lp.clamp_min(-1e30)).sum(1)
            s["g_logp"] = -torch.rand(T, generator=g, device=DEV) - 0.1
            s["g_entropy"] = 0.01 * torch.randn(T, generator=g, device=DEV)
            s["dlogits"] = torch.empty((T, V), dtype=dt, device=DEV)
    return s


# ------------------------------------------------- through the entry points --

def _run_own(s):
    from paper_2609_22755_amd import nsp
    c = s["case"]
    if c["kind"] == "rotary":
        call = nsp.nsp_rotary_fwd if c["op"] == "fwd" else nsp.nsp_rotary_bwd
        call(s["positions"], s["freqs"], s["q"], s["q_out"], s["k"], s["k_out"], scale=s["scale"],
             layout=nsp.NSP_ROTARY_HALF if c["layout"] == "half" else nsp.NSP_ROTARY_PAIRS)
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "norm":
        kind = nsp.NSP_NORM_LAYER if c["center"] else nsp.NSP_NORM_RMS
        if c["op"] == "fwd":
            nsp.nsp_norm_fwd(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], eps=s["eps"], kind=kind)
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        nsp.nsp_norm_bwd(s["x"], s["w"], s["dy"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["ws"], kind=kind)
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if c["op"] == "fwd":
        nsp.nsp_token_logp_fwd(s["logits"], s["targets"], s["logp"], s["lse"], s["entropy"], s["top_logp"], s["top_index"], s["ws"],
                               scale=c["scale"])
        return {n: s[n] for n in ("logp", "lse", "entropy", "top_logp", "top_index")}
    nsp.nsp_token_logp_bwd(s["logits"], s["targets"], s["lse"], s["dlogits"], g_logp=s["g_logp"], g_entropy=s["g_entropy"],
                           entropy=s["entropy"], scale=c["scale"])
    return {"dlogits": s["dlogits"]}


# -------------------------------------------------------------- plain forms --

def _turned(x, cos, sin, c):
    r, x = c["rot"], x.float()
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    y = torch.empty_like(x)
    p, q = a * cos - b * sin, b * cos + a * sin
    if c["layout"] == "half":
        y[..., :r // 2], y[..., r // 2:r] = p, q
    else:
        y[..., 0:r:2], y[..., 1:r:2] = p, q
    y[..., r:] = x[..., r:]
    return y.to(TYPES[c["dtype"]])


def _plain_rotary(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["freqs"][None, :]
    cos, sin = (s["scale"] * angle.cos()).float()[:, None], (s["scale"] * angle.sin()).float()[:, None]
    if c["op"] == "bwd":
        sin = -sin
    return {"q": _turned(s["q"], cos, sin, c), "k": _turned(s["k"], cos, sin, c)}


def _plain_norm(s):
    c, dt, wt = s["case"], TYPES[s["case"]["dtype"]], TYPES[s["case"]["wtype"]]
    x, w = s["x"].float(), s["w"].float()
    if c["op"] == "fwd":
        mean = x.mean(-1, keepdim=True) if c["center"] else None
        x = x - mean if c["center"] else x
        rstd = (x.square().mean(-1, keepdim=True) + s["eps"]).rsqrt()
        y = x * rstd * w
        y = y + s["b"].float() if c["center"] else y
        return {"y": y.to(dt), "mean": mean.reshape(-1) if c["center"] else None, "rstd": rstd.reshape(-1)}
    dy, rstd = s["dy"].float(), s["rstd"].reshape(x.shape[:-1] + (1,))
    xh = (x - s["mean"].reshape(rstd.shape)) * rstd if c["center"] else x * rstd
    h = dy * w
    dx = h - xh * (h * xh).mean(-1, keepdim=True)
    dx = dx - h.mean(-1, keepdim=True) if c["center"] else dx
    n = c["n"]
    dw = (dy * xh).reshape(-1, n).sum(0)
    db = dy.reshape(-1, n).sum(0).to(wt) if c["center"] else None
    return {"dx": (dx * rstd).to(dt), "dw": dw.to(wt), "db": db}


def _plain_logp(s):
    c, V = s["case"], s["case"]["vocab"]
    z = s["logits"].float() * c["scale"]
    y = s["targets"]
    given = y >= 0
    at = y.clamp_min(0)[:, None]
    if c["op"] == "fwd":
        top = z.amax(1, keepdim=True)
        e = (z - top).exp()
        lse = top + e.sum(1, keepdim=True).log()
        lp = z - lse
        entropy = -(lp.exp() * lp.clamp_min(-1e30)).sum(1)
        logp = torch.where(given, lp.gather(1, at)[:, 0], torch.zeros_like(entropy))
        out = {"logp": logp, "lse": lse[:, 0], "entropy": entropy, "top_logp": None, "top_index": None}
        if c["top"]:                  # by value, then the lowest index: one whole number orders both
            bits = (s["logits"].float() + 0.0).view(torch.int32).long()
            key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 31) + (V - torch.arange(V, device=z.device))[None, :]
            out["top_index"] = V - (key.topk(c["top"], 1).values & 0x7FFFFFFF)
            out["top_logp"] = lp.gather(1, out["top_index"])
        return out
    lp = z - s["lse"][:, None]
    p = lp.exp()
    gl = torch.where(given, s["g_logp"], torch.zeros_like(s["g_logp"]))[:, None]
    d = -p * (gl + s["g_entropy"][:, None] * (lp.clamp_min(-1e30) + s["entropy"][:, None]))
    d.scatter_add_(1, at, gl)
    return {"dlogits": (d * c["scale"]).to(TYPES[c["dtype"]])}


def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _plain_rotary, "norm": _plain_norm, "logp": _plain_logp}[s["case"]["kind"]](s)


# -------------------------------------------------------------------- work --

def work(case):
    """Every input read once, every output written once."""
    c, e = case, 4 if case["dtype"] == "f32" else 2
    T = c["T"]
    if c["kind"] == "rotary":
        x = T * (c["hq"] + c["hkv"])
        return {"bytes": 2 * e * x * c["dim"] + 8 * T + 4 * c["rot"], "flops": 3 * x * c["rot"]}
    if c["kind"] == "norm":
        rows = T * max(1, c["heads"])
        stats, w = rows * (8 if c["center"] else 4), c["n"] * (4 if c["wtype"] == "f32" else 2) * (2 if c["center"] else 1)
        if c["op"] == "fwd":
            return {"bytes": 2 * e * rows * c["n"] + stats + w, "flops": 7 * rows * c["n"]}
        return {"bytes": 3 * e * rows * c["n"] + stats + 2 * w, "flops": 13 * rows * c["n"]}
    if c["op"] == "fwd":
        return {"bytes": e * T * c["vocab"] + (20 + 12 * c["top"]) * T, "flops": 6 * T * c["vocab"]}
    return {"bytes": 2 * e * T * c["vocab"] + 24 * T, "flops": 8 * T * c["vocab"]}


# ------------------------------------------------------------------ exactly --

def _blocks(n, size):
    return [slice(a, min(n, a + size)) for a in range(0, n, size)]


def _exact_rotary(c, s):
    """A pair as a complex number, times the position's unit number."""
    unit = torch.polar(torch.full((1,), s["scale"], dtype=torch.float64, device=DEV), torch.zeros(1, dtype=torch.float64, device=DEV))
    r, sign = c["rot"], 1.0 if c["op"] == "fwd" else -1.0

    def one(x):
        out = torch.empty(x.shape, dtype=torch.float32 if c["dtype"] == "bf16" else torch.float64, device=DEV)
        for b in _blocks(c["T"], 16384):
            angle = sign * s["positions"][b].double()[:, None] * s["freqs"]
            z = x[b, :, :r].double()
            z = z.unflatten(-1, (2, r // 2)).transpose(-1, -2) if c["layout"] == "half" else z.unflatten(-1, (r // 2, 2))
            z = torch.view_as_complex(z.contiguous()) * (torch.polar(torch.ones_like(angle), angle) * unit)[:, None]
            z = torch.view_as_real(z)
            out[b, :, :r] = (z.transpose(-1, -2) if c["layout"] == "half" else z).flatten(-2).to(out.dtype)
            out[b, :, r:] = x[b, :, r:].to(out.dtype)
        return out

    return {"q": one(s["q"]), "k": one(s["k"])}


def _exact_norm(c, s):
    """The definition; its gradient by automatic differentiation."""
    n = c["n"]
    w = s["w"].double().requires_grad_(c["op"] == "bwd")
    bias = s["b"].double().requires_grad_(c["op"] == "bwd") if c["center"] else None
    shape = tuple(s["x"].shape)
    keep = torch.float32 if c["dtype"] == "bf16" else torch.float64
    first, stats = torch.empty(shape, dtype=keep, device=DEV), ([], [])
    for b in _blocks(c["T"], max(1, (1 << 26) // (n * max(1, c["heads"])))):
        x = s["x"][b].double().requires_grad_(c["op"] == "bwd")
        m = x.sum(-1, keepdim=True) / n if c["center"] else torch.zeros(x.shape[:-1] + (1,), dtype=torch.float64, device=DEV)
        v = ((x - m) ** 2).sum(-1, keepdim=True) / n
        y = (x - m) / torch.sqrt(v + s["eps"]) * w
        y = y + bias if c["center"] else y
        if c["op"] == "fwd":
            first[b] = y.to(keep)
            stats[0].append(m.reshape(-1))
            stats[1].append(1.0 / torch.sqrt(v + s["eps"]).reshape(-1))
        else:
            y.backward(s["dy"][b].double())
            first[b] = x.grad.to(keep)
    if c["op"] == "fwd":
        return {"y": first, "mean": torch.cat(stats[0]) if c["center"] else None, "rstd": torch.cat(stats[1])}
    return {"dx": first, "dw": w.grad, "db": bias.grad if c["center"] else None}


def _exact_logp(c, s):
    T, V, k = c["T"], c["vocab"], c["top"]
    out = {n: torch.empty(T, dtype=torch.float64, device=DEV) for n in ("logp", "lse", "entropy")}
    out.update(top_logp=torch.empty((T, k), dtype=torch.float64, device=DEV) if k else None, top_index=None)
    grad = torch.empty((T, V), dtype=torch.float32 if c["dtype"] == "bf16" else torch.float64, device=DEV) if c["op"] == "bwd" else None
    for b in _blocks(T, max(1, (1 << 26) // V)):
        z = s["logits"][b].double() * c["scale"]
        lse = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        entropy = torch.special.entr(p).sum(1)
        y = s["targets"][b]
        if c["op"] == "fwd":
            out["lse"][b], out["entropy"][b] = lse, entropy
            out["logp"][b] = torch.where(y < 0, torch.zeros_like(lse), z.gather(1, y.clamp_min(0)[:, None])[:, 0] - lse)
            if k:
                out["top_logp"][b] = z.sort(1, descending=True).values[:, :k] - lse[:, None]
            continue
        gl = torch.where(y < 0, 0.0, s["g_logp"][b].double())[:, None]
        d = gl * (torch.arange(V, device=DEV)[None, :] == y[:, None]) - gl * p
        d += s["g_entropy"][b].double()[:, None] * (torch.special.entr(p) - p * entropy[:, None])
        grad[b] = (d * c["scale"]).to(grad.dtype)
    return out if c["op"] == "fwd" else {"dlogits": grad}


def exact(case, seed):
    """In 64 bits from the definitions (kept in 32 where the output has 16)."""
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm": _exact_norm, "logp": _exact_logp}[case["kind"]](case, s)
