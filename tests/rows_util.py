"""Shared helpers of the row operators' GPU tests."""
import numpy as np

F32 = 2.0 ** -24                     # half a step of float32, relative


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def as64(t):
    return t.detach().double().cpu().numpy()


def draw(rng, shape, dtype, scale=1.0, shift=0.0):
    """A tensor of `dtype` on the GPU."""
    import torch
    x = torch.from_numpy((rng.standard_normal(shape) * scale + shift).astype(np.float32))
    return x.to(dtype).cuda()


def strided(t, lead, gap, token_gap=0):
    """A copy of [tokens, heads, n] (or [tokens, n]) as a view whose rows lie
    `gap` elements apart, tokens `token_gap` more, `lead` elements into a
    buffer of NaN: (view, buffer, mask of the buffer's elements outside)."""
    import torch
    sh = t.shape
    heads = sh[1] if t.dim() == 3 else 1
    hs = sh[-1] + gap
    ts = heads * hs + token_gap
    buf = torch.full((lead + max(1, sh[0]) * ts + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = torch.as_strided(buf, sh, (ts, hs, 1) if t.dim() == 3 else (ts, 1), lead)
    v.copy_(t)
    out = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    torch.as_strided(out, sh, v.stride(), lead).fill_(False)
    return v, buf, out


def untouched(buf, outside):
    return bool(buf[outside].isnan().all())


def within(name, got, want, tol):
    """|got - want| <= tol elementwise (all in float64); both may be infinite alike."""
    got, want, tol = np.broadcast_arrays(got, want, tol)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(want), np.isnan(got)), name
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), name
    off = np.abs(got[fine] - want[fine]) / np.maximum(tol[fine], 1e-300)
    worst = float(off.max()) if off.size else 0.0
    print(f"[rows] {name}: {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, (name, worst)
