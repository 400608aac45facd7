"""The row operators' calls (rotary positions, norms of rows, token log
probabilities) on torch tensors: the part of the binding that
``paper_2609_22755_amd.nsp`` offers under the same names.

Sizes, strides and types come from the tensors, which are checked here before
an address is taken: a wrong one raises TypeError or ValueError; what the C
ABI refuses raises NspError.  A call goes to the GPU that holds the tensors, by
default on its current stream.

A small call's time is this module's: every look at a tensor costs some 70 ns,
so each is made once, and rows are handed over as packed bytes.
"""
from __future__ import annotations

import struct

import torch

from . import nsp
from .nsp import NSP_BF16, NSP_F32, NSP_NORM_LAYER, NSP_ROTARY_HALF

_lib = nsp.load_library()
_CODES = {torch.bfloat16: NSP_BF16, torch.float32: NSP_F32}
_F32, _F64, _I64 = torch.float32, torch.float64, torch.int64
_pack = struct.Struct("@Pqq").pack           # nsp_rows


def _current_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


# (the raw handle alone, without a Stream object around it)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _code(dtype, name: str) -> int:
    c = _CODES.get(dtype)
    if c is None:
        raise TypeError(f"{name}: unsupported dtype {dtype} (bfloat16 or float32)")
    return c


def _elsewhere(t, dev: int, name: str):
    if dev < 0:
        raise TypeError(f"{name}: tensors must be on the GPU (got one on {t.device})")
    raise TypeError(f"{name}: a tensor on {t.device}, others on GPU {dev}")


def _device(t, name: str) -> int:
    dev = t.get_device()
    if dev < 0 or t.device.type != "cuda":
        _elsewhere(t, -1, name)
    return dev


def _rows(t, shape, dtype, dev: int, name: str) -> bytes:
    """A [tokens, n] or [tokens, heads, n] tensor as nsp_rows."""
    if t.dtype is not dtype or t.shape != shape:
        raise TypeError(f"{name}: {dtype} {tuple(shape)} is needed (got {t.dtype} {tuple(t.shape)})")
    if t.get_device() != dev:
        _elsewhere(t, dev, name)
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: a row's elements must be contiguous (strides {st})")
    return _pack(t.data_ptr(), st[0], st[1] if len(st) == 3 else 0)


def _array(t, n: int, dtype, dev: int, name: str):
    """The address of n contiguous elements; None for an argument left out."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name}: {n} contiguous elements of {dtype} are needed (got {t.dtype} {tuple(t.shape)}, strides {t.stride()})")
    if t.get_device() != dev:
        _elsewhere(t, dev, name)
    return t.data_ptr()


def _workspace(t, dev: int):
    if t is None:
        return None, 0
    if not t.is_contiguous():
        raise TypeError("workspace: contiguous memory is needed")
    if t.get_device() != dev:
        _elsewhere(t, dev, "workspace")
    return t.data_ptr(), t.numel() * t.element_size()


def _call(name: str, f, dev: int, stream, *args):
    """f(*args, stream) with the GPU `dev` current."""
    if stream is None:
        stream = _current_stream(dev)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    if dev == _current_device():
        st = f(*args, stream)
    else:
        with torch.cuda.device(dev):
            st = f(*args, stream)
    if st:
        nsp._check(st, name)


def _rotary(name, f, positions, freqs, q, q_out, k, k_out, names, scale, layout, stream):
    shape, dt = q.shape, q.dtype
    if len(shape) != 3:
        raise TypeError(f"{names[0]}: [tokens, heads, head_dim] is needed (got {tuple(shape)})")
    dev = _device(q, names[0])
    T, hq, D = shape
    half = freqs.numel()
    hk, kr, kor = 0, None, None
    if k is not None or k_out is not None:
        if k is None or k_out is None or k.dim() != 3:
            raise TypeError(f"{names[2]} and {names[3]}: [tokens, heads, head_dim] is needed of both")
        hk = k.shape[1]
        shape_k = (T, hk, D)
        kr, kor = _rows(k, shape_k, dt, dev, names[2]), _rows(k_out, shape_k, dt, dev, names[3])
        if hk == 0:
            kr = kor = None
    _call(name, f, dev, stream, layout, _code(dt, names[0]), T, D, 2 * half, _array(freqs, half, _F64, dev, "freqs"), scale,
          _array(positions, T, _I64, dev, "positions"), hq, _rows(q, shape, dt, dev, names[0]), _rows(q_out, shape, dt, dev, names[1]), hk, kr, kor)


def nsp_rotary_fwd(positions, freqs, q, q_out, k=None, k_out=None, scale: float = 1.0, layout: int = NSP_ROTARY_HALF, stream=None):
    """Rotate the query (and key) heads [tokens, heads, head_dim] by their
    positions (int64 [tokens]); freqs: float64 [rot_dim / 2] on the GPU, as
    nsp_rotary_frequencies gives them.  q_out may be q itself (in place)."""
    _rotary("nsp_rotary_fwd", _lib.nsp_rotary_fwd, positions, freqs, q, q_out, k, k_out, ("q", "q_out", "k", "k_out"), scale, layout, stream)


def nsp_rotary_bwd(positions, freqs, dq_out, dq, dk_out=None, dk=None, scale: float = 1.0, layout: int = NSP_ROTARY_HALF, stream=None):
    """Gradient of nsp_rotary_fwd: dq_out, dk_out into dq, dk (in place allowed)."""
    _rotary("nsp_rotary_bwd", _lib.nsp_rotary_bwd, positions, freqs, dq_out, dq, dk_out, dk, ("dq_out", "dq", "dk_out", "dk"), scale, layout, stream)


def _norm_sizes(shape):
    if len(shape) == 2:
        return shape[0], 1, shape[1]
    if len(shape) == 3:
        return shape
    raise TypeError(f"x: [tokens, n] or [tokens, heads, n] is needed (got {tuple(shape)})")


def nsp_norm_fwd(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-6, kind: int = NSP_NORM_LAYER, stream=None):
    """Norm of the rows of x ([tokens, n] or [tokens, heads, n]) into y (x
    itself: in place); weight, bias: [n] of one type, or None; mean, rstd:
    float32 [rows], for the backward, or None."""
    shape, dt = x.shape, x.dtype
    T, H, n = _norm_sizes(shape)
    dev = _device(x, "x")
    wd = weight.dtype if weight is not None else dt if bias is None else bias.dtype
    _call("nsp_norm_fwd", _lib.nsp_norm_fwd, dev, stream, kind, _code(dt, "x"), _code(wd, "weight"), T, H, n, _rows(x, shape, dt, dev, "x"),
          _array(weight, n, wd, dev, "weight"), _array(bias, n, wd, dev, "bias"), eps, _rows(y, shape, dt, dev, "y"),
          _array(mean, T * H, _F32, dev, "mean"), _array(rstd, T * H, _F32, dev, "rstd"))


def nsp_norm_bwd(x, weight, dy, mean, rstd, dx, dweight, dbias, workspace, kind: int = NSP_NORM_LAYER, stream=None):
    """Gradient of nsp_norm_fwd into dx, and dweight and dbias (of the
    weight's type; None: not computed)."""
    shape, dt = x.shape, x.dtype
    T, H, n = _norm_sizes(shape)
    dev = _device(x, "x")
    wt = weight if weight is not None else dweight if dweight is not None else dbias
    wd = dt if wt is None else wt.dtype
    _call("nsp_norm_bwd", _lib.nsp_norm_bwd, dev, stream, kind, _code(dt, "x"), _code(wd, "weight"), T, H, n, _rows(x, shape, dt, dev, "x"),
          _array(weight, n, wd, dev, "weight"), _rows(dy, shape, dt, dev, "dy"), _array(mean, T * H, _F32, dev, "mean"),
          _array(rstd, T * H, _F32, dev, "rstd"), _rows(dx, shape, dt, dev, "dx"), _array(dweight, n, wd, dev, "dweight"),
          _array(dbias, n, wd, dev, "dbias"), *_workspace(workspace, dev))


def _logits(t, shape, dtype, dev: int, name: str):
    """(address, row stride) of [tokens, vocab] rows."""
    if t.dtype is not dtype or t.shape != shape:
        raise TypeError(f"{name}: {dtype} {tuple(shape)} is needed (got {t.dtype} {tuple(t.shape)})")
    if t.get_device() != dev:
        _elsewhere(t, dev, name)
    st = t.stride()
    if st[1] != 1 and shape[1] > 1:
        raise ValueError(f"{name}: a row's elements must be contiguous (strides {st})")
    return t.data_ptr(), st[0]


def _vocabulary(logits):
    shape = logits.shape
    if len(shape) != 2:
        raise TypeError(f"logits: [tokens, vocab] is needed (got {tuple(shape)})")
    return shape, logits.dtype, _device(logits, "logits")


def nsp_token_logp_fwd(logits, targets, logp, lse, entropy=None, top_logp=None, top_index=None, workspace=None, scale: float = 1.0,
                       stream=None):
    """Log probabilities of the targets (int64 [tokens]; outside the vocabulary:
    ignored) under logits [tokens, vocab], with their log-sum-exp, entropy
    (float32 [tokens]) and the top alternatives ([tokens, top], float32 and
    int64).  Everything but logits and lse may be None."""
    shape, dt, dev = _vocabulary(logits)
    T, V = shape
    k = 0
    if top_logp is not None or top_index is not None:
        if top_logp is None or top_index is None or top_logp.dim() != 2:
            raise TypeError("top_logp and top_index: [tokens, top] is needed of both")
        k = top_logp.shape[1]
    _call("nsp_token_logp_fwd", _lib.nsp_token_logp_fwd, dev, stream, _code(dt, "logits"), T, V, *_logits(logits, shape, dt, dev, "logits"),
          _array(targets, T, _I64, dev, "targets"), scale, _array(logp, T, _F32, dev, "logp"), _array(lse, T, _F32, dev, "lse"),
          _array(entropy, T, _F32, dev, "entropy"), k, _array(top_logp, T * k, _F32, dev, "top_logp"),
          _array(top_index, T * k, _I64, dev, "top_index"), *_workspace(workspace, dev))


def nsp_token_logp_bwd(logits, targets, lse, dlogits, g_logp=None, g_entropy=None, entropy=None, g_lse=None, scale: float = 1.0,
                       stream=None):
    """Gradient of nsp_token_logp_fwd's logp, entropy and lse (float32
    [tokens] each, or None) with respect to the logits, into dlogits (the
    logits themselves: in place)."""
    shape, dt, dev = _vocabulary(logits)
    T, V = shape
    _call("nsp_token_logp_bwd", _lib.nsp_token_logp_bwd, dev, stream, _code(dt, "logits"), T, V, *_logits(logits, shape, dt, dev, "logits"),
          _array(targets, T, _I64, dev, "targets"), scale, _array(lse, T, _F32, dev, "lse"), _array(entropy, T, _F32, dev, "entropy"),
          _array(g_logp, T, _F32, dev, "g_logp"), _array(g_lse, T, _F32, dev, "g_lse"), _array(g_entropy, T, _F32, dev, "g_entropy"),
          *_logits(dlogits, shape, dt, dev, "dlogits"))
