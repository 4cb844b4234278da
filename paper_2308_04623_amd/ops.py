"""Operators for training a draft on its oracle (include/ssd_ops.h) on torch
tensors: attention of a batch over a shared prompt, distillation from top
logits, embedding rows and their table's gradient.

As in ssd.py, the library does the work and PyTorch supplies device memory
and streams.  Outputs and scratch come from torch's allocator on the stream of
the call (the current one, or `stream`), so calls may run on any streams that
are ordered with the tensors' own use.  Every function takes its outputs from
the caller where `out` is given.  Arguments are checked, here for what a pointer
no longer tells (devices, types, shapes) and in the library for the rest.

Nothing here is recorded for autograd: results are plain tensors whatever their
inputs' requires_grad, and the gradients are the functions that say so
(distill_backward, distill_step, embed_grad).  prefix_attention has none.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import operator
from typing import Optional

import torch

from . import ssd
from .ssd import SSDError

# every function include/ssd_ops.h declares
EXPORTS = ("ssd_prefix_attn_workspace", "ssd_prefix_attn", "ssd_distill_forward", "ssd_distill_backward",
           "ssd_distill_step", "ssd_embed", "ssd_embed_grad_workspace", "ssd_embed_grad")

_DTYPES = {torch.float32: ssd.F32, torch.bfloat16: ssd.BF16}


class _PrefixAttnDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_seq", C.c_int32), ("n_query", C.c_int32), ("n_head", C.c_int32),
                ("n_kv_head", C.c_int32), ("head_dim", C.c_int32), ("prefix_len", C.c_int32),
                ("own_rows", C.c_int32), ("scale", C.c_float)] + \
               [(n, C.c_int64) for n in ("q_seq", "q_row", "q_head", "out_seq", "out_row", "out_head", "prefix_head",
                                         "prefix_row", "own_seq", "own_head", "own_row")]


_KINDS = (torch.float32, torch.bfloat16)
_lib = None


def _ops():
    global _lib
    if _lib is None:
        L = ssd.lib()
        i32, i64, f32, vp, sz = C.c_int32, C.c_int64, C.c_float, C.c_void_p, C.c_size_t
        logits = [i32, vp, i64, i32, i32, vp, vp, i32]
        sig = {
            "ssd_prefix_attn_workspace": [C.POINTER(_PrefixAttnDesc), C.POINTER(sz)],
            "ssd_prefix_attn": [C.POINTER(_PrefixAttnDesc)] + [vp] * 9 + [sz, vp],
            "ssd_distill_forward": logits + [vp, f32, vp, vp, vp],
            "ssd_distill_backward": logits + [vp, vp, f32, vp, i64, vp],
            "ssd_distill_step": logits + [vp, f32, vp, vp, vp, i64, vp],
            "ssd_embed": [i32, i32, vp, i32, vp, i64, i32, i32, f32, vp, i64, vp],
            "ssd_embed_grad_workspace": [i32, i32, i32, C.POINTER(sz)],
            "ssd_embed_grad": [i32, i32, vp, i32, vp, i64, i32, i32, f32, i32, vp, i64, vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = C.c_int
        _lib = L
    return _lib


def _refuse(what: str, why: str, status: int = ssd.E_INVALID_ARG):
    raise SSDError(status, what, why)


def _check(status: int, what: str):
    if status != ssd.OK:
        raise SSDError(status, what, _lib.ssd_last_error().decode())


def _tensor(what, name, t, dtypes, dims, like=None):
    """t is a device tensor of one of the dtypes with `dims` dimensions, on like's device."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.dim() == dims and \
            (like is None or t.get_device() == like.get_device()):
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(what, f"{name} must be a tensor on the GPU")
    if t.dtype not in dtypes:
        _refuse(what, f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if t.dim() != dims:
        _refuse(what, f"{name} must have {dims} dimensions, not {t.dim()}")
    if like is not None and t.device != like.device:
        _refuse(what, f"{name} is on {t.device}, not {like.device}")


def _rows(what, name, t):
    """The row stride of a matrix whose rows' elements lie side by side."""
    (n, d), (ld, step) = t.shape, t.stride()
    if step != 1 and d > 1:
        _refuse(what, f"{name}'s last dimension must be contiguous")
    return ld if n > 1 else max(d, ld)


def _vector(what, name, t, dtype, n, like):
    """t is a contiguous vector of n entries (None: of any number)."""
    _tensor(what, name, t, (dtype,), 1, like)
    if n is not None and t.shape[0] != n:
        _refuse(what, f"{name} has {t.shape[0]} entries, not {n}")
    if not t.is_contiguous():
        _refuse(what, f"{name} must be contiguous")


def _elsewhere(dev: int, stream):
    """None where the call's stream and device are the current ones, else the
    context that makes them so (what is allocated inside belongs to the stream)."""
    if stream is not None:
        if stream.device_index != dev:
            _refuse("stream", f"the stream is on device {stream.device_index}, the tensors on {dev}")
        return torch.cuda.stream(stream)
    return None if dev == torch.cuda.current_device() else torch.cuda.device(dev)


# the current stream's handle (torch.cuda.current_stream() builds an object each
# time, 2.7 us where this takes 0.1; a call of these operators takes 5 to 10)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    lambda dev: torch.cuda.current_stream(dev).cuda_stream


# ---------------------------------------------------------------- attention

def _layout(t):
    return t.dtype, t.shape, t.stride(), t.get_device()


# calls' descriptions and workspaces' bytes by their tensors' layouts: what was found in order
# is not looked at again (5 of a short call's 13 us)
_attn_plans = {}


def _attn_plan(q, k_prefix, v_prefix, k_own, v_own, own_len, scale, out):
    """The description of a call's shapes (out None: contiguous) and its workspace's bytes."""
    try:
        key = (_layout(q), _layout(k_prefix), _layout(v_prefix), _layout(k_own), _layout(v_own), _layout(own_len), scale,
               None if out is None else _layout(out))
        plan = _attn_plans.get(key)
    except (AttributeError, TypeError):  # (not all tensors: refused below)
        key = plan = None
    if plan is not None:
        return plan
    _refuse_attn(q, k_prefix, v_prefix, k_own, v_own, own_len, out)
    b, t, h, d = q.shape
    g, p, _ = k_prefix.shape
    r = k_own.shape[2]
    out_strides = (t * h * d, h * d, d) if out is None else out.stride()
    a = _PrefixAttnDesc(_DTYPES[q.dtype], b, t, h, g, d, p, r, 1.0 / math.sqrt(d) if scale is None else scale,
                        *_strides(q.stride(), (b, t, h)), *_strides(out_strides, (b, t, h)),
                        *_strides(k_prefix.stride(), (g, p)), *_strides(k_own.stride(), (b, g, r)))
    need = C.c_size_t(0)
    _check(_ops().ssd_prefix_attn_workspace(C.byref(a), C.byref(need)), "ssd_prefix_attn")
    plan = C.byref(a), need.value
    if key is not None:
        if len(_attn_plans) >= 256:
            _attn_plans.clear()
        _attn_plans[key] = plan
    return plan


def _strides(strides, sizes):
    """The strides, 0 for a dimension of one entry, which has none to speak of."""
    return [x if n > 1 else 0 for x, n in zip(strides, sizes)]


def _refuse_attn(q, k_prefix, v_prefix, k_own, v_own, own_len, out):
    """Says what is wrong with prefix_attention's tensors, if anything is."""
    what = "ssd_prefix_attn"
    _tensor(what, "q", q, _KINDS, 4)
    for name, t, dims in (("k_prefix", k_prefix, 3), ("v_prefix", v_prefix, 3), ("k_own", k_own, 4),
                          ("v_own", v_own, 4)):
        _tensor(what, name, t, (q.dtype,), dims, q)
    b, t, h, d = q.shape
    g, p = k_prefix.shape[:2]
    r = k_own.shape[2]
    if k_prefix.shape != v_prefix.shape or k_prefix.shape[2] != d:
        _refuse(what, f"k_prefix {tuple(k_prefix.shape)} and v_prefix {tuple(v_prefix.shape)} must be [G][P][{d}]")
    if k_own.shape != v_own.shape or tuple(k_own.shape) != (b, g, r, d):
        _refuse(what, f"k_own {tuple(k_own.shape)} and v_own {tuple(v_own.shape)} must be [{b}][{g}][R][{d}]")
    for k, v in ((k_prefix, v_prefix), (k_own, v_own)):
        if _strides(k.stride(), k.shape) != _strides(v.stride(), v.shape):
            _refuse(what, "keys and values must have the same strides")
    _vector(what, "own_len", own_len, torch.int32, b, q)
    if out is not None:
        _tensor(what, "out", out, (q.dtype,), 4, q)
        if out.shape != q.shape:
            _refuse(what, f"out {tuple(out.shape)} must be {tuple(q.shape)}")
    for name, x in (("q", q), ("k_prefix", k_prefix), ("k_own", k_own), ("out", out)):
        if x is not None and x.numel() and x.stride(-1) != 1:
            _refuse(what, f"{name}'s last dimension must be contiguous")


def prefix_attention(q, k_prefix, v_prefix, k_own, v_own, own_len, scale: Optional[float] = None, out=None,
                     return_lse: bool = False, stream=None):
    """ssd_prefix_attn: attention of sequences that share a prefix.

    q [B][T][H][D] (a sequence's last T positions); k_prefix, v_prefix
    [G][P][D]; k_own, v_own [B][G][R][D]; own_len int32 [B].  float32 or
    bfloat16, any strides that are multiples of 16 bytes with D contiguous (K and
    V alike).  scale defaults to 1 / sqrt(D).  Returns out [B][T][H][D], or (out,
    lse float32 [B][T][H])."""
    if scale is not None and type(scale) is not float:
        scale = float(scale)  # (by its value: what is remembered of a call must not go by a tensor's identity)
    a, need = _attn_plan(q, k_prefix, v_prefix, k_own, v_own, own_len, scale, out)
    dev = q.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return prefix_attention(q, k_prefix, v_prefix, k_own, v_own, own_len, scale, out, return_lse)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if return_lse else None
    work = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(_ops().ssd_prefix_attn(a, q.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(), k_own.data_ptr(),
                                  v_own.data_ptr(), own_len.data_ptr(), out.data_ptr(),
                                  lse.data_ptr() if return_lse else None, work.data_ptr(), need, _raw_stream(dev)),
           "ssd_prefix_attn")
    return (out, lse) if return_lse else out


# ---------------------------------------------------------------- distillation

def _logits(what, logits, ids, vals, weight):
    """Checks what the calls share and gives the library's first arguments."""
    _tensor(what, "logits", logits, _KINDS, 2)
    n, v = logits.shape
    ld = _rows(what, "logits", logits)
    _tensor(what, "ids", ids, (torch.int32,), 2, logits)
    _tensor(what, "vals", vals, (torch.float32,), 2, logits)
    if ids.shape != vals.shape or ids.shape[0] != n:
        _refuse(what, f"ids {tuple(ids.shape)} and vals {tuple(vals.shape)} must be [{n}][k]")
    if not ids.is_contiguous() or not vals.is_contiguous():
        _refuse(what, "ids and vals must be contiguous")
    if weight is not None:
        _vector(what, "weight", weight, torch.float32, n, logits)
    return _DTYPES[logits.dtype], logits.data_ptr(), ld, n, v, ids.data_ptr(), vals.data_ptr(), ids.shape[1]


def _grad_out(what, logits, out):
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _tensor(what, "out", out, (logits.dtype,), 2, logits)
    if out.shape != logits.shape:
        _refuse(what, f"out {tuple(out.shape)} must be {tuple(logits.shape)}")
    return out


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _loss_lse(logits):
    n = logits.shape[0]
    return (torch.empty(n, dtype=torch.float32, device=logits.device),
            torch.empty(n, dtype=torch.float32, device=logits.device))


def distill_forward(logits, ids, vals, weight=None, temperature: float = 1.0, stream=None):
    """ssd_distill_forward: (loss float32 [N], lse float32 [N]) of logits
    [N][V] (float32 or bfloat16) against the teacher's ids int32 [N][k] and
    their logits vals float32 [N][k]; weight float32 [N] or None."""
    what = "ssd_distill_forward"
    args = _logits(what, logits, ids, vals, weight)
    dev = logits.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return distill_forward(logits, ids, vals, weight, temperature)
    loss, lse = _loss_lse(logits)
    _check(_ops().ssd_distill_forward(*args, _ptr(weight), temperature, loss.data_ptr(), lse.data_ptr(),
                                      _raw_stream(dev)), what)
    return loss, lse


def distill_backward(logits, ids, vals, lse, weight=None, temperature: float = 1.0, out=None, stream=None):
    """ssd_distill_backward: the gradient [N][V] of sum(weight * divergence)
    in the logits' type, from distill_forward's lse.  out may be logits."""
    what = "ssd_distill_backward"
    args = _logits(what, logits, ids, vals, weight)
    _vector(what, "lse", lse, torch.float32, logits.shape[0], logits)
    dev = logits.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return distill_backward(logits, ids, vals, lse, weight, temperature, out)
    out = _grad_out(what, logits, out)
    _check(_ops().ssd_distill_backward(*args, lse.data_ptr(), _ptr(weight), temperature, out.data_ptr(),
                                       _rows(what, "out", out), _raw_stream(dev)), what)
    return out


def distill_step(logits, ids, vals, weight=None, temperature: float = 1.0, out=None, stream=None):
    """ssd_distill_step: (loss, lse, gradient) in one call.  out may be logits."""
    what = "ssd_distill_step"
    args = _logits(what, logits, ids, vals, weight)
    dev = logits.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return distill_step(logits, ids, vals, weight, temperature, out)
    loss, lse = _loss_lse(logits)
    out = _grad_out(what, logits, out)
    _check(_ops().ssd_distill_step(*args, _ptr(weight), temperature, loss.data_ptr(), lse.data_ptr(), out.data_ptr(),
                                   _rows(what, "out", out), _raw_stream(dev)), what)
    return loss, lse, out


# ---------------------------------------------------------------- embedding

def _rows_out(what, like, shape, dtype, out):
    """`out`, checked, or a new tensor of the type asked for."""
    if out is None:
        if dtype not in _DTYPES:
            _refuse(what, f"dtype must be torch.float32 or torch.bfloat16, not {dtype}")
        return torch.empty(shape, dtype=dtype, device=like.device)
    _tensor(what, "out", out, _KINDS, 2, like)
    if tuple(out.shape) != shape or (dtype is not None and out.dtype != dtype):
        _refuse(what, f"out must be {list(shape)} of the type asked for")
    return out


def embed(tokens, table, scale: float = 1.0, dtype=None, out=None, stream=None):
    """ssd_embed: scale * table[tokens] as [N][d] of `dtype` (default: the
    table's); tokens int32 [N], those outside the table give zeros."""
    what = "ssd_embed"
    _tensor(what, "table", table, _KINDS, 2)
    _vector(what, "tokens", tokens, torch.int32, None, table)
    n = tokens.shape[0]
    dev = table.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return embed(tokens, table, scale, dtype, out)
    v, d = table.shape
    out = _rows_out(what, table, (n, d), dtype or (None if out is not None else table.dtype), out)
    _check(_ops().ssd_embed(_DTYPES[table.dtype], _DTYPES[out.dtype], tokens.data_ptr(), n, table.data_ptr(),
                            _rows(what, "table", table), v, d, scale, out.data_ptr(), _rows(what, "out", out),
                            _raw_stream(dev)), what)
    return out


@functools.lru_cache(maxsize=256)
def _embed_grad_bytes(n, vocab, d):
    need = C.c_size_t(0)
    _check(_ops().ssd_embed_grad_workspace(n, vocab, d, C.byref(need)), "ssd_embed_grad")
    return need.value


def embed_grad(tokens, grad, vocab: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False,
               stream=None):
    """ssd_embed_grad: the gradient [vocab][d] of embed's table from grad
    [N][d], of `dtype` (default: grad's).  accumulate adds to `out`."""
    what = "ssd_embed_grad"
    _tensor(what, "grad", grad, _KINDS, 2)
    n, d = grad.shape
    _vector(what, "tokens", tokens, torch.int32, n, grad)
    if accumulate and out is None:
        _refuse(what, "accumulate needs out")
    dev = grad.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return embed_grad(tokens, grad, vocab, scale, dtype, out, accumulate)
    vocab = operator.index(vocab)
    need = _embed_grad_bytes(n, vocab, d)
    out = _rows_out(what, grad, (vocab, d), dtype or (None if out is not None else grad.dtype), out)
    work = torch.empty(need, dtype=torch.uint8, device=grad.device)
    _check(_ops().ssd_embed_grad(_DTYPES[grad.dtype], _DTYPES[out.dtype], tokens.data_ptr(), n, grad.data_ptr(),
                                 _rows(what, "grad", grad), vocab, d, scale, int(accumulate), out.data_ptr(),
                                 _rows(what, "out", out), work.data_ptr(), need, _raw_stream(dev)), what)
    return out
