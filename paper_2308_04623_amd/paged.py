"""A paged cache in 8 bits for a batch of sequences, and the attention that
reads it (include/ssd_pages.h), on torch tensors.

Pages holds the pool.  A batch's sequences are plain int32 tensors beside it,
  table  [B][C]  pages of a sequence's rows, -1 where there is none,
  length [B]     rows of a sequence, below 0 for a slot without one,
  refs   [P]     how many table entries name a page,
and the rows of their open pages, in the model's type,
  k_tail, v_tail [L][B][G][R][D], the row of position p at p % R.
A step's new rows, [L][B][T][G][D], are attended to beside them (paged_attention, a
layer at a time), and the accepted ones join the sequences (pages_commit).

As in ops.py, the library does the work and PyTorch supplies device memory and
streams: outputs and scratch come from torch's allocator on the stream of the call (the
current one, or `stream`); table, length, refs, tails and pool are changed in place.
Nothing is recorded for autograd, and nothing has a gradient.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import ops, ssd
from .ops import _check, _DTYPES, _elsewhere, _KINDS, _raw_stream, _refuse, _strides, _tensor, _vector

# every function include/ssd_pages.h declares
EXPORTS = ("ssd_paged_attn_workspace", "ssd_paged_attn", "ssd_pages_store", "ssd_pages_load", "ssd_pages_workspace",
           "ssd_pages_take", "ssd_pages_commit", "ssd_pages_fork", "ssd_pages_compact")
CODES = {"int8": 0, "e4m3": 1}


class _Pool(C.Structure):
    _fields_ = [("code", C.c_int32), ("n_layer", C.c_int32), ("n_page", C.c_int32), ("n_kv_head", C.c_int32),
                ("page_rows", C.c_int32), ("head_dim", C.c_int32), ("data", C.c_void_p), ("scale", C.c_void_p)]


class _Seqs(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_col", C.c_int32), ("table_ld", C.c_int64), ("table", C.c_void_p),
                ("length", C.c_void_p), ("refs", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("rows", C.c_int32), ("layer", C.c_int64), ("seq", C.c_int64),
                ("head", C.c_int64), ("row", C.c_int64)]


class _AttnDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("layer", C.c_int32), ("n_query", C.c_int32), ("n_head", C.c_int32),
                ("tail_rows", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("scale", C.c_float)] + \
               [(n, C.c_int64) for n in ("q_seq", "q_row", "q_head", "out_seq", "out_row", "out_head", "tail_seq",
                                         "tail_head", "tail_row", "new_seq", "new_row", "new_head")]


_lib = None


def _ops():
    global _lib
    if _lib is None:
        L = ops._ops()
        i32, i64, vp, sz, P = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t, C.POINTER
        pool, seqs, rows, attn = P(_Pool), P(_Seqs), P(_Rows), P(_AttnDesc)
        sig = {
            "ssd_paged_attn_workspace": [pool, seqs, attn, P(sz)],
            "ssd_paged_attn": [pool, seqs, attn] + [vp] * 9 + [sz, vp],
            "ssd_pages_store": [pool, vp, i32, i32, i32, rows, vp, vp, vp],
            "ssd_pages_load": [pool, vp, i32, i32, i32, rows, vp, vp, vp],
            "ssd_pages_workspace": [pool, seqs, P(sz)],
            "ssd_pages_take": [pool, seqs, vp, vp, vp, sz, vp],
            "ssd_pages_commit": [pool, seqs, rows, vp, vp, rows, vp, vp, vp, i64, i32, vp, i32, i32, vp, vp, sz, vp],
            "ssd_pages_fork": [seqs, i32, i32, vp, rows, i32, i32, i32, vp, vp, vp],
            "ssd_pages_compact": [pool, seqs, vp, vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = C.c_int
        _lib = L
    return _lib


class Pages:
    """The pool: data uint8 [L][P][G][2][page_rows * D], scale float32 [L][P][G][2], contiguous.  It stays the pool of these
    tensors: their contents change, its attributes do not (other tensors: another Pages)."""

    def __init__(self, data, scale, page_rows: int, code: str = "int8"):
        what = "Pages"
        _tensor(what, "data", data, (torch.uint8,), 5)
        _tensor(what, "scale", scale, (torch.float32,), 4, data)
        if code not in CODES:
            _refuse(what, f"code must be one of {sorted(CODES)}, not {code!r}")
        l, p, g, two, size = data.shape
        if two != 2 or tuple(scale.shape) != (l, p, g, 2) or page_rows not in (32, 64, 128) or size % page_rows:
            _refuse(what, f"data {tuple(data.shape)} and scale {tuple(scale.shape)} must be [L][P][G][2][{page_rows} D] "
                          "and [L][P][G][2], of 32, 64 or 128 rows")
        if not data.is_contiguous() or not scale.is_contiguous():
            _refuse(what, "data and scale must be contiguous")
        self.data, self.scale, self.page_rows, self.code = data, scale, page_rows, code
        self.n_layer, self.n_page, self.n_kv_head, self.head_dim = l, p, g, size // page_rows
        self.device, self._dev = data.device, data.get_device()
        self._pool = _Pool(CODES[code], l, p, g, page_rows, self.head_dim, data.data_ptr(), scale.data_ptr())
        self._ref = C.byref(self._pool)
        self.kind = code, l, p, g, page_rows, self.head_dim, self._dev  # (all that checks depend on)

    def __setattr__(self, name, value):
        if "kind" in self.__dict__:  # (set last; the calls hold the tensors' addresses)
            _refuse("Pages", f"{name} cannot be replaced; make another Pages")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        _refuse("Pages", f"{name} cannot be taken away")

    @classmethod
    def empty(cls, n_layer: int, n_page: int, n_kv_head: int, head_dim: int, page_rows: int = 32, code: str = "int8",
              device="cuda") -> "Pages":
        """A pool of n_page pages that hold nothing yet (they read as zeros)."""
        shape = (n_layer, n_page, n_kv_head, 2)
        return cls(torch.zeros(shape + (page_rows * head_dim,), dtype=torch.uint8, device=device),
                   torch.zeros(shape, dtype=torch.float32, device=device), page_rows, code)


def _counts(what, **values):
    """They are what the descriptions' 32 bits hold (where ctypes would drop the others)."""
    for name, x in values.items():
        if not 0 <= ops.operator.index(x) < 1 << 31:
            _refuse(what, f"{name} is {x}, not a number from 0 on of 31 bits")


def _pages(what, pages):
    if not isinstance(pages, Pages):
        _refuse(what, "pages must be a paged.Pages")


def _seqs(what, table, length, refs, like, n_page=None):
    _tensor(what, "table", table, (torch.int32,), 2, like)
    b, c = table.shape
    ld, step = table.stride()
    if step != 1 and c > 1:
        _refuse(what, "table's last dimension must be contiguous")
    _vector(what, "length", length, torch.int32, b, like)
    if refs is not None:
        _vector(what, "refs", refs, torch.int32, n_page, like)
    return _Seqs(b, c, ld if b > 1 else max(c, ld), table.data_ptr(), length.data_ptr(),
                 refs.data_ptr() if refs is not None else None)


def _workspace(what, pages, seqs):
    """The bytes that take, commit and compact need."""
    size = C.c_size_t(0)
    _check(_ops().ssd_pages_workspace(pages._ref, C.byref(seqs), C.byref(size)), what)
    return size.value


def _lies(what, name, t):
    if t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse(what, f"{name}'s last dimension must be contiguous")


def _alike(what, k, v, name):
    if _strides(k.stride(), k.shape) != _strides(v.stride(), v.shape):
        _refuse(what, f"{name}'s keys and values must have the same strides")


# calls' descriptions and workspaces' bytes by their tensors' layouts (and the function): what was found in order is
# not looked at again, which is half of the host's time of a call
_plans = {}


def _plan(key, make):
    """What make() gives for this key (None: for a call that is not all tensors, and is refused)."""
    plan = _plans.get(key) if key is not None else None
    if plan is None:
        plan = make()
        if key is not None:
            if len(_plans) >= 512:
                _plans.clear()
            _plans[key] = plan
    return plan


def _key(what, values, *tensors):
    try:
        return (what, values, *[None if t is None else (t.dtype, t.shape, t.stride(), t.get_device()) for t in tensors])
    except AttributeError:
        return None


# ---------------------------------------------------------------- attention

def _attn_plan(q, pages, table, length, k_tail, v_tail, k_new, v_new, layer, anc, window, sinks, scale, out):
    _counts("ssd_paged_attn", layer=layer, window=window, sinks=sinks)
    _refuse_attn(q, pages, table, length, k_tail, v_tail, k_new, v_new, anc, out)
    b, t, h, d = q.shape
    g, r = k_tail.shape[1:3]
    out_strides = (t * h * d, h * d, d) if out is None else out.stride()
    a = _AttnDesc(_DTYPES[q.dtype], layer, t, h, r, window, sinks, 1.0 / math.sqrt(d) if scale is None else scale,
                  *_strides(q.stride(), (b, t, h)), *_strides(out_strides, (b, t, h)),
                  *_strides(k_tail.stride(), (b, g, r)), *_strides(k_new.stride(), (b, t, g)))
    need = C.c_size_t(0)
    seqs = _seqs("ssd_paged_attn", table, length, None, q)
    _check(_ops().ssd_paged_attn_workspace(pages._ref, C.byref(seqs), C.byref(a), C.byref(need)), "ssd_paged_attn")
    return C.byref(a), need.value, seqs.n_seq, seqs.n_col, seqs.table_ld


def _refuse_attn(q, pages, table, length, k_tail, v_tail, k_new, v_new, anc, out):
    """Says what is wrong with paged_attention's tensors, if anything is."""
    what = "ssd_paged_attn"
    _pages(what, pages)
    _tensor(what, "q", q, _KINDS, 4, pages.data)
    b, t, h, d = q.shape
    g = pages.n_kv_head
    for name, x in (("k_tail", k_tail), ("v_tail", v_tail), ("k_new", k_new), ("v_new", v_new)):
        _tensor(what, name, x, (q.dtype,), 4, q)
    if d != pages.head_dim:
        _refuse(what, f"q {tuple(q.shape)} must be [B][T][H][{pages.head_dim}]")
    if k_tail.shape != v_tail.shape or k_tail.shape[:2] != (b, g) or k_tail.shape[3] != d:
        _refuse(what, f"k_tail {tuple(k_tail.shape)} and v_tail {tuple(v_tail.shape)} must be [{b}][{g}][R][{d}]")
    if k_new.shape != v_new.shape or tuple(k_new.shape) != (b, t, g, d):
        _refuse(what, f"k_new {tuple(k_new.shape)} and v_new {tuple(v_new.shape)} must be [{b}][{t}][{g}][{d}]")
    _alike(what, k_tail, v_tail, "the tail")
    _alike(what, k_new, v_new, "the new rows")
    _tensor(what, "table", table, (torch.int32,), 2, q)
    if table.shape[0] != b:
        _refuse(what, f"table has {table.shape[0]} rows, not {b}")
    _seqs(what, table, length, None, q)
    if anc is not None:
        _tensor(what, "anc", anc, (torch.int64,), 2, q)
        if tuple(anc.shape) != (b, t) or not anc.is_contiguous():
            _refuse(what, f"anc {tuple(anc.shape)} must be [{b}][{t}], contiguous")
    if out is not None:
        _tensor(what, "out", out, (q.dtype,), 4, q)
        if out.shape != q.shape:
            _refuse(what, f"out {tuple(out.shape)} must be {tuple(q.shape)}")
    for name, x in (("q", q), ("k_tail", k_tail), ("k_new", k_new), ("out", out)):
        if x is not None:
            _lies(what, name, x)


def paged_attention(q, pages: Pages, table, length, k_tail, v_tail, k_new, v_new, layer: int = 0, anc=None,
                    window: int = 0, sinks: int = 0, scale: Optional[float] = None, out=None,
                    return_lse: bool = False, stream=None):
    """ssd_paged_attn: attention of each sequence's T new rows over its cached rows and each other.

    q [B][T][H][D]; k_tail, v_tail [B][G][R][D] of this layer; k_new, v_new
    [B][T][G][D]; float32 or bfloat16, strides multiples of 16 bytes with D contiguous (K and V alike); table int32
    [B][C], length int32 [B].  anc int64 [B][T]: for a tree, the new rows that each sees as bits (None: a
    chain).  window: rows that are seen back from the query, itself among them (0: all), with the first
    `sinks`.  scale defaults to 1 / sqrt(D).  Returns out [B][T][H][D], or (out, lse
    float32 [B][T][H])."""
    if scale is not None and type(scale) is not float:
        scale = float(scale)  # (by its value: what is remembered of a call must not go by a tensor's identity)
    layer, window, sinks = ops.operator.index(layer), ops.operator.index(window), ops.operator.index(sinks)
    if not isinstance(pages, Pages):
        _pages("ssd_paged_attn", pages)
    a, need, n_seq, n_col, ld = _plan(
        _key("attn", (pages.kind, layer, window, sinks, scale), q, table, length, k_tail, v_tail, k_new, v_new, anc, out),
        lambda: _attn_plan(q, pages, table, length, k_tail, v_tail, k_new, v_new, layer, anc, window, sinks, scale, out))
    dev = pages._dev
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return paged_attention(q, pages, table, length, k_tail, v_tail, k_new, v_new, layer, anc, window, sinks,
                                   scale, out, return_lse)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if return_lse else None
    work = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    seqs = _Seqs(n_seq, n_col, ld, table.data_ptr(), length.data_ptr(), None)
    _check(_ops().ssd_paged_attn(pages._ref, C.byref(seqs), a, q.data_ptr(), k_tail.data_ptr(), v_tail.data_ptr(),
                                 k_new.data_ptr(), v_new.data_ptr(), anc.data_ptr() if anc is not None else None,
                                 out.data_ptr(), lse.data_ptr() if return_lse else None,
                                 work.data_ptr() if need else None, need,
                                 _raw_stream(dev)), "ssd_paged_attn")
    return (out, lse) if return_lse else out


# ---------------------------------------------------------------- rows into pages and back

def _block_rows(what, pages, ids, k, v):
    _vector(what, "ids", ids, torch.int32, None, pages.data)
    n = ids.shape[0]
    _tensor(what, "k", k, _KINDS, 5, pages.data)
    _tensor(what, "v", v, (k.dtype,), 5, pages.data)
    shape = (n, pages.n_kv_head, pages.page_rows, pages.head_dim)
    if k.shape != v.shape or tuple(k.shape[1:]) != shape:
        _refuse(what, f"k {tuple(k.shape)} and v {tuple(v.shape)} must be [L]{list(shape)}")
    _alike(what, k, v, "the rows")
    _lies(what, "k", k)
    return _Rows(_DTYPES[k.dtype], pages.page_rows, *_strides(k.stride(), k.shape)[:4])


def pages_store(pages: Pages, ids, k, v, layer: int = 0, stream=None):
    """ssd_pages_store: k, v [L][N][G][page_rows][D] (float32 or bfloat16; the strides of attention) become
    pages ids int32 [N] in layers layer .. layer + L - 1.  A prompt's rows [L][G][n page_rows][D] are
    x.unflatten(2, (n, page_rows)).transpose(1, 2)."""
    what = "ssd_pages_store"
    _pages(what, pages)
    layer = ops.operator.index(layer)
    d = _plan(_key(what, (pages.kind, layer), ids, k, v),
              lambda: _counts(what, layer=layer) or C.byref(_block_rows(what, pages, ids, k, v)))
    where = _elsewhere(pages._dev, stream)
    if where is not None:
        with where:
            return pages_store(pages, ids, k, v, layer)
    _check(_ops().ssd_pages_store(pages._ref, ids.data_ptr(), ids.shape[0], layer, k.shape[0], d, k.data_ptr(),
                                  v.data_ptr(), _raw_stream(pages._dev)), what)


def pages_load(pages: Pages, ids, dtype=torch.float32, layer: int = 0, n_layer: Optional[int] = None, stream=None):
    """ssd_pages_load: (k, v) [L][N][G][page_rows][D] of pages ids int32 [N] in n_layer layers from
    `layer` on (default: all), as the values that the pages stand for; ids outside the pool give zeros."""
    what = "ssd_pages_load"
    _pages(what, pages)
    layer = ops.operator.index(layer)
    n_layer = pages.n_layer - layer if n_layer is None else ops.operator.index(n_layer)

    def make():
        _vector(what, "ids", ids, torch.int32, None, pages.data)
        if dtype not in _DTYPES:
            _refuse(what, f"dtype must be torch.float32 or torch.bfloat16, not {dtype}")
        if not 0 <= layer <= layer + n_layer <= pages.n_layer:
            _refuse(what, f"layers {layer} .. {layer + n_layer} are not the pool's {pages.n_layer}")
        shape = n_layer, ids.shape[0], pages.n_kv_head, pages.page_rows, pages.head_dim
        _, n, g, r, w = shape
        return shape, C.byref(_Rows(_DTYPES[dtype], r, n * g * r * w, g * r * w, r * w, w))

    shape, d = _plan(_key(what, (pages.kind, dtype, layer, n_layer), ids), make)
    where = _elsewhere(pages._dev, stream)
    if where is not None:
        with where:
            return pages_load(pages, ids, dtype, layer, n_layer)
    k = torch.empty(shape, dtype=dtype, device=pages.device)
    v = torch.empty(shape, dtype=dtype, device=pages.device)
    _check(_ops().ssd_pages_load(pages._ref, ids.data_ptr(), shape[1], layer, n_layer, d, k.data_ptr(), v.data_ptr(),
                                 _raw_stream(pages._dev)), what)
    return k, v


# ---------------------------------------------------------------- the sequences

def pages_take(pages: Pages, refs, table, length, count, stream=None):
    """ssd_pages_take: slots with count int32 [B] >= 0 get so many pages, and so many
    times page_rows rows, behind those they have; returns how many each got, int32 [B] (-1: none asked for, or not to be had)."""
    what = "ssd_pages_take"
    _pages(what, pages)

    def make():
        seqs = _seqs(what, table, length, refs, pages.data, pages.n_page)
        _vector(what, "count", count, torch.int32, seqs.n_seq, pages.data)
        return seqs.n_seq, seqs.n_col, seqs.table_ld, _workspace(what, pages, seqs)

    b, c, ld, need = _plan(_key(what, pages.kind, refs, table, length, count), make)
    where = _elsewhere(pages._dev, stream)
    if where is not None:
        with where:
            return pages_take(pages, refs, table, length, count)
    seqs = _Seqs(b, c, ld, table.data_ptr(), length.data_ptr(), refs.data_ptr())
    got = torch.empty(b, dtype=torch.int32, device=pages.device)
    work = torch.empty(need, dtype=torch.uint8, device=pages.device)
    _check(_ops().ssd_pages_take(pages._ref, C.byref(seqs), count.data_ptr(), got.data_ptr(), work.data_ptr(), need,
                                 _raw_stream(pages._dev)), what)
    return got


def _tail(what, k, v, n_layer, n_seq, g, d, like):
    _tensor(what, "k_tail", k, _KINDS, 5, like)
    _tensor(what, "v_tail", v, (k.dtype,), 5, like)
    if k.shape != v.shape or (n_layer is not None and k.shape[0] != n_layer) or k.shape[1] != n_seq or \
            (g is not None and (k.shape[2], k.shape[4]) != (g, d)):
        _refuse(what, f"k_tail {tuple(k.shape)} and v_tail {tuple(v.shape)} must be "
                      f"[{'L' if n_layer is None else n_layer}][{n_seq}][{g or 'G'}][R][{d or 'D'}]")
    _alike(what, k, v, "the tail")
    _lies(what, "k_tail", k)
    return _Rows(_DTYPES[k.dtype], k.shape[3], *_strides(k.stride(), k.shape)[:4])


def pages_commit(pages: Pages, refs, table, length, k_tail, v_tail, k_new, v_new, path, path_len, window: int = 0,
                 sinks: int = 0, stream=None):
    """ssd_pages_commit: rows path[b][:path_len[b]] of k_new, v_new [L][B][T][G][D] become sequence b's next
    rows (at most T of them).  path int32 [B][M], path_len int32 [B].  Returns how many pages of each sequence got full, int32 [B]
    (-1: pages did not suffice, and nothing of the sequence changed).  window > 0: pages that no later row
    sees, with this window and these sinks, are given back."""
    what = "ssd_pages_commit"
    _pages(what, pages)
    window, sinks = ops.operator.index(window), ops.operator.index(sinks)
    b, c, ld, tail, fresh, path_ld, need = _plan(
        _key(what, (pages.kind, window, sinks), refs, table, length, k_tail, v_tail, k_new, v_new, path, path_len),
        lambda: _counts(what, window=window, sinks=sinks) or
        _commit_plan(what, pages, refs, table, length, k_tail, v_tail, k_new, v_new, path, path_len))
    where = _elsewhere(pages._dev, stream)
    if where is not None:
        with where:
            return pages_commit(pages, refs, table, length, k_tail, v_tail, k_new, v_new, path, path_len, window, sinks)
    seqs = _Seqs(b, c, ld, table.data_ptr(), length.data_ptr(), refs.data_ptr())
    full = torch.empty(b, dtype=torch.int32, device=pages.device)
    work = torch.empty(need, dtype=torch.uint8, device=pages.device)
    _check(_ops().ssd_pages_commit(pages._ref, C.byref(seqs), tail, k_tail.data_ptr(), v_tail.data_ptr(), fresh,
                                   k_new.data_ptr(), v_new.data_ptr(), path.data_ptr(), path_ld, path.shape[1],
                                   path_len.data_ptr(), window, sinks, full.data_ptr(), work.data_ptr(), need,
                                   _raw_stream(pages._dev)), what)
    return full


def _commit_plan(what, pages, refs, table, length, k_tail, v_tail, k_new, v_new, path, path_len):
    like = pages.data
    seqs = _seqs(what, table, length, refs, like, pages.n_page)
    b, g, w = seqs.n_seq, pages.n_kv_head, pages.head_dim
    tail = _tail(what, k_tail, v_tail, pages.n_layer, b, g, w, like)
    _tensor(what, "k_new", k_new, (k_tail.dtype,), 5, like)
    _tensor(what, "v_new", v_new, (k_tail.dtype,), 5, like)
    if k_new.shape != v_new.shape or k_new.shape[:2] != (pages.n_layer, b) or tuple(k_new.shape[3:]) != (g, w):
        _refuse(what, f"k_new {tuple(k_new.shape)} and v_new {tuple(v_new.shape)} must be "
                      f"[{pages.n_layer}][{b}][T][{g}][{w}]")
    _alike(what, k_new, v_new, "the new rows")
    _lies(what, "k_new", k_new)
    s = _strides(k_new.stride(), k_new.shape)
    fresh = _Rows(_DTYPES[k_new.dtype], k_new.shape[2], s[0], s[1], s[3], s[2])
    _tensor(what, "path", path, (torch.int32,), 2, like)
    if path.shape[0] != b or (path.shape[1] > 1 and path.stride(1) != 1):
        _refuse(what, f"path {tuple(path.shape)} must be [{b}][M] with contiguous rows")
    _vector(what, "path_len", path_len, torch.int32, b, like)
    return (b, seqs.n_col, seqs.table_ld, C.byref(tail), C.byref(fresh), path.stride(0) if b > 1 else path.shape[1],
            _workspace(what, pages, seqs))


def pages_fork(refs, table, length, parents, k_tail, v_tail, page_rows: int, stream=None):
    """ssd_pages_fork: slot b becomes a copy of slot parents[b] (int32 [B]), which has to keep itself; itself: it stays as it
    is; any other value: it is freed."""
    what = "ssd_pages_fork"
    page_rows = ops.operator.index(page_rows)

    def make():
        _counts(what, page_rows=page_rows)
        _tensor(what, "table", table, (torch.int32,), 2)
        seqs = _seqs(what, table, length, refs, table)
        _vector(what, "parents", parents, torch.int32, seqs.n_seq, table)
        tail = _tail(what, k_tail, v_tail, None, seqs.n_seq, None, None, table)
        return seqs.n_seq, seqs.n_col, seqs.table_ld, C.byref(tail)

    b, c, ld, tail = _plan(_key(what, page_rows, refs, table, length, parents, k_tail, v_tail), make)
    dev = table.get_device()
    where = _elsewhere(dev, stream)
    if where is not None:
        with where:
            return pages_fork(refs, table, length, parents, k_tail, v_tail, page_rows)
    seqs = _Seqs(b, c, ld, table.data_ptr(), length.data_ptr(), refs.data_ptr())
    n_layer, _, g, _, w = k_tail.shape
    _check(_ops().ssd_pages_fork(C.byref(seqs), refs.shape[0], page_rows, parents.data_ptr(), tail, n_layer, g, w,
                                 k_tail.data_ptr(), v_tail.data_ptr(), _raw_stream(dev)), what)


def pages_compact(pages: Pages, refs, table, stream=None):
    """ssd_pages_compact: moves the pages in use to the front of the pool; returns their number, int32 [1]."""
    what = "ssd_pages_compact"
    _pages(what, pages)

    def make():
        _tensor(what, "table", table, (torch.int32,), 2, pages.data)
        _vector(what, "refs", refs, torch.int32, pages.n_page, pages.data)
        b, c = table.shape
        if c > 1 and table.stride(1) != 1:
            _refuse(what, "table's last dimension must be contiguous")
        ld = table.stride(0) if b > 1 else max(c, table.stride(0))
        at = refs.data_ptr()
        return b, c, ld, _workspace(what, pages, _Seqs(b, c, ld, table.data_ptr(), at, at))

    b, c, ld, need = _plan(_key(what, pages.kind, refs, table), make)
    where = _elsewhere(pages._dev, stream)
    if where is not None:
        with where:
            return pages_compact(pages, refs, table)
    # (lengths are not looked at)
    seqs = _Seqs(b, c, ld, table.data_ptr(), refs.data_ptr(), refs.data_ptr())
    used = torch.empty(1, dtype=torch.int32, device=pages.device)
    work = torch.empty(need, dtype=torch.uint8, device=pages.device)
    _check(_ops().ssd_pages_compact(pages._ref, C.byref(seqs), used.data_ptr(), work.data_ptr(), need,
                                    _raw_stream(pages._dev)), what)
    return used
