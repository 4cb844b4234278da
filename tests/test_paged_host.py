"""The operators of include/ssd_pages.h without a GPU: exports, workspace sizes and the
refusals of the C entry points (every check runs before anything is enqueued, so none of these
calls reaches a device), and paged_model's own arithmetic."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paged_model as M
from paper_2308_04623_amd import paged, ssd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MB = 1 << 20  # places of aligned device addresses
INVALID, UNSUPPORTED, CAPACITY = ssd.E_INVALID_ARG, ssd.E_UNSUPPORTED, ssd.E_CAPACITY


def pool(**kw):
    v = dict(code=0, n_layer=2, n_page=20, n_kv_head=4, page_rows=32, head_dim=64, data=100 * MB, scale=200 * MB)
    v.update(kw)
    return paged._Pool(*v.values())


def seqs(**kw):
    v = dict(n_seq=3, n_col=5, table_ld=5, table=300 * MB, length=301 * MB, refs=302 * MB)
    v.update(kw)
    return paged._Seqs(*v.values())


def rows(kind, **kw):
    """[2][3][4][39][64] of the tail, [2][3][8][4][64] new rows, [2][6][4][32][64] of pages."""
    v = {"tail": dict(dtype=ssd.BF16, rows=39, layer=3 * 4 * 39 * 64, seq=4 * 39 * 64, head=39 * 64, row=64),
         "new": dict(dtype=ssd.BF16, rows=8, layer=3 * 8 * 256, seq=8 * 256, head=64, row=256),
         "pages": dict(dtype=ssd.BF16, rows=32, layer=6 * 4 * 2048, seq=4 * 2048, head=2048, row=64)}[kind]
    v.update(kw)
    return paged._Rows(*v.values())


def ref(x):
    return C.byref(x) if x is not None else None


def test_library_exports_every_declared_operator():
    txt = open(os.path.join(ROOT, "include", "ssd_pages.h")).read()
    names = sorted(set(re.findall(r"\b(ssd_[a-z_0-9]+)\s*\(", re.sub(r"/\*.*?\*/", "", txt, flags=re.S))))
    assert names == sorted(paged.EXPORTS)
    for n in names:
        assert hasattr(paged._ops(), n), n


# ---------------------------------------------------------------- attention

def desc(**kw):
    v = dict(dtype=ssd.BF16, layer=1, n_query=8, n_head=8, tail_rows=39, window=0, sinks=0, scale=0.125, q_seq=8 * 512,
             q_row=512, q_head=64, out_seq=8 * 512, out_row=512, out_head=64, tail_seq=4 * 39 * 64, tail_head=39 * 64,
             tail_row=64, new_seq=8 * 256, new_row=256, new_head=64)
    v.update(kw)
    return paged._AttnDesc(**v)


def attn(p=None, s=None, d=None, q=MB, kt=2 * MB, vt=3 * MB, kn=4 * MB, vn=5 * MB, anc=None, out=6 * MB, lse=None,
         work=16 * MB, size=1 << 40):
    return paged._ops().ssd_paged_attn(ref(p or pool()), ref(s or seqs()), ref(d or desc()), q, kt, vt, kn, vn, anc, out,
                                       lse, work, size, None)


POOLS = [(dict(code=2), INVALID), (dict(code=-1), INVALID), (dict(page_rows=16), UNSUPPORTED), (dict(page_rows=96), UNSUPPORTED),
         (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(n_layer=0), INVALID),
         (dict(n_layer=4097), INVALID), (dict(n_page=0), INVALID), (dict(n_page=(1 << 20) + 1), INVALID),
         (dict(n_kv_head=0), INVALID), (dict(n_kv_head=1025), INVALID), (dict(data=None), INVALID),
         (dict(scale=None), INVALID), (dict(data=100 * MB + 8), UNSUPPORTED), (dict(scale=200 * MB + 4), UNSUPPORTED)]
SEQS = [(dict(n_seq=0), INVALID), (dict(n_seq=4097), INVALID), (dict(n_col=-1), INVALID),
        (dict(n_col=1 << 25, table_ld=1 << 25), INVALID), (dict(table_ld=4), INVALID), (dict(table=None), INVALID),
        (dict(length=None), INVALID), (dict(length=301 * MB + 2), INVALID), (dict(table=300 * MB + 1), INVALID)]


@pytest.mark.parametrize("kw,status", POOLS)
def test_pools_are_checked(kw, status):
    p, n = pool(**kw), C.c_size_t(0)
    L = paged._ops()
    d, t, f = rows("pages"), rows("tail"), rows("new")
    assert attn(p) == status
    assert L.ssd_pages_workspace(ref(p), ref(seqs()), C.byref(n)) == status
    assert L.ssd_pages_store(ref(p), MB, 6, 0, 2, ref(d), 2 * MB, 3 * MB, None) == status
    assert L.ssd_pages_load(ref(p), MB, 6, 0, 2, ref(d), 2 * MB, 3 * MB, None) == status
    assert L.ssd_pages_take(ref(p), ref(seqs()), MB, MB, 16 * MB, 1 << 40, None) == status
    assert L.ssd_pages_commit(ref(p), ref(seqs()), ref(t), 2 * MB, 3 * MB, ref(f), 4 * MB, 5 * MB, MB, 8, 8, MB, 0, 0, MB,
                              16 * MB, 1 << 40, None) == status
    assert L.ssd_pages_compact(ref(p), ref(seqs()), MB, 16 * MB, 1 << 40, None) == status


@pytest.mark.parametrize("kw,status", SEQS + [(dict(refs=None), INVALID), (dict(refs=302 * MB + 1), INVALID)])
def test_sequences_are_checked(kw, status):
    s, n, L = seqs(**kw), C.c_size_t(0), paged._ops()
    t, f = rows("tail"), rows("new")
    if "refs" not in kw:
        assert attn(s=s) == status
    assert L.ssd_pages_workspace(ref(pool()), ref(s), C.byref(n)) == status
    assert L.ssd_pages_take(ref(pool()), ref(s), MB, MB, 16 * MB, 1 << 40, None) == status
    assert L.ssd_pages_commit(ref(pool()), ref(s), ref(t), 2 * MB, 3 * MB, ref(f), 4 * MB, 5 * MB, MB, 8, 8, MB, 0, 0, MB,
                              16 * MB, 1 << 40, None) == status
    assert L.ssd_pages_fork(ref(s), 20, 32, MB, ref(t), 2, 4, 64, 2 * MB, 3 * MB, None) == status
    assert L.ssd_pages_compact(ref(pool()), ref(s), MB, 16 * MB, 1 << 40, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(n_query=0), INVALID),
    (dict(n_query=65), INVALID), (dict(n_head=6), INVALID), (dict(n_head=0), INVALID), (dict(n_head=1028), INVALID),
    (dict(tail_rows=31), INVALID), (dict(tail_rows=1 << 30), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(window=7), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID),
    (dict(q_row=516), UNSUPPORTED), (dict(tail_row=65), UNSUPPORTED), (dict(new_head=-64), INVALID), (dict(out_head=0), INVALID),
    (dict(out_row=448), INVALID), (dict(out_seq=7 * 512), INVALID), (dict(out_head=512, out_row=128), INVALID)])
def test_attention_refuses_shapes(kw, status):
    assert attn(d=desc(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(kt=None), INVALID), (dict(vt=None), INVALID), (dict(kn=None), INVALID), (dict(vn=None), INVALID),
    (dict(out=None), INVALID), (dict(work=None, s=seqs(n_col=500, table_ld=500)), INVALID), (dict(q=MB + 8), UNSUPPORTED), (dict(vn=5 * MB + 2), UNSUPPORTED),
    (dict(out=6 * MB + 4), UNSUPPORTED), (dict(anc=7 * MB + 4), INVALID), (dict(lse=7 * MB + 2), INVALID),
    (dict(size=0, s=seqs(n_col=500, table_ld=500)), CAPACITY), (dict(work=16 * MB + 4), CAPACITY), (dict(out=MB), INVALID), (dict(out=MB + 16), INVALID),
    (dict(out=2 * MB + 16 * 64), INVALID), (dict(out=5 * MB - 16), INVALID), (dict(out=3 * MB), INVALID)])
def test_attention_refuses_buffers(kw, status):
    assert attn(**kw) == status


def test_attention_refuses_more_workgroups_than_a_grid_holds():
    n = C.c_size_t(0)
    p, s = pool(n_kv_head=1, head_dim=128), seqs(n_seq=4096)
    big = dict(n_query=64, n_head=1024, dtype=ssd.F32)  # 4096 tiles of 16 queries for each sequence
    assert paged._ops().ssd_paged_attn_workspace(ref(p), ref(s), ref(desc(**big)), C.byref(n)) == CAPACITY
    assert attn(p, s, desc(**big)) == CAPACITY
    assert paged._ops().ssd_paged_attn_workspace(ref(p), ref(s), ref(desc(**{**big, "n_query": 63})), C.byref(n)) == ssd.OK


def test_workspaces_grow_with_the_call():
    a, b, L = C.c_size_t(0), C.c_size_t(0), paged._ops()
    assert L.ssd_pages_workspace(ref(pool()), ref(seqs()), C.byref(a)) == ssd.OK and a.value > 0
    assert L.ssd_pages_workspace(ref(pool(n_page=1000)), ref(seqs(n_seq=9)), C.byref(b)) == ssd.OK and b.value > a.value
    assert L.ssd_paged_attn_workspace(ref(pool()), ref(seqs(n_seq=1)), ref(desc()), C.byref(a)) == ssd.OK
    assert L.ssd_paged_attn_workspace(ref(pool()), ref(seqs(n_seq=1, n_col=2000)), ref(desc()), C.byref(b)) == ssd.OK
    assert b.value > a.value


# ---------------------------------------------------------------- blocks

@pytest.mark.parametrize("load", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=(1 << 20) + 1), INVALID), (dict(first=-1), INVALID), (dict(layers=-1), INVALID),
    (dict(first=1), INVALID), (dict(first=2**31 - 1), INVALID), (dict(d=None), INVALID), (dict(ids=None), INVALID),
    (dict(ids=MB + 2), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=2 * MB + 8), UNSUPPORTED),
    (dict(d=rows("pages", dtype=5)), INVALID), (dict(d=rows("pages", row=-64)), INVALID),
    (dict(d=rows("pages", row=65)), UNSUPPORTED), (dict(k=100 * MB + 4096), INVALID), (dict(v=100 * MB - 64), INVALID),
    (dict(v=200 * MB), INVALID)])
def test_blocks_refuse(load, kw, status):
    v = dict(ids=MB, n=6, first=0, layers=2, d=rows("pages"), k=2 * MB, v=3 * MB)
    v.update(kw)
    f = paged._ops().ssd_pages_load if load else paged._ops().ssd_pages_store
    assert f(ref(pool()), v["ids"], v["n"], v["first"], v["layers"], ref(v["d"]), v["k"], v["v"], None) == status


def test_values_that_are_read_back_may_not_overlap():
    def load(d, k, v, ids=MB):
        return paged._ops().ssd_pages_load(ref(pool()), ids, 6, 0, 2, ref(d), k, v, None)
    size = 2 * 6 * 4 * 2048 * 2
    for kw in (dict(row=0), dict(row=56), dict(head=64), dict(seq=2048), dict(layer=0)):
        assert load(rows("pages", **kw), 2 * MB, 9 * MB) == INVALID, kw
    assert load(rows("pages"), 2 * MB, 2 * MB) == load(rows("pages"), 2 * MB, 2 * MB + size - 16) == INVALID
    assert load(rows("pages"), 2 * MB, 9 * MB, ids=2 * MB + 16) == INVALID


def test_calls_over_nothing_do_nothing():
    L, p = paged._ops(), ref(pool())
    for f in (L.ssd_pages_store, L.ssd_pages_load):
        assert f(p, None, 0, 0, 2, ref(rows("pages")), None, None, None) == ssd.OK
        assert f(p, MB, 6, 2, 0, ref(rows("pages")), None, None, None) == ssd.OK


# ---------------------------------------------------------------- sequences

def commit(p=None, s=None, tail=None, kt=2 * MB, vt=3 * MB, fresh=None, kn=4 * MB, vn=5 * MB, path=MB, ld=8, most=8,
           path_len=MB, window=0, sinks=0, full=MB, work=16 * MB, size=1 << 40):
    return paged._ops().ssd_pages_commit(ref(p or pool()), ref(s or seqs()), ref(tail or rows("tail")), kt, vt,
                                         ref(fresh or rows("new")), kn, vn, path, ld, most, path_len, window, sinks, full,
                                         work, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(tail=rows("tail", rows=38)), INVALID), (dict(tail=rows("tail", rows=1 << 30)), INVALID),
    (dict(tail=rows("tail", dtype=ssd.F32)), INVALID), (dict(tail=rows("tail", row=0)), INVALID),
    (dict(tail=rows("tail", head=64)), INVALID), (dict(tail=rows("tail", row=66)), UNSUPPORTED),
    (dict(fresh=rows("new", rows=0)), INVALID), (dict(fresh=rows("new", rows=65)), INVALID),
    (dict(fresh=rows("new", row=-256)), INVALID), (dict(fresh=rows("new", head=60)), UNSUPPORTED),
    (dict(kt=None), INVALID), (dict(vn=None), INVALID), (dict(vt=3 * MB + 2), UNSUPPORTED), (dict(vt=2 * MB), INVALID),
    (dict(kn=2 * MB), INVALID), (dict(vn=3 * MB - 16), INVALID), (dict(path=None), INVALID), (dict(path=MB + 1), INVALID),
    (dict(ld=7), INVALID), (dict(most=65, ld=65), INVALID), (dict(most=-1), INVALID), (dict(path_len=None), INVALID),
    (dict(full=None), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(work=None), INVALID),
    (dict(work=16 * MB + 8), CAPACITY), (dict(size=64), CAPACITY)])
def test_commit_refuses(kw, status):
    assert commit(**kw) == status


def test_commit_refuses_more_workgroups_than_a_grid_holds():
    big = dict(p=pool(n_layer=4096), s=seqs(n_seq=4096), tail=rows("tail", layer=4096 * 4 * 39 * 64),
               fresh=rows("new", layer=4096 * 8 * 256), kt=1 << 44, vt=1 << 45, kn=1 << 46, vn=1 << 47)
    assert commit(**big) == CAPACITY
    assert b"grid" in paged._ops().ssd_last_error()


@pytest.mark.parametrize("kw", [dict(count=None), dict(got=None), dict(count=MB + 1), dict(got=MB + 2)])
def test_take_refuses(kw):
    v = dict(count=MB, got=2 * MB)
    v.update(kw)
    assert paged._ops().ssd_pages_take(ref(pool()), ref(seqs()), v["count"], v["got"], 16 * MB, 1 << 40, None) == INVALID
    assert paged._ops().ssd_pages_take(ref(pool()), ref(seqs()), MB, MB, 16 * MB, 8, None) == CAPACITY
    assert paged._ops().ssd_pages_compact(ref(pool()), ref(seqs()), None, 16 * MB, 1 << 40, None) == INVALID
    assert paged._ops().ssd_pages_compact(ref(pool()), ref(seqs()), MB, 16 * MB, 8, None) == CAPACITY


@pytest.mark.parametrize("kw,status", [
    (dict(n_page=0), INVALID), (dict(page_rows=48), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(layers=0), INVALID),
    (dict(heads=0), INVALID), (dict(parents=None), INVALID), (dict(parents=MB + 2), INVALID), (dict(tail=rows("tail", rows=31)), INVALID),
    (dict(tail=rows("tail", seq=64)), INVALID), (dict(tail=rows("tail", row=65)), UNSUPPORTED), (dict(kt=None), INVALID),
    (dict(vt=2 * MB + 64), INVALID), (dict(page_rows=64), INVALID)])
def test_fork_refuses(kw, status):
    v = dict(n_page=20, page_rows=32, parents=MB, tail=rows("tail"), layers=2, heads=4, head_dim=64, kt=2 * MB, vt=3 * MB)
    v.update(kw)
    assert paged._ops().ssd_pages_fork(ref(seqs()), v["n_page"], v["page_rows"], v["parents"], ref(v["tail"]), v["layers"],
                                       v["heads"], v["head_dim"], v["kt"], v["vt"], None) == status


def test_refusals_carry_a_message():
    assert commit(tail=rows("tail", rows=38)) == INVALID
    assert b"page_rows + new rows - 1" in paged._ops().ssd_last_error()


def test_the_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    data, scale = torch.zeros((1, 2, 1, 2, 1024), dtype=torch.uint8), torch.zeros((1, 2, 1, 2))
    with pytest.raises(ssd.SSDError):
        paged.Pages(data, scale, 32)
    x = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ssd.SSDError):
        paged.pages_fork(x, x.view(2, 1), x, x, data, data, 32)
    with pytest.raises(ssd.SSDError):
        paged.pages_store(data, x, data, data)
    with pytest.raises(ssd.SSDError):
        paged.paged_attention(data, data, x, x, x, x, x, x)


def test_the_binding_refuses_numbers_past_32_bits():
    # (they would lose their upper bits on the way: a window of 2^32 rows would be none)
    pages = object.__new__(paged.Pages)
    pages.kind = ()
    for kw in (dict(window=1 << 32), dict(window=(1 << 32) + 8), dict(sinks=1 << 31), dict(layer=1 << 32), dict(layer=-1)):
        with pytest.raises(ssd.SSDError, match=next(iter(kw))):
            paged.paged_attention(None, pages, None, None, None, None, None, None, **kw)
    with pytest.raises(ssd.SSDError, match="layer"):
        paged.pages_store(pages, None, None, None, layer=1 << 32)
    for kw in (dict(window=1 << 32), dict(sinks=-1)):
        with pytest.raises(ssd.SSDError, match=next(iter(kw))):
            paged.pages_commit(pages, *[None] * 9, **kw)
    with pytest.raises(ssd.SSDError, match="page_rows"):
        paged.pages_fork(*[None] * 6, (1 << 32) + 32)


# ---------------------------------------------------------------- the plain forms

def test_the_order_of_bytes_names_every_place_once():
    for r in (32, 64, 128):
        for d in (32, 64, 128):
            for p in M.places(r, d):
                assert sorted(p.reshape(-1).tolist()) == list(range(r * d))


def test_codes_are_the_nearest():
    grid = np.concatenate([-M.GRID, M.GRID])
    y = np.random.default_rng(0).uniform(-448, 448, 3000) * np.random.default_rng(1).choice([1, 1e-2, 1e-4], 3000)
    assert np.array_equal(np.abs(M.nearest_e4m3(y) - y), np.abs(grid[None] - y[:, None]).min(1))
    for code in M.TOP:
        block = np.random.default_rng(2).standard_normal((32, 64)).astype(np.float32)
        codes, scale = M.quantize(block, code)
        a = np.abs(block).max()
        assert np.abs(codes).max() == M.TOP[code] and abs(scale * M.TOP[code] - a) <= 2.0 ** -23 * a
        step = a / 254 if code == "int8" else np.maximum(np.abs(block) / 16, a / 448 * 2.0 ** -10)
        assert (np.abs(codes * scale - block) <= step * (1 + 1e-6)).all()
        raw = M.to_bytes(codes, code)
        assert np.array_equal(M.from_bytes(raw, code), codes)
