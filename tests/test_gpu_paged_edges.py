"""The paged cache's operators at calls that their documentation allows and a program seldom makes."""
import math

import numpy as np
import pytest

import paged_model as M
import test_gpu_paged as P

pytestmark = pytest.mark.gpu
env = P.env


# ---------------------------------------------------------------- commits

@pytest.mark.parametrize("dtype,code,rows,d,t", [("bf16", "int8", 32, 64, 2), ("f32", "int8", 32, 32, 7),
                                                 ("bf16", "e4m3", 64, 128, 1), ("f32", "e4m3", 128, 64, 33)])
def test_paths_that_name_rows_twice(env, dtype, code, rows, d, t):
    """Paths of 64 entries that name the same rows again: as many count as there are new rows, so the open page's rows stay in
    the tail (page_rows + t - 1 rows, the least there may be) until its codes are made of them."""
    torch, paged, _ = env
    b = 4
    batch = P.Batch(env, b, 6, 20, t, dtype, code, d=d, rows=rows)
    assert batch.kt.shape[3] == rows + t - 1
    for x in (batch.length, batch.host.length):
        x[:] = 0
    rng = np.random.default_rng(t)
    host_commit = batch.host.commit
    batch.host.commit = lambda path, n, *rest: host_commit([p[:t] for p in path], n, *rest)
    for step in range(3 * rows // t + 2):
        path = [(list(range(t)) * 64)[:64], [t - 1] * 64, rng.integers(0, t, 64).tolist(), list(range(t)) + [0] * (64 - t)]
        batch.step(path, [64, 40 + t, 64, max(t - 1, 1)])
    batch.open_rows()
    assert batch.host.length[0] == (3 * rows // t + 2) * t


# ---------------------------------------------------------------- attention

def sized(c, **kw):
    """(out, sum of weights times |values|) in 64 bits, and the largest sum of |q_i k_i| scale."""
    f = lambda x: x.double().numpy()  # noqa: E731
    hk, hv = c.host()
    call = lambda g: M.attention(f(c.q), c.table, c.lens, (hk, g(hv)), (f(c.kt), g(f(c.vt))), (f(c.kn), g(f(c.vn))),  # noqa: E731
                                 c.rows, c.anc, **kw)
    ref, _, big, _ = call(lambda x: x)
    return ref, call(np.abs)[0], big


def agrees(c, **kw):
    """Every element of out against its own terms' size: weights are off by twice a score's error, the sums' roundings and
    their own rounding (2^-11 or 2^-22), the result by its type's.  (As in test_gpu_paged; weights of the
    same 32 rows are near each other here, so that what is lost of those far below the largest does not count.)"""
    out, _ = c.run(**kw)
    ref, size, big = sized(c, **kw)
    off = size * (2 * P.EPS * (3 * c.d + 8) * big + 64 * P.EPS + (2.0 ** -11 if c.dtype == "bf16" else 2.0 ** -22))
    if c.dtype == "bf16":
        off = off + 2.0 ** -8 * (np.abs(ref) + off)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = (np.abs(got - ref) / np.maximum(off, 1e-300)).max()
    assert worst <= 1, worst


def alike(env, dtype, code, pages, seed=0):
    """One sequence of `pages` full pages of 32 rows and an open one, whose scores lie near each other.  (Every third of
    the first 18 pages is the same wave's.)"""
    c = P.Case(env, dtype, code, 1, 1, 2, 1, 64, 32, [32 * pages + 5], seed=seed, cols=pages + 1)
    assert pages < 24
    c.q *= 0.1
    return c


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_of_large_values_without_weight_take_no_bits_from_others(env, dtype, code):
    """Value scales 2^30 apart; the pages of the large ones have scores far below the others'."""
    for first in (0, 1):
        c = alike(env, dtype, code, 18)
        c.q = c.q.abs() + 0.1
        raw = c.data.view(1, -1, 1, 2, 32 * 64)
        for col in range(18):
            if (col // 3 + first) % 2 == 0:
                page = c.table[0, col]
                raw[0, page, 0, 0] = int(M.to_bytes(np.array([-120.0]), code)[0])
                c.scale[0, page, 0, 0] = 1.0
                c.scale[0, page, 0, 1] *= 2.0 ** 30
        # (small rows of the model's type, too)
        c.vt *= 2.0 ** -6
        c.vn *= 2.0 ** -6
        agrees(c)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_values_behind_the_window_take_no_bits_from_others(env, dtype, code):
    """The first page's scale is 2^30 times the others', for a row behind the window; its other rows are 0."""
    c = alike(env, dtype, code, 18)
    _, pv = M.places(32, 64)
    page = c.table[0, 0]
    zero, top = (int(M.to_bytes(np.array([x]), code)[0]) for x in (0.0, M.TOP[code]))
    raw = c.data.view(1, -1, 1, 2, 32 * 64)
    raw[0, page, 0, 1] = zero
    raw[0, page, 0, 1, pv[0]] = top
    c.scale[0, page, 0, 1] *= 2.0 ** 30
    agrees(c, window=c.lens[0])  # (row 0 is not seen)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_whose_values_are_powers_apart(env, dtype, code):
    """Each page's rows count to their own size: a page of values 2^-30 of its neighbours', in dims where those are 0."""
    c = alike(env, dtype, code, 18)
    _, pv = M.places(32, 64)
    zero = int(M.to_bytes(np.array([0.0]), code)[0])
    raw = c.data.view(1, -1, 1, 2, 32 * 64)
    for col in range(18):
        page, small = c.table[0, col], col // 3 % 2
        raw[0, page, 0, 1, (pv[:, :32] if small else pv[:, 32:]).reshape(-1)] = zero
        if not small:
            c.scale[0, page, 0, 1] *= 2.0 ** 30
    c.vt[..., 32:] = 0
    c.vn[..., 32:] = 0
    agrees(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("own,scale", [(2.0 ** 110, 0.022), (2.0 ** 80, 1e-14), (2.0 ** 66, 1e-20), (2.0 ** 66, 1e-38)])
def test_large_open_and_new_rows_beside_pages(env, dtype, own, scale):
    """(The wave that takes the open and new rows takes a page, too, from the 22nd on.)"""
    c = alike(env, dtype, "int8", 23)
    c.scale[0, :, :, 1] = scale
    c.vt *= own
    c.vn *= own
    c.check()
    # as many digits where the large ones are of other dims
    c.vt[..., 32:] = 0
    c.vn[..., 32:] = 0
    agrees(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_in_pages_at_the_windows_edge(env, dtype):
    """Rows of next to no weight in a page whose value scale is NaN: NaN where one of them is seen."""
    c = P.Case(env, dtype, "int8", 1, 2, 2, 1, 64, 32, [70])
    c.q = c.q.abs() + 1
    page = c.table[0, 0]
    c.data.view(1, -1, 1, 2, 32 * 64)[0, page, 0, 0] = 8
    c.scale[0, page, 0, 0] = 1.0
    c.scale[0, page, 0, 1] = math.nan
    for window, nan in ((70, [True, True]), (60, [True, True]), (40, [True, False]), (39, [False, False])):
        out, lse = c.run(window=window)
        assert lse.isfinite().all()
        assert [bool(out[0, t].isnan().all()) for t in (0, 1)] == nan, window
        assert [bool(out[0, t].isfinite().all()) for t in (0, 1)] == [not x for x in nan], window


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_at_the_windows_edge_behind_rows_of_more_weight(env, dtype):
    """(40 queries leave the first pages to one wave: the first rows' page, then the one at the window's edge.)"""
    c = P.Case(env, dtype, "int8", 1, 40, 2, 1, 64, 32, [300])
    c.q = c.q.abs() + 1
    page = c.table[0, 1]
    c.data.view(1, -1, 1, 2, 32 * 64)[0, page, 0, 0] = 8
    c.scale[0, page, 0, 0] = 1.0
    c.scale[0, page, 0, 1] = math.nan
    out, lse = c.run(window=260, sinks=1)  # query t sees rows from 41 + t on: of page 1 up to t = 22
    assert lse.isfinite().all() and out[0, :23].isnan().all() and out[0, 23:].isfinite().all()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d,lens", [(1, 64, [740, 37]), (3, 128, [740, 64]), (40, 64, [100, 0]), (17, 128, [20, 740]),
                                      (2, 32, [9000]), (33, 128, [3000])])
def test_values_up_to_the_largest(env, dtype, code, t, d, lens):
    """Results are finite where values are, whatever their sums were: open and new rows, pages, or both near the type's
    largest, in one part of a sequence and in many."""
    print(dtype, code, t, d, lens, flush=True)
    for own, top in ((2.0 ** 125, 0.0), (1.0, 2.0 ** 120), (2.0 ** 125, 2.0 ** 120)):
        c = P.Case(env, dtype, code, len(lens), t, 4, 2, d, 32, lens)
        c.q *= 0.2
        c.vt *= own
        c.vn *= own
        assert c.vt.isfinite().all() and c.vn.isfinite().all()
        if top:
            c.scale[0, ::2, :, 1] *= top / P.M.TOP[code]
        c.check()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_bfloat16_results_are_off_by_their_own_rounding(env, code):
    """What a result near 0 shows: weights of cached rows hold 20 bits (cut off, so off by 2^-19), twice that where their sum
    divides them.  Scores are small, so they add next to nothing."""
    for t, h, g, d in ((4, 8, 8, 64), (3, 16, 4, 128), (9, 16, 4, 32)):
        c = P.Case(env, "bf16", code, 2, t, h, g, d, 32, [96, 64])
        c.q *= 0.02
        c.kn *= 0.1
        c.vn *= 0.1
        out, _ = c.run()
        ref, size, big = sized(c)
        off = size * (2 * P.EPS * (3 * d + 8) * big + 64 * P.EPS + 2 * 2.0 ** -19)
        off = off + 2.0 ** -8 * (np.abs(ref) + off)
        worst = (np.abs(out.double().cpu().numpy() - ref) / off).max()
        assert worst <= 1, (t, worst)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,h,g", [(3, 2, 2), (1, 4, 4), (5, 8, 2), (9, 4, 2)])
def test_results_depend_on_no_other_sequence(env, dtype, t, h, g):
    """Bitwise: fewer queries than a tile has columns, a wave that takes open rows and pages behind them, and a first
    sequence whose first query scores those rows from far below to far above the others'."""
    c = P.Case(env, dtype, "int8", 2, t, h, g, 64, 32, [5, 740], cols=24)
    c.kt = c.kt.abs()
    c.kn = c.kn.abs()
    c.scale[0, :, :, 0] *= 4
    want = None
    for q in (0.0, -100.0, 100.0, 1e30, math.inf, math.nan):
        c.q[0, 0, 0] = q
        got = [x[1] for x in c.run()]
        want = want or got
        assert all(c.torch.equal(x, y) for x, y in zip(got, want)), q


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_of_rows_whose_score_is_minus_infinity(env, dtype, bad):
    """Such a row counts as one that is not seen, so its value may be anything."""
    c = P.Case(env, dtype, "int8", 1, 2, 2, 1, 64, 32, [40])
    c.q = c.q.abs() + 1
    c.kt[0, 0, 33 % c.kt.shape[2]] = -math.inf
    c.kn[0, 0, 0] = -math.inf
    want = c.run()
    assert all(x.isfinite().all() for x in want)
    c.vt[0, 0, 33 % c.kt.shape[2]] = bad
    c.vn[0, 0, 0, 5:9] = bad
    got = c.run()
    assert all(c.torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_page_scales_that_are_not_finite(env, dtype, code, bad):
    """All of a head's keys (out and lse) or values (out) of the page are NaN for queries that see a row of it."""
    for which in (0, 1):
        c = P.Case(env, dtype, code, 1, 2, 4, 2, 64, 32, [740], cols=24)
        c.data[0, :, 1, 0] = int(M.to_bytes(np.array([-4.0]), code)[0])  # (scores of one sign: with infinity all -infinity)
        c.q = c.q.abs() + 1
        want, lse = c.run()
        c.scale[0, c.table[0, 21], 1, which] = bad
        got, l2 = c.run()
        assert got[0, :, 2:].isnan().all() and c.torch.equal(got[0, :, :2], want[0, :, :2])
        assert l2[0, :, 2:].isnan().all() if which == 0 else c.torch.equal(l2, lse)
        assert c.torch.equal(l2[0, :, :2], lse[0, :, :2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("others", [1.0, 2.0 ** 30])
def test_queries_with_infinite_elements(env, dtype, code, others):
    """Every score is infinite, of the sign that the key's element gives it, or NaN."""
    c = P.Case(env, dtype, code, 1, 3, 2, 1, 64, 32, [100])
    raw = c.data.view(1, -1, 1, 2, 32 * 64)
    pk, _ = M.places(32, 64)
    for x in (c.kt, c.kn):
        x[..., 3] = 2.0
    for page in c.table[0, :3]:
        raw[0, page, 0, 0, pk[:, 3]] = int(M.to_bytes(np.array([5.0]), code)[0])
    c.q *= others
    want, lse = c.run()
    assert want.isfinite().all()
    c.q[0, 0, 0, 3] = -math.inf           # all rows' scores -infinity: no row is seen
    c.q[0, 1, 0, 3] = math.inf            # all +infinity
    c.q[0, 2, 0, 2:4] = math.inf          # some +infinity, some NaN
    got, l2 = c.run()
    assert not got[0, 0, 0].any() and l2[0, 0, 0] == -math.inf
    assert got[0, 1:, 0].isnan().all() and l2[0, 1:, 0].isnan().all()
    assert c.torch.equal(got[:, :, 1], want[:, :, 1]) and c.torch.equal(l2[:, :, 1], lse[:, :, 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d,code", [(4, 64, "int8"), (20, 64, "e4m3"), (20, 128, "int8")])
def test_large_values_that_are_not_seen_change_nothing(env, dtype, t, d, code):
    """Bitwise: a padded place's rows, and those of the ring that are not the sequence's."""
    c = P.Case(env, dtype, code, 2, t, 4, 2, d, 32, [740, 95], tree=True, cols=24)
    for row in c.anc:
        row[t - 1] = 0
    want = c.run()
    for bad in (2.0 ** 100, -(2.0 ** 127)):
        c.kn[:, t - 1] = bad
        c.vn[:, t - 1] = bad
        ring = c.kt.shape[2]
        for i, n in enumerate(c.lens):
            for p in range(ring):
                if p not in {j % ring for j in range(n // 32 * 32, n)}:
                    c.kt[i, :, p] = c.vt[i, :, p] = bad
        assert all(c.torch.equal(x, y) for x, y in zip(c.run(), want)), bad


# ---------------------------------------------------------------- the binding

def test_numbers_count_by_their_value(env):
    """Whole numbers of any kind, a tensor's entry whose value changes between calls among them."""
    torch, paged, _ = env
    batch = P.grown(env)
    ids = batch.i32([0, 1])
    like = paged.pages_load(batch.pages, ids, layer=1)
    which = torch.tensor(1)
    for layer in (np.int64(1), which):
        assert all(torch.equal(x, y) for x, y in zip(paged.pages_load(batch.pages, ids, layer=layer, n_layer=np.int32(1)), like))
    which.zero_()
    for x, y in zip(paged.pages_load(batch.pages, ids, layer=which, n_layer=1), paged.pages_load(batch.pages, ids, layer=0)):
        assert torch.equal(x[:1], y[:1])
    before = batch.pages.data.clone()
    paged.pages_store(batch.pages, ids.flip(0), *like, layer=np.int64(1))
    assert torch.equal(batch.pages.data[0], before[0]) and torch.equal(batch.pages.data[1, 1], before[1, 0])
    parents = batch.i32([0, 0, 2, 3, 4, 5, 6, 7])
    paged.pages_fork(*batch.seqs(), parents, batch.kt, batch.vt, np.int64(32))
    batch.host.fork(parents.tolist())
    batch.same()
    kn = torch.zeros((2, 8, 8, 2, 64), device="cuda").bfloat16()
    paged.pages_commit(batch.pages, *batch.seqs(), batch.kt, batch.vt, kn, kn, batch.i32([[0, 1]] * 8), batch.i32([2] * 8),
                       window=np.int64(40), sinks=np.int16(1))
    batch.host.commit([[0, 1]] * 8, [2] * 8, 8, 40, 1)
    batch.same()
    for bad in (1.0, "1", None):
        with pytest.raises(TypeError):
            paged.pages_store(batch.pages, ids, *like, layer=bad)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_pages_past_32_bits_are_the_ones_that_are_named(env, code):
    """A pool of 6 GB whose last page of the last layer, 4 GB and more from the first, and first page get rows of their own:
    written, read back and attended to, each to half a code of its own largest magnitude."""
    torch, paged, _ = env
    g, rows, d, n = 2, 32, 64, 370_000
    data = torch.zeros((2, n, g, 2, rows * d), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((2, n, g, 2), device="cuda")
    pages = paged.Pages(data, scale, rows, code)
    assert data[1, n - 1].data_ptr() - data.data_ptr() > 1 << 32
    k, v = P.blocks(torch, "bf16", 2, 2, g, rows, d, seed=5)
    ids = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    paged.pages_store(pages, ids, k.cuda(), v.cuda())
    wanted, scales = P.host_pages(k, v, code)
    at = [n - 1, 0]
    assert np.array_equal(M.from_bytes(data[:, at].cpu().numpy(), code), M.from_bytes(wanted, code))
    assert np.array_equal(scale[:, at].cpu().numpy(), scales)
    assert (scale.count_nonzero(dim=(2, 3)) > 0).sum() == 4  # (no other page)
    kk, vv = paged.pages_load(pages, ids, torch.float32)
    for x, y, p in ((kk, k, 0), (vv, v, 1)):
        host = M.page_values(wanted, scales, rows, d, code)[p]
        assert torch.equal(x.cpu(), torch.from_numpy(host.astype(np.float32)))
        top = y.float().abs().amax((3, 4), keepdim=True)
        # (half a code, or half of e4m3's step at the top, 16 of 448; and the roundings of r, x r and the value)
        half = top / 254 if code == "int8" else top * 16 / 448
        assert ((x.cpu() - y.float()).abs() <= half * (1 + 2.0 ** -10)).all()
    # attention over the last layer's last page gives what a pool of this page alone gives
    c = P.Case(env, "bf16", code, 1, 2, 2, g, d, rows, [rows])
    x = [getattr(c, w).cuda() for w in ("kt", "vt", "kn", "vn")]
    length = torch.tensor([rows], dtype=torch.int32, device="cuda")
    for i, page in enumerate(at):
        small = paged.Pages(data[1:, page:page + 1].contiguous(), scale[1:, page:page + 1].contiguous(), rows, code)
        outs = [paged.paged_attention(c.q.cuda(), p, torch.tensor([[where, -1]], dtype=torch.int32, device="cuda"), length, *x,
                                      layer=layer) for p, where, layer in ((pages, page, 1), (small, 0, 0))]
        assert outs[0].isfinite().all() and torch.equal(*outs), page
