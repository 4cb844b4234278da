"""The paged cache's operators against the plain host forms of paged_model.

Attention's tolerances, set from the arithmetic (eps = 2^-24, half a step of float32).  A score: codes are exact; a
float32 query is three parts, so 3 D products are added in float32, and the scale, the query's power of two and the
softmax's take 8 roundings: off by (3 D + 8) eps S with S the largest sum of |q_i k_i| scale; a weight by twice that,
relatively, and the weighted sum of the values, whose largest magnitude is vmax, by that times vmax and the
roundings of sums and rescalings (64 eps).  Weights are rounded for the product with the values: bfloat16 calls to
float16, 2^-11 relative; float32 calls to two of those, 2^-22, and both below 2^-32 of the largest to
its last place, 2^-32 a row.  A bfloat16 result is rounded, 2^-8 relative."""
import math

import numpy as np
import pytest

import paged_model as M

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2308_04623_amd import paged, ssd
    assert torch.cuda.is_available()
    return torch, paged, ssd


def tolerance(dtype, d, big, vmax, rows):
    tol = vmax * (2 * EPS * (3 * d + 8) * big + 64 * EPS + rows * 2.0 ** -32)
    return tol + vmax * (2.0 ** -11 + 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22)


class Case:
    """A batch whose pages hold normal rows (as codes), on the host and on the device."""

    def __init__(self, env, dtype, code, b, t, h, g, d, rows, lens, seed=0, cols=None, spare=2, layers=1, ring=None,
                 tree=False):
        self.torch, self.paged = env[0], env[1]
        torch = self.torch
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.code, self.rows, self.d = dtype, code, rows, d
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        rn = lambda *s: torch.randn(s, generator=gen).to(self.dt)  # noqa: E731
        self.lens = lens
        held = [max(n, 0) // rows for n in lens]
        cols = max(held + [1]) + 1 if cols is None else cols
        n_page = sum(held) + spare
        ids = torch.randperm(n_page, generator=gen).tolist()
        self.table = np.full((b, cols), -1, np.int64)
        at = 0
        for i, n in enumerate(held):
            self.table[i, :n] = ids[at:at + n]
            at += n
        top = M.TOP[code]
        raw = (torch.randn((layers, n_page, g, 2, rows * d), generator=gen) * top / 4).clamp(-top, top)
        self.data = raw.round().add(128).to(torch.uint8) if code == "int8" else raw.to(torch.float8_e4m3fn).view(torch.uint8)
        self.scale = (4 / top) * (0.5 + torch.rand((layers, n_page, g, 2), generator=gen))
        ring = rows + t if ring is None else ring
        self.q = 2 * rn(b, t, h, d)
        self.kt, self.vt, self.kn, self.vn = rn(b, g, ring, d), rn(b, g, ring, d), rn(b, t, g, d), rn(b, t, g, d)
        self.anc = None
        if tree:
            self.anc = [[0] * t for _ in range(b)]
            for row in self.anc:
                for j in range(t):
                    up = int(torch.randint(0, j, (1,), generator=gen)) if j else 0
                    row[j] = (row[up] if j else 0) | 1 << j

    def host(self, layer=0):
        return M.page_values(self.data[layer].numpy(), self.scale[layer].numpy(), self.rows, self.d, self.code)

    def masks(self):
        if self.anc is None:
            return None
        signed = [[m - (1 << 64) if m >> 63 else m for m in row] for row in self.anc]
        return self.torch.tensor(signed, dtype=self.torch.int64).cuda()

    def device(self):
        torch = self.torch
        pages = self.paged.Pages(self.data.cuda(), self.scale.cuda(), self.rows, self.code)
        return pages, torch.tensor(self.table, dtype=torch.int32).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda()

    def run(self, put=lambda name, x: x.cuda(), layer=0, **kw):
        pages, table, length = self.device()
        x = {n: put(n, getattr(self, n)) for n in ("q", "kt", "vt", "kn", "vn")}
        out = self.paged.paged_attention(x["q"], pages, table, length, x["kt"], x["vt"], x["kn"], x["vn"], layer=layer,
                                         anc=self.masks(), return_lse=True, **kw)
        self.torch.cuda.synchronize()
        return out

    def want(self, layer=0, **kw):
        f = lambda x: x.double().numpy()  # noqa: E731
        return M.attention(f(self.q), self.table, self.lens, self.host(layer), (f(self.kt), f(self.vt)),
                           (f(self.kn), f(self.vn)), self.rows, self.anc, **kw)

    def check(self, put=lambda name, x: x.cuda(), layer=0, **kw):
        out, lse = self.run(put, layer, **kw)
        ref, rl, big, vmax = self.want(layer, **{k: v for k, v in kw.items() if k != "out"})
        got = out.double().cpu().numpy()
        n = max(self.lens) + self.q.shape[1]
        assert np.isfinite(got).all()
        assert np.abs(got - ref).max() <= tolerance(self.dtype, self.d, big, vmax, n)
        got_l, live = lse.double().cpu().numpy(), np.isfinite(rl)
        assert np.array_equal(np.isneginf(got_l), np.isneginf(rl))
        if live.any():
            bound = (3 * self.d + 8) * EPS * big + 64 * EPS * (1 + np.abs(rl[live]).max())
            assert np.abs(got_l[live] - rl[live]).max() <= bound
        return out, lse


SHAPES = [
    # b, t, h, g, d, rows, lens
    (1, 1, 1, 1, 32, 32, [0]), (1, 1, 1, 1, 64, 32, [1]), (2, 1, 4, 4, 32, 32, [31, 32]), (3, 2, 6, 2, 64, 64, [63, 64, 65]),
    (5, 1, 20, 20, 64, 32, [0, 200, 333, -1, 96]), (2, 5, 8, 2, 128, 64, [257, 128]), (3, 3, 4, 1, 64, 128, [500, 127, 129]),
    (1, 64, 2, 1, 64, 32, [95]), (2, 17, 3, 3, 32, 128, [400, 3]), (1, 1, 25, 25, 64, 32, [2100]), (2, 8, 32, 2, 128, 32, [70, 700]),
    (1, 33, 40, 1, 32, 64, [190]), (7, 1, 2, 2, 128, 128, [0, 1, 127, 128, 300, 1000, -1])]


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_against_64_bits(env, dtype, code, shape):
    print(dtype, code, shape, flush=True)
    Case(env, dtype, code, *shape, seed=len(shape[6])).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 7, 4, 2, 64, 32, [0, 33, 100]), (2, 64, 2, 2, 32, 64, [70, 1]),
                                   (4, 15, 8, 2, 128, 32, [31, 64, -1, 129]), (1, 63, 1, 1, 64, 128, [300])])
def test_trees(env, dtype, shape):
    print(dtype, shape, flush=True)
    Case(env, dtype, "int8", *shape, tree=True).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_that_leave_rows_empty_or_name_rows_past_the_last(env, dtype):
    c = Case(env, dtype, "int8", 4, 5, 4, 2, 64, 32, [0, 40, 0, -1], tree=True)
    c.anc = [[0, 1, 0, 8, 31], [0, 2, 4, 0, 1], [1 << 63, (1 << 63) | 1, 32, 0, 7], [31] * 5]
    out, lse = c.check()
    assert not out[0, 0].any() and not out[0, 2].any() and not out[2, 0].any() and not out[2, 2].any() and not out[3].any()
    assert lse[2, 3].isneginf().all() and out[1, 0].any()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(3, 0), (32, 0), (33, 1), (64, 4), (100, 40), (129, 0), (500, 3), (1 << 30, 5),
                                          (50, 1 << 30), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("rows", [32, 64, 128])
def test_windows_and_sinks(env, code, window, sinks, rows):
    print(code, window, sinks, rows, flush=True)
    for tree in (False, True):
        c = Case(env, "bf16", code, 4, 3, 4, 2, 64, rows, [0, 31, 130, 517], seed=window % 1000, tree=tree)
        # pages that no query sees were given back, or hold NaN
        for i, n in enumerate(c.lens):
            for col in range(n // rows):
                if col * rows >= sinks and (col + 1) * rows <= n - window + 1:
                    if col % 2:
                        c.table[i, col] = -1
                    else:
                        c.scale[0, c.table[i, col]] = math.nan
        c.check(window=window, sinks=sinks)


def test_windows_of_long_sequences_in_parts(env):
    c = Case(env, "bf16", "int8", 1, 2, 2, 1, 64, 32, [9000], cols=400)
    c.check(window=4000, sinks=70)
    c.check(window=0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_not_seen_may_hold_anything(env, dtype):
    for bad in (math.nan, math.inf, -math.inf):
        c = Case(env, dtype, "int8", 3, 4, 4, 2, 64, 32, [33, 0, 95], tree=True)
        c.anc = [[1, 3, 5, 0], [1, 2, 4, 0], [1, 3, 7, 0]]  # row 3: a padded place
        want = c.check()
        for x in (c.kn, c.vn):
            x[:, 3] = bad
        ring = c.kt.shape[2]
        for i, n in enumerate(c.lens):
            for p in range(ring):
                if p not in {j % ring for j in range(n // 32 * 32, n)}:
                    c.kt[i, :, p] = c.vt[i, :, p] = bad
        unused = sorted(set(range(c.data.shape[1])) - set(c.table[c.table >= 0].tolist()))
        c.scale[0, unused] = bad
        got = c.run()
        assert all(c.torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinity_reach_those_that_see_them(env, dtype):
    c = Case(env, dtype, "int8", 1, 3, 2, 2, 64, 32, [40], tree=True)
    c.anc = [[1, 3, 5]]
    out, lse = c.run()
    # a value of new row 1: dim 7 of head 0, for the query that sees it
    for bad in (math.nan, math.inf):
        c.vn[0, 1, 0, 7] = bad
        got, l2 = c.run()
        assert got[0, 1, 0, 7].isnan() and not got.isnan().sum() > 1 and c.torch.equal(l2, lse)
        got[0, 1, 0, 7] = out[0, 1, 0, 7]
        assert c.torch.equal(got, out)
    c.vn[0, 1, 0, 7] = 0
    # a key
    c.kn[0, 1, 0, 7] = math.nan
    got, l2 = c.run()
    assert got[0, 1, 0].isnan().all() and l2[0, 1, 0].isnan() and c.torch.equal(got[0, 2], out[0, 2])
    assert c.torch.equal(got[0, :, 1], out[0, :, 1]) and c.torch.equal(got[0, 0], out[0, 0])
    c.kn[0, 1, 0, 7] = 0
    # a page's scale: of the values, then of the keys of head 1
    for which in (1, 0):
        keep = c.scale.clone()
        c.scale[0, c.table[0, 0], 1, which] = math.nan
        got, l2 = c.run()
        assert got[0, :, 1].isnan().all() and c.torch.equal(got[0, :, 0], c.run()[0][0, :, 0])
        assert l2[0, :, 1].isnan().all() == (which == 0) and not got[0, :, 0].isnan().any()
        c.scale = keep
    # a query
    c.q[0, 2, 1, 3] = math.nan
    got, l2 = c.run()
    assert got[0, 2, 1].isnan().all() and l2[0, 2, 1].isnan() and got.isnan().sum() == 64


def test_scores_of_minus_infinity_count_as_rows_that_are_not_seen(env):
    for dtype in ("f32", "bf16"):
        c = Case(env, dtype, "int8", 1, 2, 1, 1, 32, 32, [3])
        want = c.run()
        c.kt[:] = 0
        c.kt[0, 0, 1] = -math.inf  # with all-positive queries
        c.q = c.q.abs() + 1
        c.kn[:] = 1
        out, lse = c.run()
        assert out.isfinite().all() and lse.isfinite().all()
        f = lambda x: x.double().numpy()  # noqa: E731
        x = f(c.q)[0, 1, 0] @ np.stack([f(c.kt)[0, 0, 0], f(c.kt)[0, 0, 2], f(c.kn)[0, 0, 0], f(c.kn)[0, 1, 0]]).T / math.sqrt(32)
        e = np.exp(x - x.max())
        v = np.stack([f(c.vt)[0, 0, 0], f(c.vt)[0, 0, 2], f(c.vn)[0, 0, 0], f(c.vn)[0, 1, 0]])
        assert np.abs(out[0, 1, 0].double().cpu().numpy() - e @ v / e.sum()).max() <= 2.0 ** -8 * np.abs(v).max()
        del want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_of_any_size(env, dtype):
    """Pages whose scales are powers apart, zeros among them; queries of any size; scores far apart."""
    c = Case(env, dtype, "int8", 2, 2, 4, 2, 64, 32, [200, 321])
    n = c.scale.shape[1]
    c.scale[0, :, :, 1] *= 2.0 ** (c.torch.arange(n).view(n, 1) * 3.0 % 40 - 30)
    c.scale[0, ::5, :, 1] = 0
    c.scale[0, 1::5, :, 0] = 0
    c.check()
    for by in (2.0 ** -90, 2.0 ** -40, 2.0 ** 40):
        c.scale[0, :, :, 0] /= by
        c.q *= by
        c.check()
        c.scale[0, :, :, 0] *= by
        c.q /= by
    c.vt.zero_(), c.vn.zero_()
    c.scale[0, :, :, 1] = 0
    assert not c.run()[0].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_apart(env, dtype):
    c = Case(env, dtype, "int8", 2, 3, 4, 2, 64, 32, [400, 37])
    c.q *= 8
    c.check()
    c.check(scale=0.0)
    c.check(scale=-0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(env, dtype):
    torch = env[0]
    c = Case(env, dtype, "e4m3", 3, 4, 4, 4, 64, 32, [100, 31, 5])
    want = c.check()
    qkv = torch.empty((3, 4, 3, 4, 64), dtype=c.dt, device="cuda")  # the projections' output as it comes
    for i, x in enumerate((c.q, c.kn, c.vn)):
        qkv[:, :, i] = x.cuda()
    tails = torch.zeros((2, 3, 40, 4, 72), dtype=c.dt, device="cuda")
    tails[:, :, 1:37, :, :64] = torch.stack([c.kt, c.vt]).transpose(2, 3).cuda()
    view = {"q": qkv[:, :, 0], "kn": qkv[:, :, 1], "vn": qkv[:, :, 2],
            "kt": tails[0, :, 1:37, :, :64].transpose(1, 2), "vt": tails[1, :, 1:37, :, :64].transpose(1, 2)}
    out = torch.full((4, 3, 5, 80), 7.0, dtype=c.dt, device="cuda")
    got = c.check(lambda name, x: view[name], out=out.transpose(0, 1)[:, :, :4, :64])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (out[:, :, 4] == 7).all() and (out[:, :, :, 64:] == 7).all()
    wide = torch.full((3, c.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    pages, table, length = c.device()
    wide[:, 2:2 + table.shape[1]] = table
    again = env[1].paged_attention(c.q.cuda(), pages, wide[:, 2:2 + table.shape[1]], length, c.kt.cuda(), c.vt.cuda(),
                                   c.kn.cuda(), c.vn.cuda())
    assert torch.equal(again, want[0])


def test_tables_that_name_no_page_and_lengths_past_the_table(env):
    c = Case(env, "f32", "int8", 3, 2, 2, 2, 64, 32, [200, 130, 64])
    c.table[0, 2] = -1
    c.table[0, 3] = c.data.shape[1]      # (none of the pool)
    c.table[1, 0] = -(1 << 31)
    c.table[2, 1] = (1 << 31) - 1
    c.check()
    c.table = c.table[:, :3]             # rows behind the last column are not seen
    c.check()
    c.table = c.table[:, :0]
    c.check()


def test_layers_and_pages_past_32_bits(env):
    """A pool of 6 GB: the last page of the last layer."""
    torch, paged, _ = env
    c = Case(env, "bf16", "int8", 1, 2, 2, 2, 64, 32, [32])
    n = 370_000
    data = torch.empty((2, n, 2, 2, 32 * 64), dtype=torch.uint8, device="cuda")
    scale = torch.empty((2, n, 2, 2), device="cuda")
    data[1, n - 1], scale[1, n - 1] = c.data[0, c.table[0, 0]].cuda(), c.scale[0, c.table[0, 0]].cuda()
    pages = paged.Pages(data, scale, 32)
    x = [getattr(c, k).cuda() for k in ("kt", "vt", "kn", "vn")]
    got = paged.paged_attention(c.q.cuda(), pages, torch.tensor([[n - 1, -1]], dtype=torch.int32, device="cuda"),
                                torch.tensor([32], dtype=torch.int32, device="cuda"), *x, layer=1)
    assert torch.equal(got, c.run()[0])
    ids = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    k, v = paged.pages_load(pages, ids, torch.bfloat16, layer=1)
    paged.pages_store(pages, ids.flip(0), k, v, layer=0)
    k2, v2 = paged.pages_load(pages, ids.flip(0), torch.bfloat16, layer=0, n_layer=1)
    assert torch.equal(k2.isnan(), k.isnan())
    assert (k2 - k).abs().max() <= 2.0 ** -8 * k.abs().max() + k.abs().max() / 127


def test_results_repeat_and_other_streams_give_them(env):
    torch, paged, _ = env
    c = Case(env, "bf16", "int8", 3, 2, 4, 4, 64, 32, [2000, 31, 700])
    want = c.run()
    side = torch.cuda.Stream()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(c.run(), want))
    side.wait_stream(torch.cuda.current_stream())
    assert all(torch.equal(a, b) for a, b in zip(c.run(stream=side), want))


def test_attention_in_a_graph_follows_lengths_and_tables(env):
    torch, paged, _ = env
    c = Case(env, "bf16", "int8", 2, 2, 4, 4, 64, 32, [320, 70], cols=40)
    pages, table, length = c.device()
    x = [getattr(c, k).cuda() for k in ("kt", "vt", "kn", "vn")]
    q = c.q.cuda()
    call = lambda: paged.paged_attention(q, pages, table, length, *x)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two, whose workspaces are their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for n in ([320, 70], [5, 64], [-1, 90], [300, 0]):
        length.copy_(torch.tensor(n, dtype=torch.int32))
        want = call()
        torch.cuda.synchronize()
        for graph, out in graphs:
            out.fill_(9)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), n


# ---------------------------------------------------------------- rows into pages and back

def blocks(torch, dtype, l, n, g, rows, d, seed=0):
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    return [(torch.randn((l, n, g, rows, d), generator=gen) * torch.exp2(6 * torch.rand((l, n, g, 1, 1), generator=gen))).to(dt)
            for _ in range(2)]


def host_pages(k, v, code):
    """bytes [L][N][G][2][rows d], scales [L][N][G][2] of blocks."""
    l, n, g, rows, d = k.shape
    pk, pv = M.places(rows, d)
    data, scale = np.zeros((l, n, g, 2, rows * d), np.uint8), np.zeros((l, n, g, 2), np.float32)
    for i in np.ndindex(l, n, g):
        for w, (x, p) in enumerate(((k, pk), (v, pv))):
            codes, scale[i][w] = M.quantize(x[i].float().numpy(), code)
            data[i][w][p] = M.to_bytes(codes, code)
    return data, scale


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(32, 32), (32, 64), (32, 128), (64, 64), (128, 32), (128, 128), (64, 128)])
def test_stored_bytes_and_their_values(env, dtype, code, rows, d):
    torch, paged, _ = env
    print(dtype, code, rows, d, flush=True)
    k, v = blocks(torch, dtype, 2, 3, 2, rows, d)
    k[0, 0, 0] = 0                                # nothing
    v[0, 1, 1] *= 2.0 ** -110                     # next to nothing
    v[1, 0, 0] = (v[1, 0, 0].float() * 2.0 ** -95).to(v.dtype)
    k[1, 1, 0, 5, 7] = math.nan
    v[1, 2, 1, rows - 1, d - 1] = -math.inf
    k[0, 2, 1] = k[0, 2, 1].sign()                # (one magnitude)
    pages = paged.Pages.empty(3, 5, 2, d, rows, code)
    ids = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    paged.pages_store(pages, ids, k.cuda(), v.cuda(), layer=1)
    data, scale = host_pages(k, v, code)
    got, got_s = pages.data[1:].cpu().numpy(), pages.scale[1:].cpu().numpy()
    want_v = M.from_bytes(data, code)
    assert np.array_equal(M.from_bytes(got[:, [4, 0, 2]], code), want_v)
    assert np.array_equal(got_s[:, [4, 0, 2]], scale, equal_nan=True)
    assert not pages.data[0].any() and not pages.data[1:, [1, 3]].any() and not pages.scale[0].any()
    ask = torch.tensor([2, -1, 0, 5, 4, 4, 1 << 30], dtype=torch.int32, device="cuda")
    for dt in (torch.float32, torch.bfloat16):
        kk, vv = paged.pages_load(pages, ask, dt, layer=1)
        assert kk.shape == (2, 7, 2, rows, d)
        hk, hv = M.page_values(got, got_s, rows, d, code)
        for x, h in ((kk, hk), (vv, hv)):
            h = torch.from_numpy(h[:, [2, 0, 0, 0, 4, 4, 0]].astype(np.float32)).to(dt)
            h[:, [1, 3, 6]] = 0
            assert torch.equal(x.cpu().nan_to_num(123.0), h.nan_to_num(123.0))


def test_codes_at_ties_and_of_every_size(env):
    """Values on the borders between codes: to even; a row that runs over all of them."""
    torch, paged, _ = env
    for code, top in (("int8", 127.0), ("e4m3", 448.0)):
        x = torch.linspace(-top, top, 32 * 64).view(32, 64).clone()
        x = (x * 2).round() / 2 if code == "int8" else (x * 16).round() / 16
        x[0, 0] = top
        if code == "e4m3":
            x[1] = torch.arange(64) * 2.0 ** -10  # halves of the smallest step
            x[2, :32] = 16 + torch.arange(32) * 0.5
        k = x.view(1, 1, 1, 32, 64)
        pages = paged.Pages.empty(1, 1, 1, 64, 32, code)
        paged.pages_store(pages, torch.zeros(1, dtype=torch.int32, device="cuda"), k.cuda(), k.cuda())
        data, scale = host_pages(k, k, code)
        assert np.array_equal(M.from_bytes(pages.data.cpu().numpy(), code), M.from_bytes(data, code))
        assert (pages.scale == 1).all() and (scale == 1).all()


def test_store_takes_a_caches_rows_as_they_lie(env):
    torch, paged, _ = env
    l, g, d, rows, n = 2, 3, 64, 32, 5
    cache = torch.randn((2, l, g, 200, d), device="cuda").bfloat16()
    k, v = (x[:, :, 7:7 + n * rows].unflatten(2, (n, rows)).transpose(1, 2) for x in cache)
    pages, plain = paged.Pages.empty(l, 9, g, d, rows), paged.Pages.empty(l, 9, g, d, rows)
    ids = torch.tensor([3, 8, 0, 1, 5], dtype=torch.int32, device="cuda")
    paged.pages_store(pages, ids, k, v)
    paged.pages_store(plain, ids, k.contiguous(), v.contiguous())
    assert torch.equal(pages.data, plain.data) and torch.equal(pages.scale, plain.scale)
    # one layer, one page; ids outside the pool; none
    before = pages.data.clone()
    paged.pages_store(pages, torch.tensor([-1], dtype=torch.int32, device="cuda"), k[:1, :1], v[:1, :1], layer=1)
    paged.pages_store(pages, torch.tensor([9], dtype=torch.int32, device="cuda"), k[:1, :1], v[:1, :1], layer=1)
    paged.pages_store(pages, ids[:0], k[:, :0], v[:, :0])
    assert torch.equal(pages.data, before)
    paged.pages_store(pages, ids[2:3], k[:1, 1:2], v[:1, 1:2], layer=1)
    assert torch.equal(pages.data[1, 0], before.new_tensor(0) + _stored(paged, k[:1, 1:2], v[:1, 1:2])[0, 0])
    assert torch.equal(pages.data[0], before[0])
    k0, _ = paged.pages_load(pages, ids[:0])
    assert k0.shape == (l, 0, g, rows, d)


def _stored(paged, k, v):
    import torch
    pages = paged.Pages.empty(k.shape[0], k.shape[1], k.shape[2], k.shape[4], k.shape[3])
    paged.pages_store(pages, torch.arange(k.shape[1], dtype=torch.int32, device="cuda"), k, v)
    return pages.data


# ---------------------------------------------------------------- the sequences

class Batch:
    """The same batch on the device and as paged_model has it."""

    def __init__(self, env, b, cols, n_page, t, dtype="bf16", code="int8", layers=2, g=2, d=64, rows=32, ring=None, seed=0):
        self.torch, self.paged = env[0], env[1]
        torch = self.torch
        self.t, self.b, self.rows = t, b, rows
        self.gen = torch.Generator().manual_seed(seed)
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.pages = self.paged.Pages.empty(layers, n_page, g, d, rows, code)
        self.host = M.Sequences(np.full((b, cols), -1), np.full(b, -1), np.zeros(n_page), rows)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        self.table, self.length, self.refs = i32(self.host.table), i32(self.host.length), i32(self.host.refs)
        self.ring = rows + t - 1 if ring is None else ring
        self.kt, self.vt = (torch.zeros((layers, b, g, self.ring, d), dtype=self.dt, device="cuda") for _ in "kv")
        self.i32 = i32
        # every sequence's rows, as they are and as they are read back: {slot: [(k, v)]} of [L][G][D]
        self.truth = {i: [] for i in range(b)}

    def seqs(self):
        return self.refs, self.table, self.length

    def same(self):
        assert np.array_equal(self.table.cpu().numpy(), self.host.table)
        assert np.array_equal(self.length.cpu().numpy(), self.host.length)
        assert np.array_equal(self.refs.cpu().numpy(), self.host.refs)
        held = np.bincount(self.host.table[self.host.table >= 0], minlength=len(self.host.refs))
        assert np.array_equal(held, self.host.refs)

    def step(self, path, path_len, window=0, sinks=0):
        torch = self.torch
        l, b, g, _, d = self.kt.shape
        kn, vn = (torch.randn((l, b, self.t, g, d), generator=self.gen).to(self.dt) for _ in "kv")
        before = [x.clone() for x in (self.kt, self.vt)]
        full = self.paged.pages_commit(self.pages, *self.seqs(), self.kt, self.vt, kn.cuda(), vn.cuda(), self.i32(path),
                                       self.i32(path_len), window=window, sinks=sinks)
        want, moves = self.host.commit(path, path_len, self.t, window, sinks)
        assert full.tolist() == want
        self.same()
        for s, pos, row in moves:
            assert len(self.truth[s]) == pos
            self.truth[s].append((kn[:, s, row], vn[:, s, row]))
        # rows behind the full pages are in the tail, all others of it are left as they were
        for w, (x, old) in enumerate(zip((self.kt, self.vt), before)):
            for s, pos, row in moves:
                if pos >= self.host.length[s] // self.rows * self.rows:
                    old[:, s, :, pos % self.ring] = (kn, vn)[w][:, s, row].cuda()
            assert torch.equal(x, old)
        self.pages_hold()
        return full

    def pages_hold(self):
        """Pages that got full are the codes of the sequences' rows."""
        for s, col, page in self.host.filled:
            rows = self.truth[s][col * self.rows:(col + 1) * self.rows]
            k, v = (self.torch.stack([r[w] for r in rows], 2)[:, None] for w in (0, 1))
            data, scale = host_pages(k, v, self.pages.code)
            got = self.pages.data[:, page].cpu().numpy()
            assert np.array_equal(M.from_bytes(got, self.pages.code), M.from_bytes(data[:, 0], self.pages.code))
            assert np.array_equal(self.pages.scale[:, page].cpu().numpy(), scale[:, 0])

    def open_rows(self):
        for s in range(self.b):
            n = int(self.host.length[s])
            for pos in range(max(n, 0) // self.rows * self.rows, max(n, 0)):
                for w, x in enumerate((self.kt, self.vt)):
                    assert self.torch.equal(x[:, s, :, pos % self.ring].cpu(), self.truth[s][pos][w])


@pytest.mark.parametrize("dtype,code,rows,d,t", [("f32", "int8", 32, 32, 15), ("bf16", "int8", 32, 64, 64),
                                                 ("bf16", "e4m3", 64, 128, 9), ("f32", "e4m3", 128, 64, 64),
                                                 ("bf16", "int8", 128, 64, 1)])
def test_commits(env, dtype, code, rows, d, t):
    """Paths of all lengths, until pages run out; entries that are no row; slots without a sequence."""
    b = 5
    batch = Batch(env, b, 4, 9, t, dtype, code, d=d, rows=rows)
    batch.length[:4] = 0
    batch.host.length[:4] = 0
    rng = np.random.default_rng(t)
    for step in range(10 if t > 1 else 140):
        path, n = [], []
        for s in range(b):
            kept = sorted(rng.choice(t, rng.integers(0, t + 1), replace=False).tolist()) if t > 1 else [0]
            path.append((kept + [int(rng.choice([-1, t, 1 << 30])), 0] + [0] * t)[:t + 1])
            n.append(int(rng.choice([len(kept), len(kept) + 1])) if step % 3 else t + 1)
        batch.step([p[:min(t + 1, 64)] for p in path], n)
        if step % 20 == 0:
            batch.open_rows()
    batch.open_rows()
    assert (batch.host.length[:4] > 0).all() and batch.host.length[4] == -1


def test_a_sequence_that_gets_no_page_is_left_as_it_is(env):
    batch = Batch(env, 3, 2, 2, 8)
    for x in (batch.length, batch.host.length):
        x[:] = 0
    path = [list(range(8))] * 3
    for _ in range(3):
        assert batch.step(path, [8, 8, 8]).tolist() == [0, 0, 0]
    assert batch.step(path, [8, 7, 8]).tolist() == [1, 0, 1]
    assert batch.step(path, [8, 8, 8]).tolist() == [0, -1, 0]  # the pool is empty
    for _ in range(2):
        batch.step(path, [8, 0, 0])
    assert batch.step(path, [7, 0, 8]).tolist() == [0, 0, 0]
    assert batch.step(path, [1, 1, 0]).tolist() == [-1, -1, 0]
    assert batch.length.tolist() == [3 * 8 + 8 + 8 + 2 * 8 + 7, 3 * 8 + 7, 3 * 8 + 8 + 8 + 8]
    # a path of no columns, lengths below 0
    assert batch.step([[], [], []], [4, 4, 4]).tolist() == [0, 0, 0]
    assert batch.step(path, [-1, -5, -(1 << 31)]).tolist() == [0, 0, 0]


@pytest.mark.parametrize("window,sinks,rows", [(8, 0, 32), (40, 1, 32), (64, 33, 32), (100, 0, 64), (1, 0, 32)])
def test_pages_behind_the_window_are_given_back(env, window, sinks, rows):
    t = min(8, window)
    batch = Batch(env, 2, 12, 12, t, rows=rows)
    for x in (batch.length, batch.host.length):
        x[:] = 0
    for _ in range(160 if t == 1 else 40):
        full = batch.step([list(range(t))] * 2, [t, t - 1 or 1], window, sinks)
        assert (full >= 0).all()
    assert (batch.host.refs > 0).sum() <= 2 * ((window + t) // rows + 2 + -(-sinks // rows))


def test_takes(env):
    torch, paged, _ = env
    batch = Batch(env, 6, 5, 12, 4)
    take = lambda *n: paged.pages_take(batch.pages, *batch.seqs(), batch.i32(list(n))).tolist()  # noqa: E731
    for count in ([2, -1, 0, 3, -5, 1], [1, 2, 0, 1, 0, -1], [-1, -1, 9, 2, 1, 1], [2, 0, 0, 1, 0, 0],
                  [1 << 30, -1, -1, 2**31 - 1, -1, 0], [-1, 0, 5, 0, 1, 0], [0, 0, 0, 0, 2, 1]):
        assert take(*count) == batch.host.take(count), count
        batch.same()
    batch.length[1] += 3  # an open page
    batch.host.length[1] += 3
    assert take(-1, 0, -1, -1, -1, -1) == batch.host.take([-1, 0, -1, -1, -1, -1]) == [-1] * 6


def test_takes_of_large_pools_and_batches(env):
    """More pages than one look, more slots than threads."""
    torch, paged, _ = env
    rng = np.random.default_rng(0)
    n_page, b = 70_001, 4096
    pages = paged.Pages.empty(1, n_page, 1, 32, 32)
    refs = (rng.random(n_page) < 0.7).astype(np.int64)
    host = M.Sequences(np.full((b, 9), -1), np.full(b, -1), refs, 32)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    table, length, dref = i32(host.table), i32(host.length), i32(refs)
    for most in (3, 9, 10):
        count = rng.integers(-1, most, b).tolist()
        got = paged.pages_take(pages, dref, table, length, i32(count))
        assert got.tolist() == host.take(count)
        for x, y in ((table, host.table), (length, host.length), (dref, host.refs)):
            assert np.array_equal(x.cpu().numpy(), y)
    u, moves = host.compact()
    before = pages.scale[:, list(moves)].clone()
    assert paged.pages_compact(pages, dref, table).item() == u
    assert np.array_equal(dref.cpu().numpy(), host.refs) and np.array_equal(table.cpu().numpy(), host.table)
    assert torch.equal(pages.scale[:, list(moves.values())], before)


def grown(env, b=8, t=8, n_page=40, steps=14, **kw):
    batch = Batch(env, b, 8, n_page, t, **kw)
    for x in (batch.length, batch.host.length):
        x[:b - 2] = 0
    rng = np.random.default_rng(b)
    for _ in range(steps):
        batch.step([list(range(t))] * b, rng.integers(1, t + 1, b).tolist())
    return batch


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forks(env, dtype):
    torch, paged, _ = env
    batch = grown(env, dtype=dtype)
    for parents in ([0, 0, 2, 3, 4, 2, 2, 7], [0, 1, 0, -1, 4, 99, 6, 1], [1, 0, 2, 2, 3, 5, -(1 << 31), 2],
                    [0, 1, 2, 3, 4, 5, 6, 7], [8, 1, 1, 1, 1, 1, 1, 1]):
        tails = [x.clone() for x in (batch.kt, batch.vt)]
        paged.pages_fork(*batch.seqs(), batch.i32(parents), batch.kt, batch.vt, batch.rows)
        copied = dict(batch.host.fork(parents))
        batch.same()
        for s in range(batch.b):
            if s in copied:
                batch.truth[s] = list(batch.truth[copied[s]])
            elif parents[s] != s:
                batch.truth[s] = []
        batch.open_rows()
        for x, old in zip((batch.kt, batch.vt), tails):  # rows that are not the sequence's are left alone
            for s, p in copied.items():
                n = int(batch.host.length[s])
                for pos in range(max(n, 0) // 32 * 32, max(n, 0)):
                    old[:, s, :, pos % batch.ring] = old[:, p, :, pos % batch.ring]
            assert torch.equal(x, old)
        batch.step([list(range(8))] * 8, [5] * 8)
        batch.open_rows()


def test_compactions(env):
    torch, paged, _ = env
    batch = grown(env, n_page=60)
    for parents in ([0, 0, -1, 3, -1, 5, 5, 5], [-1, 1, 2, -1, 4, -1, 6, 7], [-1] * 8, list(range(8))):
        paged.pages_fork(*batch.seqs(), batch.i32(parents), batch.kt, batch.vt, 32)
        batch.host.fork(parents)
        data, scale = batch.pages.data.clone(), batch.pages.scale.clone()
        used = paged.pages_compact(batch.pages, batch.refs, batch.table)
        u, moves = batch.host.compact()
        assert used.item() == u and used.dtype == torch.int32
        batch.same()
        for a, b in moves.items():
            data[:, b], scale[:, b] = data[:, a], scale[:, a]
        assert torch.equal(batch.pages.data, data) and torch.equal(batch.pages.scale, scale)


def test_entries_outside_the_pool_are_left_alone(env):
    torch, paged, _ = env
    batch = grown(env)
    batch.table[5, 6], batch.table[5, 7], batch.table[4, 7] = 40, 2**31 - 1, -(1 << 31)
    refs = batch.refs.clone()
    paged.pages_compact(batch.pages, batch.refs, batch.table)
    assert batch.table[5, 6:].tolist() == [40, 2**31 - 1] and batch.table[4, 7] == -(1 << 31)
    assert torch.equal(batch.refs.sort().values, refs.sort().values)
    paged.pages_fork(*batch.seqs(), batch.i32([0, 5, 2, 3, 4, 5, 6, -1]), batch.kt, batch.vt, 32)
    assert batch.table[1, 6:].tolist() == [40, 2**31 - 1] and (batch.refs >= 0).all()


def test_a_run_of_all_of_them(env):
    """Prompts are admitted, share their pages, grow by accepted paths, end; the pool is compacted: attention reads every
    sequence's rows, in codes where its pages are full and as they are behind them."""
    torch, paged, _ = env
    b, t, rows, d, g, l = 6, 6, 32, 64, 2, 2
    batch = Batch(env, b, 10, 40, t, rows=rows, d=d, g=g, layers=l)
    rng = np.random.default_rng(3)
    prompt = {}
    for slot, n in ((0, 3 * rows + 11), (3, rows - 1)):
        k, v = (torch.randn((l, g, n, d), generator=batch.gen).bfloat16() for _ in "kv")
        full = n // rows
        count = [-1] * b
        count[slot] = full
        assert paged.pages_take(batch.pages, *batch.seqs(), batch.i32(count)).tolist() == batch.host.take(count)
        cut = [x[:, :, :full * rows].unflatten(2, (full, rows)).transpose(1, 2).cuda() for x in (k, v)]
        paged.pages_store(batch.pages, batch.table[slot, :full], *cut)
        batch.truth[slot] = [(k[:, :, p], v[:, :, p]) for p in range(full * rows)]
        prompt[slot] = k, v
        for p in range(full * rows, n):  # the open page's rows, one commit each
            step = [x[:, None, None, :, p].expand(l, b, t, g, d).contiguous().cuda() for x in (k, v)]
            n_new = [int(s == slot) for s in range(b)]
            paged.pages_commit(batch.pages, *batch.seqs(), batch.kt, batch.vt, *step, batch.i32([[0]] * b), batch.i32(n_new))
            batch.host.commit([[0]] * b, n_new, t)
            batch.truth[slot].append((k[:, :, p], v[:, :, p]))
    batch.same()

    def check():
        q, kn, vn = (torch.randn((b, t, g * (2 if i == 0 else 1), d), generator=batch.gen).bfloat16() for i in range(3))
        data, scale = batch.pages.data.cpu().numpy(), batch.pages.scale.cpu().numpy()
        for layer in range(l):
            out = paged.paged_attention(q.cuda(), batch.pages, batch.table, batch.length, batch.kt[layer], batch.vt[layer],
                                        kn.cuda(), vn.cuda(), layer=layer)
            f = lambda x: x.double().cpu().numpy()  # noqa: E731
            tails = [f(x[layer]) for x in (batch.kt, batch.vt)]
            for s in range(b):  # (open rows as the test knows them)
                for pos in range(max(int(batch.host.length[s]), 0) // rows * rows, max(int(batch.host.length[s]), 0)):
                    for w in (0, 1):
                        tails[w][s, :, pos % batch.ring] = f(batch.truth[s][pos][w][layer])
            hk, hv = M.page_values(data[layer], scale[layer], rows, d, "int8")
            for s in range(b):  # pages hold the sequence's rows, to half a code
                for c in range(max(int(batch.host.length[s]), 0) // rows):
                    for w, h in ((0, hk), (1, hv)):
                        mine = np.stack([f(batch.truth[s][c * rows + r][w][layer]) for r in range(rows)], 1)
                        a = np.abs(mine).max((1, 2), keepdims=True)
                        assert (np.abs(h[batch.host.table[s, c]] - mine) <= a / 127 * (0.5 + 2.0 ** -16)).all()
            ref, _, big, vmax = M.attention(f(q), batch.host.table, batch.host.length, (hk, hv), tails, (f(kn), f(vn)), rows)
            assert np.abs(f(out) - ref).max() <= tolerance("bf16", d, big, vmax, 400)

    check()
    for parents in ([0, 0, 0, 3, 3, -1], [0, 1, 2, -1, 0, 1], [0, 0, 2, 2, 4, 4]):
        paged.pages_fork(*batch.seqs(), batch.i32(parents), batch.kt, batch.vt, rows)
        for s, p in batch.host.fork(parents):
            batch.truth[s] = list(batch.truth[p])
        batch.same()
        for _ in range(7):
            path = [sorted(rng.choice(t, 4, replace=False).tolist()) for _ in range(b)]
            batch.step(path, rng.integers(1, 5, b).tolist())
        check()
        before = batch.pages.data.clone()
        u, moves = batch.host.compact()
        assert paged.pages_compact(batch.pages, batch.refs, batch.table).item() == u
        assert all(torch.equal(batch.pages.data[:, to], before[:, at]) for at, to in moves.items())
        batch.same()
        check()


def test_the_sequences_operators_in_a_graph(env):
    """Captured once: fork, commit (with the window's release) and compaction, replayed on other states."""
    torch, paged, _ = env
    a, e = grown(env), grown(env)  # (alike)
    path, n = a.i32([[0, 2, 5]] * 8), a.i32([3] * 8)
    parents = a.i32(list(range(8)))
    gen = torch.Generator().manual_seed(9)
    kn, vn = (torch.randn((2, 8, 8, 2, 64), generator=gen).bfloat16().cuda() for _ in "kv")

    def step(x):
        paged.pages_fork(*x.seqs(), parents, x.kt, x.vt, 32)
        full = paged.pages_commit(x.pages, *x.seqs(), x.kt, x.vt, kn, vn, path, n, window=70, sinks=4)
        return full, paged.pages_compact(x.pages, x.refs, x.table)

    warm = grown(env)
    step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(a)
    for i, p in enumerate(([0, 0, 2, 3, 4, 4, -1, 7], list(range(8)), [0, 1, 0, 1, 0, 1, 0, 1], list(range(8)), [-1] * 4 + [4] * 4)):
        parents.copy_(torch.tensor(p, dtype=torch.int32))
        kn.add_(0.01)
        n.fill_(1 + i % 3)
        graph.replay()
        want = step(e)
        torch.cuda.synchronize()
        for x, y in zip(out + (a.table, a.length, a.refs, a.kt, a.vt, a.pages.data, a.pages.scale),
                        want + (e.table, e.length, e.refs, e.kt, e.vt, e.pages.data, e.pages.scale)):
            assert torch.equal(x, y), i


def test_the_operators_run_on_the_stream_they_are_given(env):
    torch, paged, _ = env
    a, e = grown(env), grown(env)
    side = torch.cuda.Stream()
    kn, vn = (torch.randn((2, 8, 8, 2, 64), device="cuda").bfloat16() for _ in "kv")
    for x, kw in ((a, {}), (e, {"stream": side})):
        torch.cuda.synchronize()
        got = paged.pages_take(x.pages, *x.seqs(), x.i32([-1] * 7 + [2]), **kw)
        side.synchronize()
        ids = x.table[7, :2].contiguous()
        torch.cuda.synchronize()
        k, v = paged.pages_load(x.pages, x.i32([0, 1]), torch.bfloat16, **kw)
        paged.pages_store(x.pages, ids, k, v, **kw)
        paged.pages_fork(*x.seqs(), x.i32([0, 7, 2, 3, 4, 5, 6, 7]), x.kt, x.vt, 32, **kw)
        x.full = paged.pages_commit(x.pages, *x.seqs(), x.kt, x.vt, kn, vn, x.i32([[1, 2]] * 8), x.i32([2] * 8), **kw)
        x.used = paged.pages_compact(x.pages, x.refs, x.table, **kw)
        torch.cuda.synchronize()
        assert got.tolist() == [-1] * 7 + [2]
    for n in ("table", "length", "refs", "kt", "vt", "full", "used"):
        assert torch.equal(getattr(a, n), getattr(e, n)), n
    assert torch.equal(a.pages.data, e.pages.data)


# ---------------------------------------------------------------- attention, cut by the sequences' lengths

@pytest.mark.parametrize("dtype,code,b,t,h,g,d,rows,lens,kw", [
    ("bf16", "int8", 3, 1, 2, 1, 64, 32, [3000, 40, 1500], {}),
    ("bf16", "e4m3", 4, 5, 8, 2, 128, 64, [0, 2500, -1, 777], {"tree": True}),
    ("f32", "int8", 2, 9, 4, 2, 64, 128, [2222, 1031], {}),
    ("bf16", "int8", 2, 40, 6, 2, 32, 32, [1800, 64], {}),
    ("f32", "e4m3", 130, 1, 1, 1, 32, 32, [(37 * i) % 90 if i % 41 else 2600 for i in range(130)], {}),
    ("bf16", "int8", 70, 2, 2, 2, 64, 32, [-1 if i % 7 == 0 else (53 * i) % 200 if i != 66 else 1900 for i in range(70)], {})])
def test_batches_of_long_and_short_sequences(env, dtype, code, b, t, h, g, d, rows, lens, kw):
    """Tables wide enough that sequences are cut by their lengths (more than 512 times 32 rows)."""
    print(dtype, code, b, t, lens[:4], flush=True)
    c = Case(env, dtype, code, b, t, h, g, d, rows, lens, cols=600 * 32 // rows + 1, **kw)
    want = c.check()
    again = c.run()
    assert all(env[0].equal(x, y) for x, y in zip(want, again))


def test_windows_where_sequences_are_cut_by_their_lengths(env):
    c = Case(env, "bf16", "int8", 3, 2, 2, 1, 64, 32, [2900, 900, 100], cols=1300)
    c.check(window=17000, sinks=5)  # (wide enough to be cut so)
    c.check(window=2000, sinks=16500)
    c.check(window=1000, sinks=70)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_any_size(env, dtype):
    """Scores around 2^26, 2^45 and 2^90: the row with the largest by far is all that is left of a query's."""
    for by in (2.0 ** 22, 2.0 ** 41, 2.0 ** 86):
        c = Case(env, dtype, "int8", 1, 1, 2, 1, 64, 32, [140])
        c.q = c.q.abs() + 1
        pk, _ = M.places(32, 64)
        for row in (3, 77, 127):
            x = Case(env, dtype, "int8", 1, 1, 2, 1, 64, 32, [140])
            x.q = (c.q * by).to(x.dt)
            x.kt.fill_(0.1), x.kn.fill_(0.2)
            raw = x.data.clone().view(1, -1, 1, 2, 32 * 64)
            raw[:, :, :, 0] = 128 + 16   # all keys alike ...
            raw[0, x.table[0, row // 32], 0, 0, pk[row % 32]] = 128 + 120  # ... but one
            x.data = raw.view(x.data.shape)
            x.scale[0, :, :, 0] = 0.03
            out, lse = x.run()
            v = x.host()[1][x.table[0, row // 32], 0, row % 32]
            got = out[0, 0].double().cpu().numpy()
            assert np.abs(got - v[None]).max() <= np.abs(v).max() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -21)
            assert lse.isfinite().all()


def test_scales_below_zero(env):
    """(Stored pages have none.)"""
    for dtype in ("f32", "bf16"):
        c = Case(env, dtype, "e4m3", 2, 2, 4, 2, 64, 32, [200, 321])
        c.scale[0, ::3, :, 0] *= -1
        c.scale[0, ::4, :, 1] *= -1
        c.check()
        c.check(scale=-0.2)
