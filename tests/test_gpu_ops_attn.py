"""ops.prefix_attention against the definition in 64 bits on the host.

Tolerances, set from the arithmetic: a score is a float32 sum of D products,
so it is off by at most (D + 4) eps S with S the largest sum of |q_i k_i|
scale; a softmax weight by twice that, relatively, and the weighted sum of the
values (whose absolute maximum is vmax) by that times vmax, plus the few
roundings of the sums and rescalings (64 eps).  bfloat16: the weights for the
value product and the output are rounded to 8 bits each, 2^-9 vmax apiece."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2308_04623_amd import ops
    assert torch.cuda.is_available()
    return torch, ops


def make(torch, dtype, b, t, h, g, d, p, r, seed=0, lens=None):
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rn = lambda *s: torch.randn(s, generator=gen).to(dt)  # noqa: E731
    x = {"q": rn(b, t, h, d) * 2, "kp": rn(g, p, d), "vp": rn(g, p, d), "ko": rn(b, g, r, d), "vo": rn(b, g, r, d)}
    if lens is None:
        lens = torch.randint(0, r + 1, (b,), generator=gen).tolist()
    return x, lens


def reference(x, lens, scale=None):
    """(out, lse, S, vmax) in 64 bits."""
    q, kp, vp, ko, vo = (x[k].double().numpy() for k in ("q", "kp", "vp", "ko", "vo"))
    b, t, h, d = q.shape
    g, p, r = kp.shape[0], kp.shape[1], ko.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse, big = np.zeros(q.shape), np.full((b, t, h), -np.inf), 0.0
    vmax = 0.0
    for i in range(b):
        n = min(lens[i], r)
        if lens[i] < 0:
            continue
        for j in range(t):
            own = max(0, n - t + 1 + j)
            for hh in range(h):
                kv = hh // (h // g)
                k = np.concatenate([kp[kv], ko[i, kv, :own]])
                v = np.concatenate([vp[kv], vo[i, kv, :own]])
                if not len(k):
                    continue
                s = k @ q[i, j, hh] * scale
                m = s.max()
                e = np.exp(s - m)
                out[i, j, hh] = e @ v / e.sum()
                lse[i, j, hh] = m + math.log(e.sum())
                big = max(big, (np.abs(k) @ np.abs(q[i, j, hh])).max() * abs(scale))
                vmax = max(vmax, np.abs(v).max())
    return out, lse, big, vmax


def tolerance(dtype, d, big, vmax):
    tol = vmax * (2 * EPS * (d + 4) * big + 64 * EPS)
    return tol + (2.0 ** -8 * vmax if dtype == "bf16" else 0.0)


def check(torch, ops, dtype, x, lens, scale=None, put=None, **kw):
    put = put or (lambda name, t: t.cuda())
    dev = {k: put(k, v) for k, v in x.items()}
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ops.prefix_attention(dev["q"], dev["kp"], dev["vp"], dev["ko"], dev["vo"], n, scale=scale,
                                    return_lse=True, **kw)
    torch.cuda.synchronize()
    ref, rl, big, vmax = reference(x, lens, scale)
    d = x["q"].shape[3]
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert np.abs(got - ref).max() <= tolerance(dtype, d, big, vmax)
    got_l = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got_l), np.isneginf(rl))
    live = np.isfinite(rl)
    if live.any():
        assert np.abs(got_l[live] - rl[live]).max() <= (d + 4) * EPS * big + 64 * EPS * (1 + np.abs(rl[live]).max())
    return out


SHAPES = [
    # b, t, h, g, d, p, r
    (1, 1, 1, 1, 32, 1, 1), (1, 1, 4, 4, 32, 64, 24), (6, 1, 4, 4, 32, 65, 7), (3, 2, 6, 2, 64, 31, 33),
    (5, 1, 20, 20, 64, 130, 40), (2, 5, 8, 2, 128, 257, 100), (17, 3, 4, 1, 64, 500, 9), (33, 1, 2, 2, 128, 129, 65),
    (2, 64, 2, 1, 64, 96, 70), (70, 8, 4, 2, 32, 200, 12), (1, 1, 25, 25, 64, 3000, 5), (4, 17, 3, 3, 64, 1, 300),
    (260, 1, 2, 1, 64, 513, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(env, dtype, shape):
    torch, ops = env
    print(dtype, shape, flush=True)
    x, lens = make(torch, dtype, *shape)
    check(torch, ops, dtype, x, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [1, 15, 16, 17, 32, 33, 63, 64, 127, 128, 129, 255, 1023])
def test_prefix_lengths(env, dtype, p):
    torch, ops = env
    x, lens = make(torch, dtype, 3, 2, 4, 2, 64, p, 20, seed=p)
    check(torch, ops, dtype, x, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_prefix_no_own_rows_and_empty_slots(env, dtype):
    torch, ops = env
    # no prefix: sequences of length 0 see nothing, length 1 one row; a slot that is off
    x, lens = make(torch, dtype, 6, 1, 4, 2, 64, 0, 40, lens=[0, 1, -1, 40, 41, 17])
    out = check(torch, ops, dtype, x, lens)
    assert not out[0].any() and not out[2].any()
    # queries before a sequence's first row
    x, lens = make(torch, dtype, 4, 5, 4, 2, 64, 0, 40, lens=[0, 2, 5, -3])
    out = check(torch, ops, dtype, x, lens)
    assert not out[1, :3].any() and out[1, 3:].any() and not out[3].any()
    # no own rows at all
    x, lens = make(torch, dtype, 4, 2, 4, 2, 64, 77, 0, lens=[0, 0, -1, 3])
    check(torch, ops, dtype, x, lens)
    # nothing to look at
    x, lens = make(torch, dtype, 2, 2, 4, 2, 64, 0, 0, lens=[0, -1])
    assert not check(torch, ops, dtype, x, lens).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_not_seen_may_hold_anything(env, dtype):
    torch, ops = env
    x, lens = make(torch, dtype, 5, 3, 4, 2, 64, 70, 48, lens=[0, 1, 20, 47, -1])
    want = check(torch, ops, dtype, x, lens)
    for i, n in enumerate(lens):
        for name in ("ko", "vo"):
            x[name][i, :, max(0, n):] = float("nan") if name == "vo" else float("inf")

    def put(name, t):  # and beyond the prefix, within the same buffer
        if name in ("kp", "vp"):
            room = torch.full((t.shape[0], t.shape[1] + 64, t.shape[2]), float("nan"), dtype=t.dtype, device="cuda")
            room[:, :t.shape[1]] = t.cuda()
            return room[:, :t.shape[1]]
        return t.cuda()

    dev = {k: put(k, v) for k, v in x.items()}
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = ops.prefix_attention(dev["q"], dev["kp"], dev["vp"], dev["ko"], dev["vo"], n)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_of_infinite_size_stay_with_their_rows(env, dtype):
    """A NaN value that is seen reaches its own sequence alone, a shared one every one."""
    torch, ops = env
    x, lens = make(torch, dtype, 4, 1, 2, 2, 64, 40, 30, lens=[10, 30, 1, -1])
    x["vo"][1, 0, 5, 3] = float("nan")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    run = lambda: ops.prefix_attention(*(x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")), n)  # noqa: E731
    bad = torch.isnan(run())
    assert bad[1, 0, 0, 3] and bad.sum() == 1
    x["vp"][1, 7, 9] = float("nan")
    bad = torch.isnan(run())
    assert bad[:3, 0, 1, 9].all() and bad.sum() == 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_apart_and_equal(env, dtype):
    torch, ops = env
    x, lens = make(torch, dtype, 3, 1, 2, 2, 64, 200, 50, lens=[50, 3, 0])
    x["q"] = x["q"] * 20  # one key takes nearly everything
    check(torch, ops, dtype, x, lens)
    x["q"] = x["q"] * 0  # all alike
    check(torch, ops, dtype, x, lens)
    x, lens = make(torch, dtype, 3, 1, 2, 2, 64, 200, 50, lens=[50, 3, 0])
    check(torch, ops, dtype, x, lens, scale=-0.3)
    check(torch, ops, dtype, x, lens, scale=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(env, dtype):
    """Keys and values with the tokens outside the heads, queries inside a wider
    projection, an output inside a wider buffer."""
    torch, ops = env
    x, lens = make(torch, dtype, 5, 3, 4, 2, 64, 90, 21)

    def put(name, t):
        if name in ("kp", "vp"):
            return t.cuda().transpose(0, 1).contiguous().transpose(0, 1)
        if name in ("ko", "vo"):
            return t.cuda().transpose(1, 2).contiguous().transpose(1, 2)
        wide = torch.full((5, 3, 3 * 4 * 64), 7.0, dtype=t.dtype, device="cuda")
        q = wide[:, :, :256].unflatten(2, (4, 64))
        q.copy_(t)
        return q

    room = torch.full((5, 3, 6, 64), 3.0, dtype=x["q"].dtype, device="cuda")
    check(torch, ops, dtype, x, lens, put=put, out=room[:, :, 1:5])
    assert (room[:, :, 0] == 3).all() and (room[:, :, 5] == 3).all()
    plain = check(torch, ops, dtype, x, lens)
    assert torch.equal(plain, room[:, :, 1:5])


def test_broadcast_queries(env):
    torch, ops = env
    x, lens = make(torch, "bf16", 4, 1, 4, 4, 64, 50, 16)
    x["q"] = x["q"][:1].expand(4, 1, 4, 64)
    check(torch, ops, "bf16", x, lens, put=lambda k, t: t[:1].cuda().expand(4, 1, 4, 64) if k == "q" else t.cuda())


def test_offsets_past_32_bits(env):
    """Rows 2^26 elements apart: the last ones lie 5 GB into the buffer."""
    torch, ops = env
    p, d, step = 45, 64, 1 << 26
    x, lens = make(torch, "bf16", 3, 1, 2, 1, d, p, 4)
    big = torch.empty(p * step, dtype=torch.bfloat16, device="cuda")
    kp = big.as_strided((1, p, d), (0, step, 1))
    vp = big[4096:].as_strided((1, p, d), (0, step, 1))

    def put(name, t):
        if name == "kp":
            return kp.copy_(t)
        return vp.copy_(t) if name == "vp" else t.cuda()

    check(torch, ops, "bf16", x, lens, put=put)


def test_a_sequence_does_not_depend_on_the_batch_around_it(env):
    """Bitwise, from run to run and on another stream."""
    torch, ops = env
    x, lens = make(torch, "bf16", 9, 2, 4, 2, 64, 777, 64)
    args = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
    a = ops.prefix_attention(*args)
    for _ in range(3):
        assert torch.equal(a, ops.prefix_attention(*args))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = ops.prefix_attention(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b)


def test_captured_in_a_graph(env):
    torch, ops = env
    x, lens = make(torch, "bf16", 9, 1, 4, 2, 64, 777, 64)
    args = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
    out = torch.empty_like(args[0])
    ops.prefix_attention(*args, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.prefix_attention(*args, out=out)
    for i in range(3):
        args[0].add_(0.25)
        args[5].fill_(10 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.prefix_attention(*args))


def test_refusals_of_the_binding(env):
    torch, ops = env
    from paper_2308_04623_amd.ssd import SSDError
    x, lens = make(torch, "bf16", 2, 1, 4, 2, 64, 8, 4)
    a = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]

    def refused(i, t):
        b = list(a)
        b[i] = t
        with pytest.raises(SSDError):
            ops.prefix_attention(*b)

    refused(0, a[0].float())
    refused(0, a[0][0])
    refused(1, a[1][:, :, :32])
    refused(2, a[2][:, :4])
    refused(3, a[3][:1])
    refused(4, a[4].transpose(1, 2).contiguous().transpose(1, 2))
    refused(5, a[5].long())
    refused(5, a[5].cpu())
    refused(0, torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16, device="cuda")[..., ::2])
    with pytest.raises(SSDError):
        ops.prefix_attention(*a, out=torch.empty(2, 1, 4, 32, dtype=torch.bfloat16, device="cuda"))


# a prefix that one workgroup takes with the sequence's own rows, and one that is cut
# into parts: 128 bfloat16 (64 float32) rows are a step, two steps the limit with few queries
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps,more", [(2, 0), (2, 1), (5, 13), (18, 1)])
@pytest.mark.parametrize("b,t,h,g,d", [(3, 1, 4, 4, 64), (6, 2, 6, 2, 32), (40, 3, 2, 1, 128), (9, 16, 4, 2, 64)])
def test_short_and_long_prefixes(env, dtype, steps, more, b, t, h, g, d):
    """Unseen rows hold NaN; sequences are off, empty, shorter than their queries, full."""
    torch, ops = env
    p = steps * (64 if dtype == "f32" else 128) + more
    lens = [(-1, 0, 1, 37, 5)[i % 5] for i in range(b)]
    x, lens = make(torch, dtype, b, t, h, g, d, p, 37, seed=p + b, lens=lens)
    for i, n in enumerate(lens):
        x["ko"][i, :, max(0, n):] = 0.0
        x["vo"][i, :, max(0, n):] = 0.0
    want = check(torch, ops, dtype, x, lens)
    for i, n in enumerate(lens):
        x["ko"][i, :, max(0, n):] = float("inf")
        x["vo"][i, :, max(0, n):] = float("nan")
    args = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    assert torch.equal(ops.prefix_attention(*args, n), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,p", [(2, 0), (2, 300), (40, 64), (1, 1500)])
def test_long_own_rows(env, dtype, b, p):
    torch, ops = env
    x, lens = make(torch, dtype, b, 2, 4, 2, 64, p, 1333, seed=p, lens=[1333 - 700 * (i % 2) for i in range(b)])
    check(torch, ops, dtype, x, lens)


def test_more_queries_than_a_launch_joins(env):
    torch, ops = env
    x, _ = make(torch, "bf16", 2, 64, 136, 8, 32, 2060, 2)  # 4096 x 64 x 136 queries, 2^25 a launch
    ref, _, big, vmax = reference(x, [2, 0])
    q, ko, vo = (x[k].cuda().repeat(2048, 1, 1, 1) for k in ("q", "ko", "vo"))
    n = torch.tensor([2, 0], dtype=torch.int32, device="cuda").repeat(2048)
    out = ops.prefix_attention(q, x["kp"].cuda(), x["vp"].cuda(), ko, vo, n)
    ref = torch.from_numpy(ref).cuda()
    for i in range(0, 4096, 2):
        assert float((out[i:i + 2].double() - ref).abs().max()) <= tolerance("bf16", 32, big, vmax)


def test_out_is_not_the_queries(env):
    torch, ops = env
    from paper_2308_04623_amd.ssd import SSDError
    x, lens = make(torch, "bf16", 2, 1, 4, 2, 64, 8, 4)
    a = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
    with pytest.raises(SSDError):
        ops.prefix_attention(*a, out=a[0])


def test_calls_of_other_layouts_in_turn(env):
    torch, ops = env
    from paper_2308_04623_amd.ssd import SSDError
    cases = [make(torch, dtype, b, t, 4, 2, 64, p, 8, seed=b) for dtype, b, t, p in
             [("bf16", 2, 1, 40), ("f32", 2, 1, 40), ("bf16", 3, 1, 40), ("bf16", 2, 2, 40), ("bf16", 2, 1, 700)]]
    for turn in range(3):
        for i, (x, lens) in enumerate(cases):
            dtype = "f32" if i == 1 else "bf16"
            out = check(torch, ops, dtype, x, lens, scale=None if turn < 2 else 0.3)
            wide = torch.empty(out.shape[:2] + (4, 128), dtype=out.dtype, device="cuda")[..., :64]
            assert torch.equal(check(torch, ops, dtype, x, lens, scale=None if turn < 2 else 0.3, out=wide), out)
        x, lens = cases[0]
        a = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
        for bad in (x["vp"], x["vp"].cuda()[:, :39], x["vp"].cuda().transpose(0, 1).contiguous().transpose(0, 1), None,
                    x["vp"].numpy() if x["vp"].dtype == torch.float32 else 3):
            with pytest.raises(SSDError):
                ops.prefix_attention(a[0], a[1], bad, *a[3:])
        with pytest.raises(SSDError):
            ops.prefix_attention(*a, scale=float("nan"))


def test_more_layouts_than_are_remembered(env):
    torch, ops = env
    q = torch.randn(1, 1, 2, 32, device="cuda")
    k = torch.randn(2, 300, 32, device="cuda")
    own = torch.zeros(1, 2, 1, 32, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    for turn in range(2):
        for p in range(1, 301):
            out = ops.prefix_attention(q, k[:, :p], k[:, :p], own, own, n)
            if p % 60 == 0:
                w = torch.softmax((q[0, 0, :, None].double() * k[:, :p].double()).sum(2) / 32 ** 0.5, 1)
                assert float((out[0, 0] - (w[:, :, None] * k[:, :p].double()).sum(1)).abs().max()) < 1e-5


# how a call is cut: one launch, the waves split the rows, the waves split the queries (one and two tiles each)
FORMS = {"alone": (4, 1, 4, 2, 60), "rows": (4, 1, 4, 2, 3000), "queries": (21, 2, 4, 4, 3000),
         "many": (24, 3, 6, 2, 3000)}


def check_with_nan(torch, ops, dtype, x, lens):
    """As check, where some results are NaN: the same ones, out and lse."""
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ops.prefix_attention(*(x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")), n, return_lse=True)
    clean = {k: torch.nan_to_num(v) for k, v in x.items()}
    ref, rl, _, _ = reference(x, lens)
    _, _, big, vmax = reference(clean, lens)
    d = x["q"].shape[3]
    for got, want, tol in ((out, ref, tolerance(dtype, d, big, vmax)),
                           (lse, rl, (d + 4) * EPS * big + 64 * EPS * (1 + np.abs(rl[np.isfinite(rl)]).max()))):
        got = got.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.isneginf(got), np.isneginf(want))
        live = np.isfinite(want)
        assert np.abs(got[live] - want[live]).max() <= tol
    return ref


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_nan_scores_are_not_lost(env, dtype, d, form):
    """A NaN in a query, in the only row of a sequence's own, in all keys of a stretch
    of the prefix: the queries that see it are NaN, with their lse, and no others."""
    torch, ops = env
    b, t, h, g, p = FORMS[form]
    # (the longest own rows are one chunk: a part of their own where the prefix is cut)
    lens = [(20, 1, -1, 0)[i % 4] for i in range(b)]
    nan = float("nan")
    x, lens = make(torch, dtype, b, t, h, g, d, p, 20, seed=d, lens=lens)
    x["q"][1, 0, 2, 5] = nan
    x["q"][2, t - 1, 0, 0] = nan  # of a slot that is off
    assert np.isnan(check_with_nan(torch, ops, dtype, x, lens)).all(3).sum() == 1
    x, lens = make(torch, dtype, b, t, h, g, d, p, 20, seed=d, lens=lens)
    x["ko"][1, 0, 0, 7] = nan
    assert np.isnan(check_with_nan(torch, ops, dtype, x, lens)).all(3).sum() == h // g  # (the last query alone sees it)
    x, lens = make(torch, dtype, b, t, h, g, d, p, 20, seed=d, lens=lens)
    x["kp"][g - 1, p // 3:2 * p // 3, 1] = nan
    x["kp"][0, 0, 0] = nan if g > 2 else 0.0
    assert np.isnan(check_with_nan(torch, ops, dtype, x, lens)).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_query_of_nan_that_sees_no_row(env, dtype):
    torch, ops = env
    x, lens = make(torch, dtype, 3, 2, 4, 2, 64, 0, 20, lens=[0, 1, 20])
    x["q"][:2] = float("nan")
    check_with_nan(torch, ops, dtype, x, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("power", [10, 22, 24, 27, 31, 34, 60, 115])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(env, dtype, form, power, sign):
    """Scores that are exact, whole multiples of 2^power up to 2^(power + 7), and whose
    largest a few rows share: out is the mean of these rows' values, by the roundings of sums
    and output alone, and lse the score and the logarithm of their number."""
    torch, ops = env
    b, t, h, g, p = FORMS[form]
    d, r = 64, 20
    lens = [(20, 1, -1, 0)[i % 4] for i in range(b)]
    x, lens = make(torch, dtype, b, t, h, g, d, p, r, seed=power, lens=lens)
    gen = torch.Generator().manual_seed(power)
    x["q"].zero_()
    half = power // 2
    x["q"][..., 3] = sign * 8 * 2.0 ** half  # (1 / sqrt(64) = 1 / 8)
    for name in ("kp", "ko"):
        x[name][..., 3] = torch.randint(-100, 101, x[name].shape[:-1], generator=gen).to(x[name].dtype) * 2.0 ** (power - half)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ops.prefix_attention(*(x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")), n, return_lse=True)
    ref, rl, _, vmax = reference(x, lens)
    tol = vmax * (64 * EPS + (2.0 ** -8 if dtype == "bf16" else 0))
    assert np.abs(out.double().cpu().numpy() - ref).max() <= tol
    got = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), np.isneginf(rl))
    live = np.isfinite(rl)
    assert (np.abs(got[live] - rl[live]) <= 8 * EPS * np.abs(rl[live]) + 64 * EPS).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_scores_of_very_different_sizes_in_one_tile(env, dtype, form):
    """Queries of ordinary size beside ones with scores of 2^40: each as if alone."""
    torch, ops = env
    b, t, h, g, p = FORMS[form]
    x, lens = make(torch, dtype, b, t, h, g, 64, p, 20, seed=9, lens=[(20, 1, 7, 0)[i % 4] for i in range(b)])
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    big = {k: v.clone() for k, v in x.items()}
    big["q"][1::2] *= 2.0 ** 40
    out = ops.prefix_attention(*(big[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")), n)
    assert torch.isfinite(out).all()
    ref, _, s, vmax = reference(x, lens)
    got = out.double().cpu().numpy()[::2]
    assert np.abs(got - ref[::2]).max() <= tolerance(dtype, 64, s, vmax)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["queries", "cache", "own rows"])
def test_an_out_between_its_inputs_elements(env, dtype, where):
    """Beside the queries in one projection's rows, in a cache's rows behind the prefix, in
    the heads of own rows that are not read: no element is shared, none but out's is written."""
    torch, ops = env
    b, t, h, g, d, p, r = 5, 3, 4, 4, 64, 300, 21
    x, lens = make(torch, dtype, b, t, h, g, d, p, r)
    want = check(torch, ops, dtype, x, lens)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    a = {k: v.cuda() for k, v in x.items()}
    zeros = lambda *s: torch.zeros(s, dtype=x["q"].dtype, device="cuda")  # noqa: E731
    if where == "queries":
        room = zeros(b, t, 2, h, d)
        a["q"], out = room[:, :, 0].copy_(a["q"]), room[:, :, 1]
    elif where == "cache":
        room = zeros(g, p + b * t, d)
        a["kp"], out = room[:, :p].copy_(a["kp"]), room[:, p:].unflatten(1, (b, t)).permute(1, 2, 0, 3)
        a["vp"] = zeros(g, p + b * t, d)[:, :p].copy_(a["vp"])
    else:
        room = zeros(b, 2, g, r, d)
        a["ko"], out = room[:, 0].copy_(a["ko"]), room[:, 1, :, :t].transpose(1, 2)
        a["vo"] = zeros(b, 2, g, r, d)[:, 0].copy_(a["vo"])
    before = room.clone()
    ops.prefix_attention(a["q"], a["kp"], a["vp"], a["ko"], a["vo"], n, out=out)
    assert torch.equal(out, want)
    out.zero_()
    assert torch.equal(room, before)


@pytest.mark.parametrize("heads,rows,seqs", [(192, 128, 512), (64, 128, 384), (384, 64, 192), (64, 136, 1000)])
def test_an_out_of_any_order(env, heads, rows, seqs):
    """2 heads, 3 queries, 2 sequences of 64 elements: one with strides that do not nest."""
    torch, ops = env
    x, lens = make(torch, "bf16", 2, 3, 2, 2, 64, 100, 9)
    want = check(torch, ops, "bf16", x, lens)
    room = torch.full((8192,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room.as_strided(want.shape, (seqs, rows, heads, 1))
    args = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
    ops.prefix_attention(*args, out=out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert (room == 7).all()


def test_a_scale_that_changes_in_place(env):
    torch, ops = env
    x, lens = make(torch, "f32", 3, 1, 2, 2, 64, 40, 8, lens=[8, 3, 0])
    scale = torch.tensor(0.1)
    args = [x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")] + [torch.tensor(lens, dtype=torch.int32, device="cuda")]
    for _ in range(2):
        assert torch.equal(ops.prefix_attention(*args, scale=scale), ops.prefix_attention(*args, scale=float(scale)))
        scale.mul_(3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("kind", ["nan-queries", "large-queries", "nan-rows", "off", "other-lengths"])
def test_other_sequences_of_the_batch(env, dtype, form, kind):
    """Every second sequence is replaced: the others' results stay right (not bitwise, the
    columns of a tile take new references together)."""
    torch, ops = env
    b, t, h, g, p = FORMS[form]
    x, lens = make(torch, dtype, b, t, h, g, 64, p, 20, seed=4, lens=[(20, 13, 7, 1)[i % 4] for i in range(b)])
    ref, rl, big, vmax = reference(x, lens)
    if kind == "nan-queries":
        x["q"][1::2] = float("nan")
    elif kind == "large-queries":
        x["q"][1::2] *= 2.0 ** 33
    elif kind == "nan-rows":
        x["ko"][1::2] = x["vo"][1::2] = float("nan")
    else:
        lens = [n if i % 2 == 0 else -1 if kind == "off" else 20 - n for i, n in enumerate(lens)]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ops.prefix_attention(*(x[k].cuda() for k in ("q", "kp", "vp", "ko", "vo")), n, return_lse=True)
    assert np.abs(out[::2].double().cpu().numpy() - ref[::2]).max() <= tolerance(dtype, 64, big, vmax)
    assert np.abs(lse[::2].double().cpu().numpy() - rl[::2]).max() <= 68 * EPS * big + 64 * EPS * (1 + np.abs(rl).max())
    if kind == "off":
        assert not out[1::2].any() and torch.isneginf(lse[1::2]).all()
    if kind == "nan-queries":
        assert torch.isnan(out[1::2]).all() and torch.isnan(lse[1::2]).all()


def test_strides_of_dimensions_of_one_entry_do_not_matter(env):
    """One kv head or one sequence: keys from one cache, values from a longer one."""
    torch, ops = env

    def inside(t, dim):  # t in a buffer with more entries of a dimension
        shape = list(t.shape)
        shape[dim] += 3
        room = torch.full(shape, float("nan"), dtype=t.dtype, device="cuda")
        return room[tuple(slice(n) for n in t.shape)].copy_(t)

    x, lens = make(torch, "bf16", 3, 1, 4, 1, 64, 40, 8)
    check(torch, ops, "bf16", x, lens, put=lambda name, t: inside(t, 1) if name == "vp" else t.cuda())
    x, lens = make(torch, "bf16", 1, 1, 4, 2, 64, 40, 8)
    check(torch, ops, "bf16", x, lens, put=lambda name, t: inside(t, 1) if name == "vo" else t.cuda())
    x, lens = make(torch, "bf16", 1, 1, 4, 1, 64, 1, 1, lens=[1])
    check(torch, ops, "bf16", x, lens, put=lambda name, t: inside(t, 1) if name in ("vp", "vo") else t.cuda())
