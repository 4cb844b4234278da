"""ops.distill_forward / _backward / _step against the definition in 64 bits.

Tolerances, set from the arithmetic (eps = 2^-24): x = z / T carries |x| eps; an
exponential of an argument up to |x| apart is then off by a few |x| eps
relatively, the sum's error is that plus the roundings of a chain of at most
some hundred additions.  So lse is off by at most eps (4 X + 256) with X the
largest |x| of the row or its teacher, a probability relatively by the same,
the loss by twice that per unit of weight; bfloat16 gradients are rounded once,
2^-9 of themselves."""
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


def make(torch, dtype, n, v, k, seed=0):
    gen = torch.Generator().manual_seed(seed)
    z = (torch.randn(n, v, generator=gen) * 2.5).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    teacher = z.float() + torch.randn(n, v, generator=gen)
    top = teacher.topk(min(k, v), 1)
    w = torch.rand(n, generator=gen) + 0.25
    return z, top.indices.int().contiguous(), top.values.contiguous(), w


def reference(z, ids, vals, w, T, lse=None):
    """loss, lse, gradient and X in 64 bits."""
    z, ids = z.double().numpy(), ids.numpy()
    vals, w = vals.double().numpy(), w.double().numpy()
    n, v = z.shape
    loss, ls, g, X = np.zeros(n), np.zeros(n), np.zeros((n, v)), np.zeros(n)
    with np.errstate(all="ignore"):
        for i in range(n):
            x = z[i] / T
            m = x.max()
            l = m + math.log(np.exp(x - m).sum())
            ls[i] = l
            if lse is not None:
                l = float(lse[i])
            ok = (ids[i] >= 0) & (ids[i] < v) & ~np.isneginf(vals[i])
            fin = x[np.isfinite(x)]
            X[i] = max(np.abs(fin).max(initial=0.0), np.abs(vals[i][ok] / T).max(initial=0.0))
            if w[i] == 0 or not ok.any():
                continue
            t = vals[i][ok] / T
            p = np.exp(t - t.max())
            p /= p.sum()
            q = np.exp(x - l)
            logq = x[ids[i][ok]] - l
            live = p > 0
            loss[i] = w[i] * (p[live] * (np.log(p[live]) - logq[live])).sum()
            np.subtract.at(q, ids[i][ok], p)
            g[i] = w[i] / T * q
    return loss, ls, g, X


def close(dtype, got, ref, tol):
    assert (np.abs(got - ref) <= tol + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-37).all()


def check(torch, ops, dtype, z, ids, vals, w, T=1.0, put=lambda t: t.cuda(), **kw):
    dz, di, dv, dw = put(z), ids.cuda(), vals.cuda(), w.cuda()
    rloss, rlse, rg, X = reference(z, ids, vals, w, T)
    unit = EPS * (4 * X + 256)
    wn = w.double().numpy()
    loss, lse = ops.distill_forward(dz, di, dv, dw, temperature=T)
    back = ops.distill_backward(dz, di, dv, lse, dw, temperature=T)
    loss2, lse2, grad = ops.distill_step(dz, di, dv, dw, temperature=T, **kw)
    torch.cuda.synchronize()
    scale = (np.abs(wn) / T * unit)[:, None]
    mag = np.abs(rg) * T / np.maximum(np.abs(wn), 1e-30)[:, None]
    for i in range(z.shape[0]):  # p + q where p is
        for j in range(ids.shape[1]):
            if 0 <= ids[i, j] < z.shape[1]:
                mag[i, ids[i, j]] += 2
    for a, b in ((loss, lse), (loss2, lse2)):
        assert (np.abs(a.double().cpu().numpy() - rloss) <= 2 * wn * unit).all()
        assert (np.abs(b.double().cpu().numpy() - rlse) <= unit).all()
    close(dtype, grad.double().cpu().numpy(), rg, scale * mag)
    rb = reference(z, ids, vals, w, T, lse=lse.cpu())[2]
    close(dtype, back.double().cpu().numpy(), rb, scale * mag)
    return loss2, lse2, grad


SHAPES = [(1, 1, 1), (1, 2, 1), (3, 7, 3), (15, 512, 8), (5, 511, 8), (4, 1000, 64), (3, 1025, 65), (2, 4097, 128),
          (2, 8193, 16), (3, 16411, 50), (2, 50257, 8), (3, 65536, 8), (2, 65537, 50), (1, 131072, 100),
          (2, 131075, 128), (1, 200003, 7), (700, 33, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v,k", SHAPES)
def test_against_64_bits(env, dtype, n, v, k):
    torch, ops = env
    print(dtype, n, v, k, flush=True)
    check(torch, ops, dtype, *make(torch, dtype, n, v, k, seed=v))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [100, 20000, 131072])
@pytest.mark.parametrize("T", [0.5, 3.0])
def test_temperatures(env, dtype, v, T):
    torch, ops = env
    check(torch, ops, dtype, *make(torch, dtype, 4, v, 20), T=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 40001, 140000])
def test_slots_and_rows_that_are_left_out(env, dtype, v):
    torch, ops = env
    z, ids, vals, w = make(torch, dtype, 7, v, 9)
    w[0] = 0.0                        # a row of weight 0
    ids[1] = -1                       # no token at all
    vals[2] = -math.inf               # no probability at all
    ids[3, 2], ids[3, 5] = v, -7      # outside the vocabulary
    vals[4, 1] = -math.inf
    ids[5] = ids[5, 0]                # one token in every slot
    vals[6] = -300.0                  # far below, all alike
    loss, lse, grad = check(torch, ops, dtype, z, ids, vals, w)
    assert not loss[:3].any() and not grad[:3].any()
    z[:3] = float("nan")              # such rows may hold anything
    loss, lse, grad = ops.distill_step(z.cuda(), ids.cuda(), vals.cuda(), w.cuda())
    assert not loss[:3].any() and not grad[:3].any()
    assert torch.isfinite(grad).all() and torch.isfinite(loss).all()
    back = ops.distill_backward(z.cuda(), ids.cuda(), vals.cuda(), lse, w.cuda())
    assert not back[:3].any() and torch.isfinite(back).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 40001, 140000])
def test_infinities(env, dtype, v):
    torch, ops = env
    z, ids, vals, w = make(torch, dtype, 4, v, 5)
    keep = torch.zeros(4, v, dtype=torch.bool).scatter_(1, ids.long(), True)
    z[0][~keep[0]] = -math.inf        # the student allows the teacher's tokens only
    z[1][~keep[1]] = torch.finfo(z.dtype).min
    loss, lse, grad = check(torch, ops, dtype, z, ids, vals, w)
    assert not grad[0][~keep[0].cuda()].any()
    z[2, ids[2, 1]] = -math.inf       # it forbids one of them
    loss, _, grad = ops.distill_step(z.cuda(), ids.cuda(), vals.cuda(), w.cuda())
    assert math.isinf(loss[2]) and loss[2] > 0 and torch.isfinite(grad[2]).all()
    z[3, v // 2] = math.nan
    loss, lse, grad = ops.distill_step(z.cuda(), ids.cuda(), vals.cuda(), w.cuda())
    assert torch.isnan(loss[3]) and torch.isnan(lse[3]) and torch.isnan(grad[3]).all()
    assert torch.isfinite(grad[:3]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(env, dtype):
    torch, ops = env
    z, ids, vals, w = make(torch, dtype, 3, 5000, 8)
    z[0] += 1e4
    z[1] *= 30
    check(torch, ops, dtype, z, ids, vals, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [333, 50257, 131200])
def test_strides_and_alignment(env, dtype, v):
    """Rows at any element; what lies between them is left alone."""
    torch, ops = env
    z, ids, vals, w = make(torch, dtype, 4, v, 8)
    for off in (0, 1, 3):
        room = torch.full((4 * (v + 5) + off,), 7.0, dtype=z.dtype, device="cuda")
        view = room[off:].view(4, v + 5)[:, :v]
        view.copy_(z)
        dest = torch.full((4 * (v + 9) + off,), 5.0, dtype=z.dtype, device="cuda")
        dview = dest[off:].view(4, v + 9)[:, :v]
        check(torch, ops, dtype, z, ids, vals, w, put=lambda t: view, out=dview)
        assert (dest[off:].view(4, v + 9)[:, v:] == 5).all() and (dest[:off] == 5).all()
        assert (room[off:].view(4, v + 5)[:, v:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [90, 50257, 140001])
def test_in_place(env, dtype, v):
    torch, ops = env
    z, ids, vals, w = (t.cuda() for t in make(torch, dtype, 5, v, 12))
    loss, lse, grad = ops.distill_step(z, ids, vals, w)
    back = ops.distill_backward(z, ids, vals, lse, w)
    a, b = z.clone(), z.clone()
    l2, s2, g2 = ops.distill_step(a, ids, vals, w, out=a)
    assert g2 is a and torch.equal(a, grad) and torch.equal(l2, loss) and torch.equal(s2, lse)
    ops.distill_backward(b, ids, vals, lse, w, out=b)
    assert torch.equal(b, back)


def test_without_weights_and_again(env):
    torch, ops = env
    z, ids, vals, w = (t.cuda() for t in make(torch, "f32", 6, 3001, 8))
    a = ops.distill_step(z, ids, vals)
    b = ops.distill_step(z, ids, vals, torch.ones_like(w))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = ops.distill_step(z, ids, vals, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(a, c))
    assert ops.distill_forward(z[:0], ids[:0], vals[:0])[0].shape == (0,)


def test_gradient_against_differences(env):
    """Central differences of the loss, step h: the loss is off by at most the
    tolerance above (twice, over 2h), and the remainder is h^2 / 6 times the
    third derivative of a log-sum-exp, at most 0.1 / T^3 w."""
    torch, ops = env
    v, k, T, h = 11, 4, 0.8, 2e-2
    z, ids, vals, w = make(torch, "f32", 1, v, k)
    loss, lse, grad = ops.distill_step(z.cuda(), ids.cuda(), vals.cuda(), w.cuda(), temperature=T)
    up, down = z.repeat(v, 1) + h * torch.eye(v), z.repeat(v, 1) - h * torch.eye(v)
    many = lambda t: t.repeat(v, *([1] * (t.dim() - 1))).cuda()  # noqa: E731
    lu = ops.distill_forward(up.cuda(), many(ids), many(vals), many(w), temperature=T)[0].double()
    ld = ops.distill_forward(down.cuda(), many(ids), many(vals), many(w), temperature=T)[0].double()
    step = (up.double() - down.double()).diagonal().cuda()
    X = max(float(z.abs().max()), float(vals.abs().max())) / T
    tol = 2 * 2 * float(w[0]) * EPS * (4 * X + 256) / (2 * h) + h * h / 6 * 0.1 * float(w[0]) / T ** 3
    assert float(((lu - ld) / step - grad[0].double()).abs().max()) <= tol


def test_offsets_past_32_bits(env):
    torch, ops = env
    z, ids, vals, w = make(torch, "bf16", 3, 700, 5)
    step = 1500000000
    room = torch.empty(2 * step + 700, dtype=torch.bfloat16, device="cuda")
    view = room.as_strided((3, 700), (step, 1))
    view.copy_(z)
    check(torch, ops, "bf16", z, ids, vals, w, put=lambda t: view)
    a = ops.distill_step(z.cuda(), ids.cuda(), vals.cuda(), w.cuda())[2]
    ops.distill_step(view, ids.cuda(), vals.cuda(), w.cuda(), out=view)
    assert torch.equal(view, a)


def test_captured_in_a_graph(env):
    torch, ops = env
    z, ids, vals, w = (t.cuda() for t in make(torch, "bf16", 40, 5001, 8))
    out = torch.empty_like(z)
    ops.distill_step(z, ids, vals, w, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, lse, _ = ops.distill_step(z, ids, vals, w, out=out)
    for _ in range(3):
        z.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        a = ops.distill_step(z, ids, vals, w)
        assert torch.equal(a[0], loss) and torch.equal(a[1], lse) and torch.equal(a[2], out)


def test_refusals_of_the_binding(env):
    torch, ops = env
    from paper_2308_04623_amd.ssd import SSDError
    z, ids, vals, w = (t.cuda() for t in make(torch, "f32", 4, 100, 6))
    for bad in ((z.half(), ids, vals, w), (z, ids.long(), vals, w), (z, ids, vals.double(), w), (z, ids[:3], vals, w),
                (z, ids, vals, w[:3]), (z, ids, vals, w.cpu()), (z.t(), ids, vals, w), (z[0], ids, vals, w),
                (z, ids[:, ::2], vals[:, ::2], w)):
        with pytest.raises(SSDError):
            ops.distill_forward(*bad)
    with pytest.raises(SSDError):
        ops.distill_step(z, ids, vals, w, temperature=0.0)
    with pytest.raises(SSDError):
        ops.distill_step(z, ids, vals, w, out=z.bfloat16())
    both = torch.zeros(5, 100, device="cuda")
    with pytest.raises(SSDError):
        ops.distill_step(both[:4], ids, vals, w, out=both[1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("chunks", [900, 1024, 1025, 2560, 2561, 4096, 4097, 6400, 6401, 6656, 6657, 8192, 8193, 13312,
                                    13313, 16384, 16385, 24576, 24577])
@pytest.mark.parametrize("odd", [0, 3])
def test_many_rows_of_every_length(env, dtype, chunks, odd):
    """More rows than compute units, five of them distinct, of as many 16-byte chunks as
    the registers hold and one more; odd: rows that begin at any element."""
    torch, ops = env
    v = chunks * (4 if dtype == "f32" else 8) + odd
    z, ids, vals, w = make(torch, dtype, 5, v, 9, seed=chunks)
    rows = torch.arange(260) % 5
    wide = torch.empty(260, v + odd, dtype=z.dtype, device="cuda")
    many = wide[:, :v]
    many.copy_(z.cuda()[rows.cuda()])
    args = [x.cuda()[rows.cuda()] for x in (ids, vals, w)]
    rloss, rlse, rg, X = reference(z, ids, vals, w, 1.0)
    unit, wn = EPS * (4 * X + 256), w.double().numpy()
    mag = np.abs(rg) / wn[:, None]
    np.put_along_axis(mag, ids.numpy().astype(np.int64), np.take_along_axis(mag, ids.numpy().astype(np.int64), 1) + 2, 1)
    forward = ops.distill_forward(many, *args)
    back = ops.distill_backward(many, *args[:2], forward[1], args[2])
    step = ops.distill_step(many, *args, out=many)  # in place
    assert step[2].data_ptr() == many.data_ptr()
    for loss, lse in (forward, step[:2]):
        assert (np.abs(loss[:5].double().cpu().numpy() - rloss) <= 2 * wn * unit).all()
        assert (np.abs(lse[:5].double().cpu().numpy() - rlse) <= unit).all()
    rb = reference(z, ids, vals, w, 1.0, lse=forward[1][:5].cpu())[2]
    close(dtype, many[:5].double().cpu().numpy(), rg, (wn * unit)[:, None] * mag)
    close(dtype, back[:5].double().cpu().numpy(), rb, (wn * unit)[:, None] * mag)
    if not odd:  # rows alike give the same, wherever they stand
        for x in (*forward, back, *step):
            assert torch.equal(x[5:10], x[:5]) and torch.equal(x[255:], x[:5])


# more rows than one launch takes (2^21): rows of both sides of the cut and of the ends
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_a_launch(env, dtype):
    torch, ops = env
    cut, v, k, T = 1 << 21, 24, 2, 1.25
    z, ids, vals, w = make(torch, dtype, 64, v, k)
    n = cut + 77
    big = [torch.cat([t.cuda()] * (n // 64 + 1))[:n].contiguous() for t in (z, ids, vals, w)]
    loss, lse, grad = ops.distill_step(*big, temperature=T)
    loss2, lse2 = ops.distill_forward(*big, temperature=T)
    back = ops.distill_backward(*big[:3], lse, big[3], temperature=T)
    small = [t.cuda() for t in (z, ids, vals, w)]
    a = ops.distill_step(*small, temperature=T)
    b = ops.distill_backward(*small[:3], a[1], small[3], temperature=T)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    for got, want in ((loss, a[0]), (lse, a[1]), (grad, a[2]), (back, b)):
        want = torch.cat([want] * (n // 64 + 1))[:n]
        assert torch.equal(got, want)
    check(torch, ops, dtype, z, ids, vals, w, T=T)


def far_rows(torch, dtype, v, k, sizes):
    """Rows of one value each, then two of ordinary spread around one whose maximum is the
    teacher's first token."""
    z, ids, vals, w = make(torch, dtype, len(sizes) + 2, v, k, seed=v)
    for i, c in enumerate(sizes):
        z[i] = c
    ids[-2:, 0] = v // 2
    z[-2, v // 2] = max(sizes) / 2
    z[-1] -= max(sizes)
    z[-1, v // 2] = -max(sizes) / 2
    return z, ids, vals, w


# Against 64 bits with tolerances that do not grow with the logits: an entry z enters by
# (z - max) / T alone, off by a few eps of itself, so everything but lse, which is rounded as a
# number of its size, is off by EPS (4 Y + 256) with Y the largest such difference that matters: of the
# entries whose exponential is not 0 (120 and a little), and of the teacher's tokens for the loss.
# Exponentials below 2^-126 are 0.
def far_check(torch, ops, dtype, z, ids, vals, w, T):
    dev = [x.cuda() for x in (z, ids, vals, w)]
    T = float(np.float32(T))
    forward = ops.distill_forward(*dev, temperature=T)
    step = ops.distill_step(*dev, temperature=T)
    zz, tv, wn = z.double().numpy(), vals.double().numpy(), w.double().numpy()
    x = (zz - zz.max(1, keepdims=True)) / T
    total = np.exp(x).sum(1)
    lse = zz.max(1) / T + np.log(total)
    p = np.exp((tv - tv.max(1, keepdims=True)) / T)
    p /= p.sum(1, keepdims=True)
    at = ids.long().numpy()
    logq = np.take_along_axis(x, at, 1) - np.log(total)[:, None]
    loss = wn * np.where(p > 0, p * (np.log(np.where(p > 0, p, 1)) - logq), 0).sum(1)
    q = np.exp(x) / total[:, None]
    grad = q.copy()
    for i in range(len(at)):
        np.subtract.at(grad[i], at[i], p[i])
    grad *= (wn / T)[:, None]
    spread = np.abs(tv - tv.max(1, keepdims=True)).max(1) / T
    unit = EPS * (4 * (120 + spread) + 256)
    unit_loss = EPS * (4 * (np.abs(np.take_along_axis(x, at, 1)).max(1) + spread) + 256)
    mag = q
    np.put_along_axis(mag, at, np.take_along_axis(mag, at, 1) + 2, 1)
    for l, s in (forward, step[:2]):
        assert (np.abs(l.double().cpu().numpy() - loss) <= 2 * wn * unit_loss).all()
        assert (np.abs(s.double().cpu().numpy() - lse) <= EPS * (8 * np.abs(lse) + 256)).all()
    close(dtype, step[2].double().cpu().numpy(), grad, (wn / T)[:, None] * (unit[:, None] * mag + 2.0 ** -125))


# below 2^23 everywhere, beyond in rows that no registers hold
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,sizes", [(300, (-1e6, 5e6)), (40001, (-5e6, 1e6)), (200003, (-1e6, 1e10, -1e20))])
def test_the_loss_does_not_carry_the_logits_rounding(env, dtype, v, sizes):
    torch, ops = env
    far_check(torch, ops, dtype, *far_rows(torch, dtype, v, 6, sizes), 1.0)


# both sides of 2^24 (in units of log 2), where a row is done again by sweeps
SIZES = (-1e6, 1.1e7, 1.2e7, -1.2e7, 5e8, -1e9, 1e10, -1e10, -3e10, 1e20, -1e20, -1e29, 1e38)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 5000, 40001, 70001, 140000, 200003])
@pytest.mark.parametrize("T", [1.0, 0.5])
def test_logits_of_any_size(env, dtype, v, T):
    torch, ops = env
    far_check(torch, ops, dtype, *far_rows(torch, dtype, v, 6, SIZES), T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 40001, 200003])
@pytest.mark.parametrize("T", [1e-5, 2.0 ** -17, 1e-7])
def test_small_temperatures(env, dtype, v, T):
    """Masks of -65504 and logits around 5e4."""
    torch, ops = env
    z, ids, vals, w = make(torch, dtype, 4, v, 6, seed=3)
    z[0] = -65504.0
    z[1, v // 3] = 5e4
    z[2] += 5e4
    vals = vals * T  # (the teacher's distribution stays one)
    far_check(torch, ops, dtype, z, ids, vals, w, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [200, 5001])
def test_a_gradient_beside_the_logits_rows(env, dtype, v):
    """Columns of one buffer: no element is shared."""
    torch, ops = env
    z, ids, vals, w = (t.cuda() for t in make(torch, dtype, 5, v, 12))
    room = torch.zeros(5, 2 * v, dtype=z.dtype, device="cuda")
    left, right = room[:, :v].copy_(z), room[:, v:]
    # (from the same places: where a row begins decides the order of its sum)
    loss, lse, grad = ops.distill_step(left, ids, vals, w)
    assert torch.equal(ops.distill_step(left, ids, vals, w, out=right)[2], grad)
    back = ops.distill_backward(left, ids, vals, lse, w)
    assert torch.equal(ops.distill_backward(left, ids, vals, lse, w, out=right), back)
    assert torch.equal(left, z)
