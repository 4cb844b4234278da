"""Tree verification of a batch over the paged cache (batch.py) against the verification pass of one sequence.

The pass reads a dense cache that holds what the pages stand for, and the open rows; so both are float32 chains over
the same numbers with sums in other orders: 1e-4 of the logits' scale, as between the rollout and the pass
(test_gpu_distill), bfloat16 2e-2."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2308_04623_amd import batch, paged, ssd, staged, workloads
    assert torch.cuda.is_available()
    return torch, batch, paged, ssd, staged, workloads


def setup(env, dtype, prompts, n_seq, nodes, **kw):
    torch, batch, _, ssd, staged, W = env
    cfg = W.TINY.with_(dtype=dtype)
    session = ssd.Session(ssd.Model(cfg, W.make_weights(cfg, 0, perturb_affine=True)), 160, 64)
    b = batch.Batch(session.model, n_seq, 160, nodes, **kw)
    for slot, n in prompts.items():
        prompt = W.prefix_tokens(n, cfg.vocab, seed=slot + 1)
        assert staged.GpuBackend(session, session).prefill(prompt) == n
        b.admit(slot, session, n)
    return session, b


def dense(env, session, b, slot):
    """The session's cache becomes what slot's pages stand for and its open rows."""
    torch, _, paged, *_ = env
    n, rows = int(b.length[slot]), b.page_rows
    full = n // rows
    k, v = paged.pages_load(b.pages, b.table[slot, :full].contiguous(), b.k_tail.dtype)
    at = torch.arange(full * rows, n, device=k.device)
    for cache, x, tail in ((session.k_cache, k, b.k_tail), (session.v_cache, v, b.v_tail)):
        cache[:, :, :full * rows] = x.transpose(1, 2).flatten(2, 3)
        cache[:, :, at] = tail[:, slot][:, :, at % b.ring]
    return n


def trees(rng, n_seq, nodes, vocab):
    parents = np.full((n_seq, nodes), -2, np.int32)
    for b in range(n_seq):
        for i in range(nodes - b % 3):
            parents[b, i] = rng.integers(0, i) if i else -1
    return rng.integers(0, vocab, (n_seq, nodes)).astype(np.int32), parents


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("code,rows", [("int8", 32), ("e4m3", 64)])
def test_the_batch_agrees_with_the_verification_pass(env, dtype, tol, code, rows):
    torch, *_ = env
    session, b = setup(env, dtype, {0: 70, 1: 1, 3: 131}, 5, 9, code=code, page_rows=rows)
    b.fork([0, 1, 0, 3, -1])
    rng = np.random.default_rng(0)
    for step in range(4):
        tokens, parents = trees(rng, 5, 9, 512)
        got = b.verify(torch.from_numpy(tokens).cuda(), parents)
        for slot in (0, 1, 2, 3):
            n = dense(env, session, b, slot)
            keep = parents[slot] >= -1
            want = session.verify(n, tokens[slot][keep], parents[slot][keep])
            err = (got[slot][torch.from_numpy(keep).cuda()] - want).abs().max()
            assert err <= tol * want.abs().max(), (step, slot)
        path = torch.zeros((5, 9), dtype=torch.int32)
        length = torch.zeros(5, dtype=torch.int32)
        for slot in range(4):  # any path from the root
            node, nodes = int(rng.integers(0, 7)), []
            while node >= 0:
                nodes.append(node)
                node = int(parents[slot, node])
            path[slot, :len(nodes)] = torch.tensor(nodes[::-1], dtype=torch.int32)
            length[slot] = len(nodes)
        before = b.length.clone()
        assert (b.commit(path.cuda(), length.cuda()) >= 0).all()
        assert torch.equal(b.length[:4], (before + length.cuda())[:4]) and int(b.length[4]) == -1
        b.compact()


def test_greedy_decoding_in_a_batch(env):
    """Every token is the model's choice after those before it; sequences that share a prompt's pages and are fed alike emit
    alike; pages add up."""
    torch, batch, *_ = env
    out, b = batch.main(n_seq=6, n_steps=10)
    assert all(len(o) >= 11 for o in out)
    held = torch.bincount(b.table[b.table >= 0], minlength=b.pages.n_page)
    assert torch.equal(held.int(), b.refs)
    session, b = setup(env, "f32", {0: 50}, 3, 8)
    b.fork([0, 0, -1])
    succ = np.tile(np.arange(8), (512, 1))
    out = batch.staged_greedy(b, [7, 7, 0], 6, succ)
    assert out[0] == out[1] and out[2] == [0]
    # one token a step, from the same prompt, over the same cache as it was before the last step
    session, b = setup(env, "f32", {0: 50}, 1, 1)
    toks = [7]
    for _ in range(6):
        t = torch.tensor([[toks[-1]]], dtype=torch.int32, device="cuda")
        n = dense(env, session, b, 0)
        want = session.verify(n, [toks[-1]], np.array([-1], np.int32))
        path, length, after = b.accept(t, [[-1]], b.verify(t, [[-1]]))
        b.commit(path, length)
        assert int(after[0]) == int(want[0].argmax()) and int(length[0]) == 1
        toks.append(int(after[0]))
    assert toks == out[0][:7]


def test_a_windowed_batch_gives_pages_back(env):
    torch, batch, *_ = env
    session, b = setup(env, "f32", {0: 90, 1: 64}, 2, 4, window=40, sinks=3)
    tokens, parents = np.zeros((2, 4), np.int32), np.tile(np.arange(-1, 3, dtype=np.int32), (2, 1))
    path = torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1)
    for step in range(12):
        b.verify(torch.from_numpy(tokens).cuda(), parents)
        assert (b.commit(path, torch.full((2,), 4, dtype=torch.int32, device="cuda")) >= 0).all()
    assert b.length.tolist() == [138, 112]
    # pages 1 and 2 of rows 32 .. 95 lie behind 138 - 40, page 1 behind 112 - 40
    assert (b.table >= 0).tolist() == [[True, False, False, True, False], [True, False, True, False, False]]


def test_refusals(env):
    torch, batch, _, ssd, staged, W = env
    session, b = setup(env, "f32", {0: 50}, 2, 4, n_page=1)
    for slot, n in ((0, 10), (2, 10), (-1, 10), (1, 161), (1, -1)):
        with pytest.raises(ValueError):
            b.admit(slot, session, n)
    with pytest.raises(RuntimeError):
        b.admit(1, session, 64)
    b.admit(1, session, 31)  # (an open page is the tail's)
    tokens = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        b.verify(tokens, [[-1, 0, 1, 3], [-1, 0, 1, 2]])
    with pytest.raises(ValueError):
        b.verify(tokens[:, :3], [[-1, 0, 1], [-1, 0, 1]])
    with pytest.raises(ValueError):
        batch.Batch(session.model, 2, 256, 4)
    for kw in (dict(max_nodes=65), dict(max_nodes=0), dict(n_seq=0), dict(page_rows=48), dict(window=3), dict(sinks=-1)):
        with pytest.raises(ValueError):
            batch.Batch(**{**dict(model=session.model, n_seq=2, max_ctx=96, max_nodes=4), **kw})
    # another model's cache is refused before pages are taken for it
    cfg = W.TINY.with_(dtype="bf16")
    other = ssd.Session(ssd.Model(cfg, W.make_weights(cfg, 0)), 160, 64)
    b.fork([0, -1])
    used = b.refs.clone()
    with pytest.raises(ValueError):
        b.admit(1, other, 40)
    assert torch.equal(b.refs, used) and int(b.length[1]) == -1
