"""The operators together (distill.py): continuations over one cached prompt,
their distillation into a bigram student, its gradients.

Tolerances.  The rollout's float32 logits against the verification pass: both
are float32 chains over the same weights with sums in other orders; a layer's
rounding is some sqrt(width) eps of its size, so 1e-4 of the logits' scale leaves
more than a factor of ten.  bfloat16: activations are rounded to 2^-9 at other
places, the parity bound of the verification pass against its oracle, 2e-2
of the logits' scale.  Gradients against differences of the loss in 64 bits
with a step of 1e-5: the quotient is good to 1e-9, the float32 gradient to some
hundred eps of its largest terms, so 1e-4 of the largest entry."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2308_04623_amd import distill, ssd, staged, workloads
    assert torch.cuda.is_available()
    return torch, distill, ssd, staged, workloads


def oracle_at(env, dtype, prefix):
    torch, _, ssd, staged, W = env
    cfg = W.TINY.with_(dtype=dtype)
    session = ssd.Session(ssd.Model(cfg, W.make_weights(cfg, 0, perturb_affine=True)), 128, 32)
    prompt = W.prefix_tokens(prefix + 1, cfg.vocab)
    assert staged.GpuBackend(session, session).prefill(prompt[:-1]) == prefix
    return session, int(prompt[-1])


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("prefix", [1, 37, 90])
def test_rollout_agrees_with_the_verification_pass(env, dtype, tol, prefix):
    torch, distill, ssd, staged, W = env
    session, root = oracle_at(env, dtype, prefix)
    rollout = distill.Rollout(session, 3, 12)
    tokens = torch.from_numpy(np.stack([W.prefix_tokens(12, 512, seed=s) for s in (5, 6, 7)])).int().cuda()
    got = torch.stack([rollout.logits(prefix, tokens[:, i].contiguous(), i) for i in range(12)], 1)
    for b in range(3):
        want = session.verify(prefix, tokens[b].cpu().numpy(), np.arange(-1, 11, dtype=np.int32))
        assert (got[b] - want).abs().max() <= tol * want.abs().max()


def test_sampled_tokens_are_the_teachers(env):
    torch, distill, *_ = env
    session, root = oracle_at(env, "f32", 20)
    rollout = distill.Rollout(session, 40, 6)  # (more sequences than the session's nodes)
    draw = lambda: rollout.sample(20, root, 6, 4, generator=torch.Generator("cuda").manual_seed(3))  # noqa: E731
    tokens, ids, vals = draw()
    assert tokens.shape == (240,) and ids.shape == vals.shape == (240, 4)
    assert (tokens[:40] == root).all()
    assert (tokens[40:, None] == ids[:-40]).any(1).all()  # every token is one of the four before it
    assert (vals[:, :-1] >= vals[:, 1:]).all()
    assert all(torch.equal(a, b) for a, b in zip(draw(), (tokens, ids, vals)))
    with pytest.raises(ValueError):
        rollout.logits(20, tokens[:40], 6)


def test_gradients_against_differences(env):
    torch, distill, *_ = env
    gen = torch.Generator().manual_seed(0)
    v, d, n, k = 60, 16, 40, 5
    student = distill.BigramStudent(v, d, seed=2)
    tokens = torch.randint(0, 20, (n,), generator=gen).int()  # some often, some never
    ids = torch.rand(n, v, generator=gen).topk(k, 1).indices.int()
    vals, weight = torch.randn(n, k, generator=gen), torch.rand(n, generator=gen)
    weight[3] = 0
    T = 1.3
    _, dtable, dmix = student.gradients(tokens.cuda(), ids.cuda(), vals.cuda(), weight.cuda(), T)

    def objective(table, mix):
        logp = torch.log_softmax((student.scale * table[tokens.long()] @ mix) @ table.t() / T, 1)
        p = torch.softmax(vals.double() / T, 1)
        return (weight.double() * (p * (p.log() - logp.gather(1, ids.long()))).sum(1)).sum()

    table, mix = student.table.double().cpu(), student.mix.double().cpu()
    for got, x, other in ((dtable, table, lambda y: objective(y, mix)), (dmix, mix, lambda y: objective(table, y))):
        got = got.double().cpu()
        for i in torch.randint(0, x.numel(), (60,), generator=gen).tolist():
            plus, minus = x.clone(), x.clone()
            plus.view(-1)[i] += 1e-5
            minus.view(-1)[i] -= 1e-5
            assert abs((other(plus) - other(minus)).item() / 2e-5 - got.view(-1)[i].item()) <= 1e-4 * got.abs().max()


def test_a_student_learns_the_oracles_continuations(env):
    _, distill, *_ = env
    before, after = distill.main(n_seq=16, n_new=16, steps=40)
    assert after[0] < 0.5 * before[0] and after[1] < before[1]


def test_successors_feed_the_staged_loop(env):
    torch, distill, ssd, staged, W = env
    session, root = oracle_at(env, "f32", 20)
    succ = distill.BigramStudent(512, 64).successors(session)
    assert succ.shape == (512, staged.BIGRAM_TOP) and succ.min() >= 0 and succ.max() < 512
    tokens, parents = staged.bigram_tree(root, succ)
    depth = [0]
    for p in parents[1:]:
        depth.append(depth[p] + 1)
    assert ssd.validate_tree(tokens, parents, 512) == max(depth)  # (raises on a tree that is none)


@pytest.mark.parametrize("prefix,step", [(129, 0), (200, 3), (-1, 0), (20, -1), (20, 12)])
def test_a_rollout_refuses_places_outside_its_caches(env, prefix, step):
    """The session's cache has 128 rows, the rollout's 12, the model 256 positions."""
    torch, distill, *_ = env
    session, root = oracle_at(env, "f32", 20)
    rollout = distill.Rollout(session, 2, 12)
    with pytest.raises(ValueError):
        rollout.logits(prefix, torch.zeros(2, dtype=torch.int32, device="cuda"), step)
