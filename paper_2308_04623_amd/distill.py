"""Training a draft^2 on the oracle's own continuations of a prompt.

A draft is worth what it agrees with the oracle on the text that the oracle
writes (Sec. 3.2).  Here the oracle's session holds a prompt's keys and values;
Rollout writes a batch of continuations of it, all over that one cache
(ops.prefix_attention), and keeps the oracle's top logits at every position
(Session.topk).  BigramStudent is a bigram model with a tied table (its logits
after a token are (scale table[token] mix) table^T) that is fitted to those
logits (ops.embed, ops.distill_step, ops.embed_grad); its successors take the
place of staged.bigram_table's.

The dense products around the operators, the layers' and the student's, are
PyTorch's.  Run as a program for a small one from end to end:

    python -m paper_2308_04623_amd.distill
"""
from __future__ import annotations

import math
from typing import Tuple

import numpy as np
import torch
import torch.nn.functional as F

from . import ops, ssd
from .staged import BIGRAM_TOP


class Rollout:
    """Continuations of the prompt in a session's cache: n_seq sequences of up
    to max_new tokens each, with their own keys and values beside the cache's."""

    def __init__(self, session, n_seq: int, max_new: int):
        cfg, model = session.model.cfg, session.model
        if not isinstance(model, ssd.Model) or model.q8:
            raise ValueError("a rollout needs a Model with its weights as they are, not a view or 8-bit codes")
        self.session, self.model, self.cfg, self.n_seq, self.max_new = session, model, cfg, n_seq, max_new
        shape = (cfg.n_layer, n_seq, cfg.n_head, max_new, cfg.head_dim)
        self.k = torch.empty(shape, dtype=session.k_cache.dtype, device=model.device)
        self.v = torch.empty(shape, dtype=session.k_cache.dtype, device=model.device)

    def logits(self, prefix_len: int, tokens, step: int):
        """float32 logits [n_seq][vocab] after each sequence's token number
        `step` (int32 [n_seq]), whose keys and values join the sequence's."""
        cfg, w, b = self.cfg, self.model.tensors, self.n_seq
        if prefix_len + step >= cfg.n_pos or not 0 <= step < self.max_new:
            raise ValueError(f"position {prefix_len + step}, token {step}: outside the model's or the rollout's rows")
        if not 0 <= prefix_len <= self.session.max_ctx:
            raise ValueError(f"a prefix of {prefix_len} rows in a cache of {self.session.max_ctx}")
        own_len = torch.full((b,), step + 1, dtype=torch.int32, device=self.model.device)
        x = ops.embed(tokens, w["wte"], dtype=torch.float32) + w["wpe"][prefix_len + step].float()
        norm = lambda g, bias: F.layer_norm(x, (cfg.d_model,), g.float(), bias.float(), cfg.ln_eps)  # noqa: E731
        dense = lambda a, name, l: F.linear(a.to(w[name][l].dtype), w[name][l], w["b" + name[1:]][l])  # noqa: E731
        for l in range(cfg.n_layer):
            qkv = dense(norm(w["ln1_g"][l], w["ln1_b"][l]), "w_qkv", l).view(b, 3, cfg.n_head, cfg.head_dim)
            self.k[l, :, :, step], self.v[l, :, :, step] = qkv[:, 1], qkv[:, 2]
            att = ops.prefix_attention(qkv[:, :1], self.session.k_cache[l][:, :prefix_len],
                                       self.session.v_cache[l][:, :prefix_len], self.k[l], self.v[l], own_len)
            x = x + dense(att.view(b, cfg.d_model), "w_o", l).float()
            up = F.gelu(dense(norm(w["ln2_g"][l], w["ln2_b"][l]), "w_fc", l).float(), approximate="tanh")
            x = x + dense(up, "w_pr", l).float()
        return (norm(w["lnf_g"], w["lnf_b"]).to(w["wte"].dtype) @ w["wte"].t()).float()

    def sample(self, prefix_len: int, root: int, n_new: int, k: int, temperature: float = 1.0, generator=None
               ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(tokens int32 [n_new * n_seq], ids int32 [..][k], vals float32 [..][k]):
        the tokens that were fed, all from `root` on, and the oracle's top k
        logits after each; the next token is drawn from these."""
        tokens = torch.full((self.n_seq,), root, dtype=torch.int32, device=self.model.device)
        fed, ids, vals = [], [], []
        rows = self.session.max_nodes
        for step in range(n_new):
            logits = self.logits(prefix_len, tokens, step)
            top = [self.session.topk(logits[i:i + rows], k) for i in range(0, self.n_seq, rows)]
            idx, val = torch.cat([t[0] for t in top]), torch.cat([t[1] for t in top])
            fed.append(tokens)
            ids.append(idx)
            vals.append(val)
            pick = torch.multinomial(torch.softmax(val / temperature, 1), 1, generator=generator)
            tokens = idx.gather(1, pick)[:, 0]
        return torch.cat(fed), torch.cat(ids), torch.cat(vals)


class BigramStudent:
    """logits after a token: (scale table[token] mix) table^T."""

    def __init__(self, vocab: int, d: int, device="cuda", seed: int = 0, lr: float = 1e-2):
        gen = torch.Generator(device).manual_seed(seed)
        self.vocab, self.scale = vocab, math.sqrt(d)
        self.table = torch.randn((vocab, d), generator=gen, device=device) * (0.5 / math.sqrt(d))
        self.mix = torch.randn((d, d), generator=gen, device=device) / math.sqrt(d)
        self.optim = torch.optim.Adam([self.table, self.mix], lr=lr)

    def forward(self, tokens):
        """(embedding rows, hidden rows, float32 logits)."""
        e = ops.embed(tokens, self.table, scale=self.scale)
        h = e @ self.mix
        return e, h, h @ self.table.t()

    def loss(self, tokens, ids, vals, temperature: float = 1.0) -> float:
        """The mean divergence from the oracle's top logits."""
        return ops.distill_forward(self.forward(tokens)[2], ids, vals, temperature=temperature)[0].mean().item()

    def gradients(self, tokens, ids, vals, weight=None, temperature: float = 1.0):
        """(losses [N], the table's gradient, mix's gradient) of sum weight * divergence."""
        e, h, logits = self.forward(tokens)
        loss, _, g = ops.distill_step(logits, ids, vals, weight, temperature, out=logits)
        dh = g @ self.table
        dtable = g.t() @ h                       # as the output's table ...
        ops.embed_grad(tokens, dh @ self.mix.t(), self.vocab, scale=self.scale, out=dtable, accumulate=True)  # ... the input's
        return loss, dtable, e.t() @ dh

    def fit(self, tokens, ids, vals, temperature: float = 1.0):
        """One step on a batch; the losses before it."""
        n = tokens.shape[0]
        weight = torch.full((n,), 1.0 / n, device=tokens.device)
        loss, self.table.grad, self.mix.grad = self.gradients(tokens, ids, vals, weight, temperature)
        self.optim.step()
        return loss

    def successors(self, session, k: int = BIGRAM_TOP) -> np.ndarray:
        """The k likeliest tokens after every token, as staged.bigram_table gives them."""
        out = []
        for s in range(0, self.vocab, session.max_nodes):
            tokens = torch.arange(s, min(self.vocab, s + session.max_nodes), dtype=torch.int32,
                                  device=self.table.device)
            out.append(session.topk(self.forward(tokens)[2], k)[0])
        return torch.cat(out).cpu().numpy()


def main(n_seq: int = 16, n_new: int = 24, k: int = BIGRAM_TOP, steps: int = 60):
    from . import staged, workloads
    cfg = workloads.TINY
    model = ssd.Model(cfg, workloads.make_weights(cfg, 0))
    session = ssd.Session(model, 128, 64)
    prompt = workloads.prefix_tokens(65, cfg.vocab)
    prefix_len = staged.GpuBackend(session, session).prefill(prompt[:-1])
    gen = torch.Generator(model.device).manual_seed(1)
    rollout = Rollout(session, n_seq, n_new)
    batch = rollout.sample(prefix_len, int(prompt[-1]), n_new, k, generator=gen)
    held_out = rollout.sample(prefix_len, int(prompt[-1]), n_new, k, generator=gen)
    student = BigramStudent(cfg.vocab, cfg.d_model, model.device)
    before = student.loss(*batch), student.loss(*held_out)
    seen = [batch]
    for _ in range(steps):  # on all continuations so far, new ones with every step
        student.fit(*(torch.cat(x) for x in zip(*seen)))
        seen.append(rollout.sample(prefix_len, int(prompt[-1]), n_new, k, generator=gen))
    after = student.loss(*batch), student.loss(*held_out)
    print(f"{n_seq} continuations of {n_new} tokens over a prompt of {prefix_len}; divergence from the oracle's top {k}: "
          f"{before[0]:.3f} -> {after[0]:.3f} (other continuations {before[1]:.3f} -> {after[1]:.3f}), "
          f"successors {student.successors(session).shape}")
    return before, after


if __name__ == "__main__":
    main()
