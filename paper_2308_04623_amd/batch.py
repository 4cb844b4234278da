"""Tree verification for a batch of sequences over one paged cache in 8 bits.

A Session verifies one sequence's tree over its own dense cache.  Batch does so for many, each
somewhere else: prompts come from a session's cache, samples of one prompt share its
pages (fork), every step scores a tree (Sec. 3.1) of each sequence, and the accepted paths join
the cache (paged.py).  The layers' dense products around the operators are PyTorch's, as in
distill.Rollout.  Run as a program for a small one from end to end:

    python -m paper_2308_04623_amd.batch
"""
from __future__ import annotations

from typing import Sequence

import numpy as np
import torch
import torch.nn.functional as F

from . import ops, paged, ssd


class Batch:
    """n_seq slots for sequences of up to max_ctx rows (rounded down to pages, and an open page), whose steps have
    max_nodes new rows.  n_page: pages of the pool (default: enough for all slots without sharing).  window > 0: only
    so many rows back, and the first `sinks`, are looked at, and pages behind them are given back."""

    def __init__(self, model, n_seq: int, max_ctx: int, max_nodes: int, n_page: int = 0, page_rows: int = 32,
                 code: str = "int8", window: int = 0, sinks: int = 0):
        cfg = model.cfg
        if not isinstance(model, ssd.Model) or model.q8:
            raise ValueError("a batch needs a Model with its weights as they are, not a view or 8-bit codes")
        if n_seq < 1 or not 1 <= max_nodes <= 64 or max_ctx < 0 or page_rows not in (32, 64, 128):
            raise ValueError(f"{n_seq} sequences, {max_nodes} nodes (1 to 64), {max_ctx} rows in pages of {page_rows} (32, 64 or "
                             "128)")
        if window < 0 or sinks < 0 or 0 < window < max_nodes:
            raise ValueError(f"a window of {window} rows and {sinks} sinks for {max_nodes} nodes")
        n_col = max_ctx // page_rows
        if (n_col + 1) * page_rows + max_nodes > cfg.n_pos + 1:
            raise ValueError(f"{max_ctx} rows, an open page of {page_rows} and {max_nodes} nodes: more than the model's "
                             f"{cfg.n_pos} positions")
        self.model, self.cfg, self.n_seq, self.max_nodes, self.page_rows = model, cfg, n_seq, max_nodes, page_rows
        self.window, self.sinks = window, sinks
        dev, dt = model.device, ssd.storage_torch_dtype(cfg)
        self.pages = paged.Pages.empty(cfg.n_layer, n_page or max(1, n_seq * n_col), cfg.n_head, cfg.head_dim, page_rows,
                                       code, dev)
        self.table = torch.full((n_seq, n_col), -1, dtype=torch.int32, device=dev)
        self.length = torch.full((n_seq,), -1, dtype=torch.int32, device=dev)
        self.refs = torch.zeros(self.pages.n_page, dtype=torch.int32, device=dev)
        self.ring = page_rows + max_nodes - 1
        self.k_tail, self.v_tail = (torch.zeros((cfg.n_layer, n_seq, cfg.n_head, self.ring, cfg.head_dim), dtype=dt,
                                                device=dev) for _ in "kv")
        self.k_new, self.v_new = (torch.zeros((cfg.n_layer, n_seq, max_nodes, cfg.n_head, cfg.head_dim), dtype=dt,
                                              device=dev) for _ in "kv")

    def admit(self, slot: int, session, prefix_len: int):
        """The first prefix_len rows of a session's cache become the sequence of a slot without one."""
        if not 0 <= slot < self.n_seq or not 0 <= prefix_len <= session.max_ctx:
            raise ValueError(f"slot {slot}, {prefix_len} rows: outside the batch or the session's cache")
        like, cache = self.k_tail, session.k_cache
        if (cache.dtype, cache.device, cache.shape[0], cache.shape[1], cache.shape[3]) != \
                (like.dtype, like.device, like.shape[0], like.shape[2], like.shape[4]):
            raise ValueError("the session's cache is not of the batch's model's shape")
        if int(self.length[slot]) >= 0:
            raise ValueError(f"slot {slot} holds a sequence")
        rows, full = self.page_rows, prefix_len // self.page_rows
        count = torch.full((self.n_seq,), -1, dtype=torch.int32, device=self.model.device)
        count[slot] = full
        if int(paged.pages_take(self.pages, self.refs, self.table, self.length, count)[slot]) < 0:
            raise RuntimeError(f"{full} pages for {prefix_len} rows are not to be had")
        whole = [x[:, :, :full * rows].unflatten(2, (full, rows)).transpose(1, 2) if full else None
                 for x in (session.k_cache, session.v_cache)]
        if full:
            paged.pages_store(self.pages, self.table[slot, :full], *whole)
        at = torch.arange(full * rows, prefix_len, device=self.model.device)
        for tail, cache in ((self.k_tail, session.k_cache), (self.v_tail, session.v_cache)):
            tail[:, slot, :, at % self.ring] = cache[:, :, at]
        self.length[slot] = prefix_len

    def fork(self, parents: Sequence[int]):
        """Slot b becomes a copy of slot parents[b], which keeps itself; -1: it is freed."""
        p = torch.tensor(parents, dtype=torch.int32, device=self.model.device)
        paged.pages_fork(self.refs, self.table, self.length, p, self.k_tail, self.v_tail, self.page_rows)

    def masks(self, parents) -> torch.Tensor:
        """int64 [n_seq][max_nodes] of trees parents [n_seq][max_nodes]: -1 a root, below -1 no node (and no node's parent)."""
        anc = np.zeros(parents.shape, np.uint64)
        for b, row in enumerate(parents):
            for i, p in enumerate(row):
                if p >= i or p >= 0 and row[p] < -1:
                    raise ValueError(f"node {i} of sequence {b} has parent {p}")
                if p >= -1:
                    anc[b, i] = (anc[b, p] if p >= 0 else np.uint64(0)) | np.uint64(1 << i)
        return torch.from_numpy(anc.view(np.int64)).to(self.model.device)

    def verify(self, tokens, parents):
        """float32 logits [n_seq][max_nodes][vocab] of every sequence's tree: tokens int32 [n_seq][max_nodes]
        on the device, parents on the host (see masks).  Their keys and values wait for commit."""
        cfg, w, b, t = self.cfg, self.model.tensors, self.n_seq, self.max_nodes
        parents = np.asarray(parents)
        if tuple(tokens.shape) != (b, t) or parents.shape != (b, t):
            raise ValueError(f"tokens and parents must be [{b}][{t}]")
        anc = self.masks(parents)
        depth = torch.from_numpy(_depths(parents)).to(anc.device)
        pos = self.length.clamp(min=0).long().view(b, 1) + depth
        x = ops.embed(tokens.reshape(-1), w["wte"], dtype=torch.float32).view(b, t, -1) + w["wpe"][pos].float()
        norm = lambda g, bias: F.layer_norm(x, (cfg.d_model,), g.float(), bias.float(), cfg.ln_eps)  # noqa: E731
        dense = lambda a, name, l: F.linear(a.to(w[name][l].dtype), w[name][l], w["b" + name[1:]][l])  # noqa: E731
        for l in range(cfg.n_layer):
            qkv = dense(norm(w["ln1_g"][l], w["ln1_b"][l]), "w_qkv", l).view(b, t, 3, cfg.n_head, cfg.head_dim)
            self.k_new[l], self.v_new[l] = qkv[:, :, 1], qkv[:, :, 2]
            att = paged.paged_attention(qkv[:, :, 0], self.pages, self.table, self.length, self.k_tail[l], self.v_tail[l],
                                        qkv[:, :, 1], qkv[:, :, 2], layer=l, anc=anc, window=self.window, sinks=self.sinks)
            x = x + dense(att.view(b, t, cfg.d_model), "w_o", l).float()
            up = F.gelu(dense(norm(w["ln2_g"][l], w["ln2_b"][l]), "w_fc", l).float(), approximate="tanh")
            x = x + dense(up, "w_pr", l).float()
        return (norm(w["lnf_g"], w["lnf_b"]).to(w["wte"].dtype) @ w["wte"].t()).float()

    def accept(self, tokens, parents, logits):
        """Greedy walk (Sec. 2.3): (path int32 [n_seq][max_nodes], path_len int32 [n_seq], next token int32
        [n_seq]): the deepest node (lowest index on ties) all of whose ancestors' predictions are the tree's tokens."""
        parents = np.asarray(parents)
        best, toks = logits.argmax(2).cpu().numpy(), tokens.cpu().numpy()
        path, length, after = np.zeros(parents.shape, np.int32), np.zeros(self.n_seq, np.int32), np.zeros(self.n_seq, np.int32)
        for b, row in enumerate(parents):
            kept, deep = {}, -1
            for i, p in enumerate(row):
                if p == -1 and i == 0 or p >= 0 and p in kept and toks[b, i] == best[b, p]:
                    kept[i] = kept.get(p, 0) + 1
                    if deep < 0 or kept[i] > kept[deep]:
                        deep = i
            if deep < 0:
                continue
            after[b], nodes = best[b, deep], []
            while deep >= 0:
                nodes.append(deep)
                deep = row[deep]
            length[b] = len(nodes)
            path[b, :len(nodes)] = nodes[::-1]
        return [torch.from_numpy(x).to(self.model.device) for x in (path, length, after)]

    def commit(self, path, path_len):
        """The paths' rows join the sequences; int32 [n_seq]: pages that got full, -1 where there were none to be had (and
        nothing changed)."""
        return paged.pages_commit(self.pages, self.refs, self.table, self.length, self.k_tail, self.v_tail, self.k_new,
                                  self.v_new, path, path_len, window=self.window, sinks=self.sinks)

    def compact(self) -> int:
        """Moves the pages in use to the front of the pool; their number."""
        return int(paged.pages_compact(self.pages, self.refs, self.table))


def _depths(parents) -> np.ndarray:
    out = np.zeros(parents.shape, np.int64)
    for i in range(parents.shape[1]):
        p = parents[:, i]
        out[:, i] = np.where(p >= 0, out[np.arange(len(p)), np.maximum(p, 0)] + 1, 0)
    return out


def staged_greedy(batch: Batch, roots: Sequence[int], n_steps: int, succ):
    """n_steps of greedy decoding of every sequence in the batch with bigram trees (staged.bigram_tree over the
    successors `succ`): lists of the tokens that each emitted, its root first."""
    from .staged import bigram_tree
    out = [[int(r)] for r in roots]
    live = (batch.length >= 0).cpu().numpy()
    for _ in range(n_steps):
        tokens = np.full((batch.n_seq, batch.max_nodes), -1, np.int32)
        parents = np.full((batch.n_seq, batch.max_nodes), -2, np.int32)
        for b in np.flatnonzero(live):
            t, p = bigram_tree(out[b][-1], succ, cap=batch.max_nodes)
            tokens[b, :len(t)], parents[b, :len(p)] = t, p
        dev = torch.from_numpy(tokens).to(batch.model.device)
        path, length, after = batch.accept(dev, parents, batch.verify(dev, parents))
        full = batch.commit(path, length).cpu().numpy()
        path, length, after = path.cpu().numpy(), length.cpu().numpy(), after.cpu().numpy()
        for b in np.flatnonzero(live):
            if full[b] < 0:  # (no page: the sequence ends here)
                live[b] = False
                continue
            out[b] += [int(tokens[b, i]) for i in path[b, 1:length[b]]] + [int(after[b])]
    return out


def main(n_seq: int = 8, n_steps: int = 12):
    from . import staged, workloads
    cfg = workloads.TINY
    model = ssd.Model(cfg, workloads.make_weights(cfg, 0))
    session = ssd.Session(model, 128, 64)
    backend = staged.GpuBackend(session, session)
    succ = staged.build_bigram_gpu(backend, cfg.vocab, n_tokens=1 << 12, window=64)
    batch = Batch(model, n_seq, 160, 16)
    roots = []
    for slot in range(0, n_seq, 2):  # prompts of several lengths, two samples of each
        prompt = workloads.prefix_tokens(40 + 9 * slot, cfg.vocab, seed=slot)
        batch.admit(slot, session, backend.prefill(prompt[:-1]))
        roots += [int(prompt[-1]), (int(prompt[-1]) + 1) % cfg.vocab]
    batch.fork([s // 2 * 2 for s in range(n_seq)])
    shared = int((batch.refs > 1).sum())
    out = staged_greedy(batch, roots, n_steps, succ)
    used = batch.compact()
    per_step = sum(len(o) - 1 for o in out) / (n_seq * n_steps)
    print(f"{n_seq} sequences, {n_steps} steps: {per_step:.2f} tokens a sequence and step; {shared} pages shared at the start, "
          f"{used} of {batch.pages.n_page} in use; lengths {batch.length.tolist()}")
    return out, batch


if __name__ == "__main__":
    main()
