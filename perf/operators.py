"""The operators of training a draft on the oracle's own continuations, as measurable cases.

A case is a dict of plain values; its "kind" says which operator it goes
through (paper_2308_04623_amd.ops):

  attn     attention of a batch of sequences that continue one prompt: the
           prompt's keys and values are shared, each sequence has its own
           beside them                                    ops.prefix_attention
  distill  divergence of a student's logits from a teacher's top logits:
           "forward" (loss), "backward" (gradient from the saved log-sum-exp)
           or "step" (both at once)      ops.distill_forward / _backward / _step
  embed    "lookup": scaled rows of a table; "grad": the table's gradient
                                                   ops.embed / ops.embed_grad

Sizes are those of the package's models (the toy: 4 heads of 32, vocabulary
512, width 128; GPT-2-Large: 20 heads of 64, vocabulary 50257, width 1280)
and, for grouped heads, generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

VOCAB = 50257


def listed():
    return [
        # the toy float32 model's heads: the smallest call, all launches and host work
        {"name": "attn_f32_b6_p64", "kind": "attn", "dtype": "f32", "b": 6, "t": 1, "h": 4, "hkv": 4, "d": 32, "p": 64,
         "r": 24},
        # one decoding step of 32 samples of a prompt that fills the benchmark's longest context
        {"name": "attn_b32_p2048", "kind": "attn", "dtype": "bf16", "b": 32, "t": 1, "h": 20, "hkv": 20, "d": 64,
         "p": 2048, "r": 256},
        # grouped heads, five speculated tokens per sequence: the products outweigh the bytes
        {"name": "attn_gqa_b48_t5_p8191", "kind": "attn", "dtype": "bf16", "b": 48, "t": 5, "h": 32, "hkv": 8,
         "d": 128, "p": 8191, "r": 512},
        # a document as the prompt: the shared rows are nearly all of the traffic
        {"name": "attn_b16_p100000", "kind": "attn", "dtype": "bf16", "b": 16, "t": 1, "h": 20, "hkv": 20, "d": 64,
         "p": 100000, "r": 333},
        # the toy's tree of 15 nodes: launches and host work
        {"name": "distill_step_n15_v512", "kind": "distill", "what": "step", "dtype": "f32", "n": 15, "v": 512, "k": 8,
         "temperature": 1.0},
        # the float32 logits of the benchmark's widest tree, with the top 8 that Session.topk gives
        {"name": "distill_step_n256", "kind": "distill", "what": "step", "dtype": "f32", "n": 256, "v": VOCAB, "k": 8,
         "temperature": 1.0},
        # a held-out set's loss, top 50 as in the sampling setting
        {"name": "distill_forward_n1000", "kind": "distill", "what": "forward", "dtype": "bf16", "n": 1000,
         "v": VOCAB, "k": 50, "temperature": 2.0},
        # the gradient alone, for a caller whose weights are known after the forward pass
        {"name": "distill_backward_n1500", "kind": "distill", "what": "backward", "dtype": "f32", "n": 1500,
         "v": VOCAB, "k": 16, "temperature": 1.0},
        # a training batch of 4096 tokens
        {"name": "distill_step_n4096", "kind": "distill", "what": "step", "dtype": "bf16", "n": 4096, "v": VOCAB,
         "k": 64, "temperature": 1.5},
        # a tree's nodes through the embedding: launches and host work
        {"name": "embed_lookup_n32", "kind": "embed", "what": "lookup", "table": "bf16", "out": "f32", "n": 32,
         "v": VOCAB, "d": 1280},
        # the toy's gradient
        {"name": "embed_grad_n200_v512", "kind": "embed", "what": "grad", "table": "f32", "out": "f32", "n": 200,
         "v": 512, "d": 128},
        # a training batch's gradient: a few tokens are very frequent, most of the vocabulary does not occur
        {"name": "embed_grad_n16384", "kind": "embed", "what": "grad", "table": "f32", "out": "bf16", "n": 16384,
         "v": VOCAB, "d": 1280},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "distill", "distill", "distill", "embed", "embed"])
    if kind == "attn":
        h, hkv, d = rng.choice([(4, 4, 32), (20, 20, 64), (20, 20, 64), (25, 25, 64), (16, 2, 64), (32, 8, 128)])
        t = rng.choice([1, 1, 1, 2, 3, 5, 8])
        b = _log_int(rng, 1, 64)
        dtype = rng.choice(["f32", "bf16"]) if d == 32 else rng.choice(["bf16", "bf16", "bf16", "f32"])
        # no more rows than leave the products and the traffic below the listed cases'
        most = min(100000, 60_000_000 // (b * t * h), 100_000_000 // (hkv * d * (2 if dtype == "f32" else 1)))
        return {"kind": "attn", "dtype": dtype, "b": b, "t": t, "h": h, "hkv": hkv, "d": d,
                "p": _log_int(rng, 1, most), "r": _log_int(rng, t, 512)}
    if kind == "distill":
        what, dtype = rng.choice(["step", "step", "forward", "backward"]), rng.choice(["f32", "bf16"])
        v = VOCAB if rng.random() < 0.5 else _log_int(rng, 400, 131072)
        n = _log_int(rng, 1, min(8192, (60_000_000 if dtype == "f32" else 120_000_000) // v))
        return {"kind": "distill", "what": what, "dtype": dtype, "n": n, "v": v, "k": _log_int(rng, 1, 128),
                "temperature": rng.choice([1.0, 1.0, 0.7, 2.0])}
    v = VOCAB if rng.random() < 0.5 else _log_int(rng, 400, 131072)
    d = rng.choice([128, 768, 1280, 1600, _log_int(rng, 32, 2048)])
    d = min(d, 60_000_000 // v)
    return {"kind": "embed", "what": rng.choice(["lookup", "grad", "grad"]), "table": rng.choice(["f32", "bf16"]),
            "out": rng.choice(["f32", "bf16"]), "n": _log_int(rng, 1, min(32768, 20_000_000 // d)), "v": v, "d": d}


DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
SCALE = 1.7  # of the embedding


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(s, generator=gen, device="cuda")  # noqa: E731
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    state = {"case": case}
    if case["kind"] == "attn":
        dt, b, t, h, hkv, d, p, r = (DTYPES[case["dtype"]],) + tuple(case[k] for k in ("b", "t", "h", "hkv", "d", "p", "r"))
        state["q"] = (2.0 * randn(b, t, h, d)).to(dt)
        for name, shape in (("k_prefix", (hkv, p, d)), ("v_prefix", (hkv, p, d)), ("k_own", (b, hkv, r, d)),
                            ("v_own", (b, hkv, r, d))):
            state[name] = (0.7 * randn(*shape)).to(dt)
        # every sequence is somewhere else in its answer
        own_len = (t + rand(b) * (r - t + 1)).to(torch.int32).clamp(max=r)
        if b > 4:  # one slot of the batch that holds no sequence
            own_len[b // 3] = -1
        state["own_len"] = own_len
    elif case["kind"] == "distill":
        dt, n, v, k = DTYPES[case["dtype"]], case["n"], case["v"], case["k"]
        k = min(k, v)
        logits = torch.empty((n, v), dtype=dt, device="cuda")
        ids = torch.empty((n, k), dtype=torch.int32, device="cuda")
        vals = torch.empty((n, k), dtype=torch.float32, device="cuda")
        for i in range(0, n, 512):
            m = min(512, n - i)
            x = 2.0 * randn(m, v)
            logits[i:i + m] = x.to(dt)
            top = (x + 0.8 * randn(m, v)).topk(k, 1)  # a teacher whom the student follows roughly
            vals[i:i + m], ids[i:i + m] = top.values, top.indices.to(torch.int32)
        weight = rand(n) + 0.5
        weight[torch.rand(n, generator=gen, device="cuda") < 0.05] = 0.0  # padding
        ids[rand(n, k) < 0.02] = -1  # slots that hold no token
        state.update(logits=logits, ids=ids, vals=vals, weight=weight)
        if case["what"] == "backward":  # as the forward pass leaves it
            state["lse"] = torch.cat([torch.logsumexp(logits[i:i + 512].float() / case["temperature"], 1)
                                      for i in range(0, n, 512)])
    else:
        n, v, d = case["n"], case["v"], case["d"]
        # frequencies fall with the inverse of the rank; ranks are spread over the vocabulary
        rank = torch.exp(rand(n) * math.log(v + 1.0)).long() - 1
        tokens = torch.randperm(v, generator=gen, device="cuda")[rank.clamp(0, v - 1)].to(torch.int32)
        tokens[rand(n) < 0.02] = -1  # padding
        state["tokens"] = tokens
        if case["what"] == "lookup":
            state["table"] = (0.02 * randn(v, d)).to(DTYPES[case["table"]])
        else:
            state["grad"] = (0.01 * randn(n, d)).to(DTYPES[case["out"]])
    return state


def run(state):
    case = state["case"]
    if case["kind"] == "attn":
        return _attn_own(state) if own else _attn_plain(state)
    if case["kind"] == "distill":
        return _distill_own(case, state) if own else _distill_plain(case, state)
    return _embed_own(case, state) if own else _embed_plain(case, state)


# ---------------------------------------------------------------- the package's operators

def _attn_own(s):
    from paper_2308_04623_amd import ops
    return ops.prefix_attention(s["q"], s["k_prefix"], s["v_prefix"], s["k_own"], s["v_own"], s["own_len"])


def _distill_own(case, s):
    from paper_2308_04623_amd import ops
    t = case["temperature"]
    if case["what"] == "forward":
        loss, lse = ops.distill_forward(s["logits"], s["ids"], s["vals"], s["weight"], temperature=t)
        return {"loss": loss, "lse": lse}
    if case["what"] == "backward":
        return {"grad": ops.distill_backward(s["logits"], s["ids"], s["vals"], s["lse"], s["weight"], temperature=t)}
    loss, lse, grad = ops.distill_step(s["logits"], s["ids"], s["vals"], s["weight"], temperature=t)
    return {"loss": loss, "lse": lse, "grad": grad}


def _embed_own(case, s):
    from paper_2308_04623_amd import ops
    if case["what"] == "lookup":
        return ops.embed(s["tokens"], s["table"], scale=SCALE, dtype=DTYPES[case["out"]])
    return ops.embed_grad(s["tokens"], s["grad"], case["v"], scale=SCALE, dtype=DTYPES[case["table"]])


# ---------------------------------------------------------------- plain forms

def _attn_plain(s):
    q, own_len = s["q"].float(), s["own_len"].long()
    kp, vp, ko, vo = (s[k].float() for k in ("k_prefix", "v_prefix", "k_own", "v_own"))
    b, t, h, d = q.shape
    hkv, p, r = kp.shape[0], kp.shape[1], ko.shape[2]
    g = h // hkv
    q = q.view(b, t, hkv, g, d).permute(2, 0, 1, 3, 4).contiguous()  # [hkv][b][t][g][d]
    sp = torch.bmm(q.view(hkv, b * t * g, d), kp.transpose(1, 2).contiguous()).view(hkv, b, t, g, p)
    so = torch.matmul(q.view(hkv, b, t * g, d).transpose(0, 1).contiguous(), ko.transpose(2, 3).contiguous())
    so = so.view(b, hkv, t, g, r).transpose(0, 1)
    # query i is row own_len - t + i of its sequence and sees the rows up to itself
    seen = own_len.view(b, 1) - t + 1 + torch.arange(t, device=q.device)
    so = so.masked_fill(~(torch.arange(r, device=q.device) < seen.view(1, b, t, 1, 1)), -math.inf)
    sp = sp.masked_fill((own_len < 0).view(1, b, 1, 1, 1), -math.inf)
    x = torch.cat([sp, so], 4) * (1.0 / math.sqrt(d))
    top = x.amax(4, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(4, keepdim=True)
    w = torch.where(total > 0, e / total, torch.zeros_like(e))
    o = torch.bmm(w[..., :p].reshape(hkv, b * t * g, p), vp).view(hkv, b, t, g, d)
    wo = w[..., p:].transpose(0, 1).reshape(b, hkv, t * g, r)
    # rows past a sequence's end may hold anything: they take no part
    vo = torch.where(torch.arange(r, device=q.device).view(1, 1, r, 1) < own_len.view(b, 1, 1, 1), vo, torch.zeros_like(vo))
    o = o + torch.matmul(wo, vo).view(b, hkv, t, g, d).transpose(0, 1)
    return o.permute(1, 2, 0, 3, 4).reshape(b, t, h, d).to(s["q"].dtype)


def _teacher(ids, vals, v, temperature):
    ok = (ids >= 0) & (ids < v) & (vals > -math.inf)
    x = torch.where(ok, vals / temperature, torch.full_like(vals, -math.inf))
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(ok.any(1, keepdim=True), top, torch.zeros_like(top)))
    total = e.sum(1, keepdim=True)
    return ok, torch.where(total > 0, e / total, torch.zeros_like(e))


def _distill_plain(case, s):
    z, ids, vals, weight = s["logits"].float(), s["ids"], s["vals"], s["weight"]
    temperature, v = case["temperature"], case["v"]
    ok, pr = _teacher(ids, vals, v, temperature)
    at = torch.where(ok, ids, torch.zeros_like(ids)).long()
    live = ok.any(1) & (weight != 0)
    z = z / temperature
    if case["what"] == "backward":
        lse = s["lse"]
    else:
        top = z.amax(1, keepdim=True)
        lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True))).squeeze(1)
    out = {}
    if case["what"] != "backward":
        terms = torch.where(pr > 0, pr * (torch.log(pr) - (z.gather(1, at) - lse.view(-1, 1))), torch.zeros_like(pr))
        out["loss"] = torch.where(live, weight * terms.sum(1), torch.zeros_like(weight))
        out["lse"] = lse
    if case["what"] != "forward":
        g = torch.exp(z - lse.view(-1, 1)).scatter_add_(1, at, -pr)
        g = g * (weight / temperature).view(-1, 1)
        out["grad"] = g.masked_fill_(~live.view(-1, 1), 0.0).to(s["logits"].dtype)
    return out


def _embed_plain(case, s):
    tokens, v = s["tokens"].long(), case["v"]
    ok = (tokens >= 0) & (tokens < v)
    if case["what"] == "lookup":
        x = s["table"].index_select(0, torch.where(ok, tokens, torch.zeros_like(tokens))).float() * SCALE
        return x.masked_fill_(~ok.view(-1, 1), 0.0).to(DTYPES[case["out"]])
    g = torch.zeros((v + 1, case["d"]), dtype=torch.float32, device=tokens.device)
    g.index_add_(0, torch.where(ok, tokens, torch.full_like(tokens, v)), s["grad"].float())
    return (g[:v] * SCALE).to(DTYPES[case["table"]])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "attn":
        b, t, h, hkv, d, p, r = (case[k] for k in ("b", "t", "h", "hkv", "d", "p", "r"))
        es, live = BYTES[case["dtype"]], b - (b > 4)
        rows = live * (t + r) / 2  # own rows of an average batch
        return {"bytes": es * (2 * live * t * h * d + 2 * hkv * d * (p + rows)) + 4 * b,
                "flops": 4.0 * d * h * t * (live * p + rows)}
    if case["kind"] == "distill":
        n, v, k, es = case["n"], case["v"], min(case["k"], case["v"]), BYTES[case["dtype"]]
        moved = n * v * es * (1 if case["what"] == "forward" else 2)
        # an exponential is one operation, as is each product or sum beside it
        return {"bytes": moved + n * (8 * k + 12), "flops": 4.0 * n * v}
    n, v, d = case["n"], case["v"], case["d"]
    if case["what"] == "lookup":
        return {"bytes": n * (4 + d * (BYTES[case["table"]] + BYTES[case["out"]])), "flops": 1.0 * n * d}
    return {"bytes": n * (4 + d * BYTES[case["out"]]) + v * d * BYTES[case["table"]], "flops": 1.0 * n * d}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _attn_exact, "distill": _distill_exact, "embed": _embed_exact}[case["kind"]](case, s)


def _attn_exact(case, s):
    b, t, h, d = s["q"].shape
    out = torch.zeros((b, t, h, d), dtype=torch.float64, device="cuda")
    group = h // case["hkv"]
    kp, vp = s["k_prefix"].double(), s["v_prefix"].double()
    for i, n in enumerate(s["own_len"].tolist()):
        if n < 0:
            continue
        for kv in range(case["hkv"]):
            k = torch.cat([kp[kv], s["k_own"][i, kv, :n].double()])
            v = torch.cat([vp[kv], s["v_own"][i, kv, :n].double()])
            heads = slice(kv * group, (kv + 1) * group)
            q = s["q"][i, :, heads].double()  # [t][group][d]
            scores = (q.reshape(t * group, d) @ k.T / math.sqrt(d)).view(t, group, -1)
            for j in range(t):
                keys = case["p"] + max(0, n - t + 1 + j)
                if keys:
                    out[i, j, heads] = torch.softmax(scores[j, :, :keys], 1) @ v[:keys]
    return out


def _distill_exact(case, s):
    n, v, temperature = case["n"], case["v"], case["temperature"]
    parts = []
    for i in range(0, n, 256):
        z = s["logits"][i:i + 256].double() / temperature
        ids, weight = s["ids"][i:i + 256].long(), s["weight"][i:i + 256].double()
        vals = s["vals"][i:i + 256].double().masked_fill((ids < 0) | (ids >= v), -math.inf)
        empty = ~torch.isfinite(vals).any(1)
        p = torch.softmax((vals / temperature).masked_fill(empty.view(-1, 1), 0.0), 1)
        lse = torch.logsumexp(z, 1) if "lse" not in s else s["lse"][i:i + 256].double()
        logq = z - lse.view(-1, 1)
        at = ids.clamp(0, v - 1)
        weight = weight.masked_fill(empty, 0.0)
        part = {}
        if case["what"] != "backward":
            part["loss"] = weight * (torch.special.xlogy(p, p) - p * logq.gather(1, at)).sum(1)
            part["lse"] = lse
        if case["what"] != "forward":
            p_full = torch.zeros_like(z).scatter_add_(1, at, p)
            part["grad"] = (weight / temperature).view(-1, 1) * (logq.exp() - p_full)
        parts.append(part)
    return {k: torch.cat([x[k] for x in parts]) for k in parts[0]}


def _embed_exact(case, s):
    tokens, v, d = s["tokens"].long(), case["v"], case["d"]
    if case["what"] == "lookup":
        out = torch.zeros((case["n"], d), dtype=torch.float64, device="cuda")
        held = (tokens >= 0) & (tokens < v)
        out[held] = s["table"].double()[tokens[held]] * SCALE
        return out
    # in the tokens' order, a strip of columns at a time
    held = torch.nonzero((tokens >= 0) & (tokens < v)).squeeze(1)
    out = torch.zeros((v, d), dtype=torch.float64, device="cuda")
    order = held[torch.argsort(tokens[held])]
    for c in range(0, d, 256):
        out[:, c:c + 256].index_add_(0, tokens[order], s["grad"][order, c:c + 256].double() * SCALE)
    return out
