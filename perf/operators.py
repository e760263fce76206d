"""Serving a batch from bounded K,V caches: the attention of new tokens over them, the attention of requests that share a
long prefix, and the eviction of tokens by accumulated attention weight, each through its public entry point.

listed() names the cases, draw() gives further ones of the same ranges; prepare() makes what a serving program holds
in front of one layer of one step (the caches, the step's q, k, v, the workspace), run() is that layer's call.

The head layouts are those of the shapes in paper_2407_14057_amd.synth: "tiny" 4 heads of 64, "7b" 32 heads of 128,
"gqa8b" 32 query heads of 128 on 8 K,V heads.  Caches are [batch, capacity, K,V heads, head_dim] in bf16.  Lengths
differ from request to request, spread evenly over their logarithm between a case's `low` and `high`; `spread` seeds them.
"""
import math
import random

import numpy as np
import torch

own = False

HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "gqa8b": (32, 8, 128)}      # query heads, K,V heads, head_dim


def listed():
    return [
        # one request of the small model after a short question: launches and nothing else
        {"name": "step_tiny", "op": "attention", "heads": "tiny", "batch": 1, "low": 97, "high": 97, "spread": 0, "new": 1},
        # chat turns of a grouped-query model, one token each
        {"name": "step_chat", "op": "attention", "heads": "gqa8b", "batch": 32, "low": 150, "high": 2100, "spread": 1, "new": 1},
        # the packed batch of eight prompts of 1 k to 8 k tokens goes on: plain multi-head attention: 16 KB of K,V a token
        {"name": "step_7b_batch8", "op": "attention", "heads": "7b", "batch": 8, "low": 1024, "high": 8192, "spread": 2, "new": 1},
        # a token and four drafted ones of each request, to be verified together
        {"name": "draft_gqa8b", "op": "attention", "heads": "gqa8b", "batch": 16, "low": 700, "high": 7900, "spread": 3, "new": 5},
        # one very long document
        {"name": "step_long", "op": "attention", "heads": "gqa8b", "batch": 1, "low": 131071, "high": 131071, "spread": 4, "new": 1},
        # a few short requests behind a common instruction, small model
        {"name": "prefix_tiny", "op": "prefix", "heads": "tiny", "batch": 3, "low": 1, "high": 30, "spread": 5, "new": 1, "prefix": 512},
        # chats behind one system prompt of the benchmark's prompt length
        {"name": "prefix_chat", "op": "prefix", "heads": "gqa8b", "batch": 32, "low": 20, "high": 300, "spread": 6, "new": 1, "prefix": 3376},
        # questions about one document, plain multi-head attention: the prefix is read for 16 rows of a head
        {"name": "prefix_7b", "op": "prefix", "heads": "7b", "batch": 16, "low": 50, "high": 500, "spread": 7, "new": 1, "prefix": 8192},
        # many samples of one long prompt, four tokens each: 2048 query rows of a K,V head, bound by the matrix cores
        {"name": "prefix_many", "op": "prefix", "heads": "gqa8b", "batch": 128, "low": 10, "high": 200, "spread": 8, "new": 4, "prefix": 32768},
        # one token too many in a small cache
        {"name": "evict_tiny", "op": "evict", "heads": "tiny", "batch": 1, "low": 257, "high": 257, "spread": 9, "budget": 256},
        # every generated token makes one of each cache leave: the steady state of a bounded cache
        {"name": "evict_step", "op": "evict", "heads": "gqa8b", "batch": 32, "low": 2049, "high": 2049, "spread": 10, "budget": 2048},
        # eight prompts are brought down to the budget after their prefill, plain multi-head attention
        {"name": "evict_prompts", "op": "evict", "heads": "7b", "batch": 8, "low": 1024, "high": 8192, "spread": 11, "budget": 1100},
    ]


def draw(rng):
    """One more case: one to 64 requests of one token to 128 k tokens, 128 k in all (32 k with plain multi-head attention of 32 heads)."""
    op = rng.choice(["attention", "attention", "prefix", "evict"])
    heads = rng.choice(["tiny", "7b", "gqa8b", "gqa8b"])
    room = {"tiny": 131072, "7b": 32768, "gqa8b": 131072}[heads]             # batch x longest request, as in the listed cases

    def log(low, high):
        return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))

    case = {"op": op, "heads": heads, "batch": log(1, 64)}
    case["high"] = log(16, max(16, room // case["batch"]))
    case["low"] = log(1, case["high"])
    case["spread"] = rng.randrange(1 << 20)
    if op == "evict":
        case["budget"] = log(max(8, case["high"] // 8), case["high"] + 1)
        return case
    case["new"] = rng.choice([1, 1, 1, 2, 3, 5, 8])
    if op == "prefix":
        case["high"], case["low"] = min(case["high"], 700), min(case["low"], 700)
        case["prefix"] = log(100, 16384 if heads == "7b" else 32768)
    return case


def _lengths(case):
    r, low, high = random.Random(case["spread"]), math.log(case["low"]), math.log(case["high"])
    return [max(case["low"], min(case["high"], int(round(math.exp(r.uniform(low, high)))))) for _ in range(case["batch"])]


def prepare(case, seed):
    H, kvh, hd = HEADS[case["heads"]]
    n, batch = _lengths(case), case["batch"]
    new = case.get("new", 0)
    capacity = (max(n) + new + 15) // 16 * 16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        return x.normal_(0.0, scale, generator=g)

    lengths = torch.tensor(n, dtype=torch.int32, device="cuda")
    # Eq. 1-like weights of what is cached: a few tokens carry most of them, some share a value, some have none
    w = torch.empty(batch, capacity, device="cuda").normal_(0.0, 1.5, generator=g).exp_()
    w = (w / lengths[:, None]).to(torch.bfloat16).float()
    w *= torch.rand(batch, capacity, generator=g, device="cuda") > 0.05
    # original positions with gaps, as a pruned prefill leaves them
    pos = torch.randint(1, 4, (batch, capacity), generator=g, device="cuda").cumsum(1).to(torch.int32) - 1
    s = {"op": case["op"], "H": H, "kvh": kvh, "hd": hd, "n": n, "max": max(n), "lengths": lengths, "weight": w, "pos": pos,
         "weight_out": torch.zeros_like(w), "k": normal(batch, capacity, kvh, hd), "v": normal(batch, capacity, kvh, hd)}
    if case["op"] == "evict":
        s.update(budget=case["budget"], sinks=min(4, case["budget"] // 4), recent=min(64, case["budget"] // 4),
                 pos_out=torch.zeros_like(pos), lengths_out=torch.zeros_like(lengths))
        return _with_buffers(s)
    s.update(q=normal(batch, new, H, hd, scale=1.5), k_new=normal(batch, new, kvh, hd), v_new=normal(batch, new, kvh, hd),
             new=new, o=torch.empty(batch, new, H, hd, dtype=torch.bfloat16, device="cuda"))
    if case["op"] == "prefix":
        s.update(prefix_k=normal(case["prefix"], kvh, hd), prefix_v=normal(case["prefix"], kvh, hd))
    return _with_buffers(s)


def _with_buffers(s):
    """The handle of the caches and the workspace, which a program makes once; a tree without the operators has neither."""
    if not own:
        return s
    from paper_2407_14057_amd import binding as B
    s["cache"] = B.make_kv_cache(s["k"], s["v"])
    if s["op"] == "evict":
        size = B.lazyllm_op_cache_evict_workspace_bytes(s["cache"], s["budget"])
    else:
        size = B.lazyllm_op_cache_attention_workspace_bytes(s["cache"], s["H"], s["new"], s["max"],
                                                            s["prefix_k"].shape[0] if s["op"] == "prefix" else 0, s["op"] == "attention")
    s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


def run(s):
    if s["op"] == "attention":
        _own_attention(s) if own else _attention(s, None, None)
        return {"o": s["o"], "weight": s["weight_out"], "k": s["k"], "v": s["v"]}
    if s["op"] == "prefix":
        _own_prefix(s) if own else _attention(s, s["prefix_k"], s["prefix_v"])
        return {"o": s["o"], "k": s["k"], "v": s["v"]}
    _own_evict(s) if own else _evict(s)
    return {"k": s["k"], "v": s["v"], "weight": s["weight_out"], "pos": s["pos_out"], "lengths": s["lengths_out"]}


def _own_attention(s):
    from paper_2407_14057_amd import binding as B
    B.lazyllm_op_cache_attention(s["cache"], s["q"], s["k_new"], s["v_new"], s["lengths"], s["H"], s["new"], s["max"], s["o"], s["ws"],
                                 weight=s["weight"], weight_out=s["weight_out"])


def _own_prefix(s):
    from paper_2407_14057_amd import binding as B
    B.lazyllm_op_prefix_attention(s["cache"], s["prefix_k"], s["prefix_v"], s["q"], s["k_new"], s["v_new"], s["lengths"], s["H"], s["new"],
                                  s["max"], s["o"], s["ws"])


def _own_evict(s):
    from paper_2407_14057_amd import binding as B
    B.lazyllm_op_cache_evict(s["cache"], s["weight"], s["pos"], s["lengths"], s["budget"], s["sinks"], s["recent"], s["weight_out"],
                             s["pos_out"], s["lengths_out"], s["ws"])


def _attention(s, prefix_k, prefix_v):
    """The plain form: the new rows go into the caches, then one softmax per query row over prefix and cache."""
    batch, new, H, hd = s["q"].shape
    kvh, group, lengths = s["kvh"], H // s["kvh"], s["lengths"].long()
    slots = lengths[:, None] + torch.arange(new, device="cuda")
    rows = torch.arange(batch, device="cuda")[:, None].expand_as(slots)
    s["k"][rows, slots] = s["k_new"]
    s["v"][rows, slots] = s["v_new"]
    top = s["max"] + new
    # query rows of a K,V head: (token, query head of the group)
    q = s["q"].float().view(batch, new, kvh, group, hd).permute(0, 2, 1, 3, 4).reshape(batch, kvh, new * group, hd) / math.sqrt(hd)
    k = s["k"][:, :top].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"][:, :top].float().permute(0, 2, 1, 3).contiguous()
    key = torch.arange(top, device="cuda")
    last = slots.repeat_interleave(group, dim=1)                              # the last slot that a query row sees
    z = torch.matmul(q, k).masked_fill_((key > last[:, :, None])[:, None], -math.inf)
    high = z.amax(-1, keepdim=True)
    if prefix_k is None:
        p = (z - high).exp_()
        p /= p.sum(-1, keepdim=True)
        o = torch.matmul(p, v)
        mean = p.sum((1, 2)) / H
        before = torch.where(key < lengths[:, None], s["weight"][:, :top], 0.0)
        s["weight_out"][:, :top] = torch.where(key < lengths[:, None] + new, before + mean, s["weight_out"][:, :top])
    else:
        qs = q.transpose(0, 1).reshape(kvh, batch * new * group, hd)
        zp = torch.matmul(qs, prefix_k.float().permute(1, 2, 0).contiguous())
        high = torch.maximum(high, zp.amax(-1).view(kvh, batch, -1).transpose(0, 1)[..., None])
        p = (z - high).exp_()
        pp = zp.sub_(high.transpose(0, 1).reshape(kvh, -1, 1)).exp_()
        total = p.sum(-1) + pp.sum(-1).view(kvh, batch, -1).transpose(0, 1)
        op = torch.matmul(pp, prefix_v.float().transpose(0, 1).contiguous()).view(kvh, batch, -1, hd).transpose(0, 1)
        o = (torch.matmul(p, v) + op) / total[..., None]
    s["o"].copy_(o.view(batch, kvh, new, group, hd).permute(0, 2, 1, 3, 4).reshape(batch, new, H, hd))


def _evict(s):
    """The plain form: two stable sorts (by weight, then protected tokens first and empty slots last) and gathers."""
    batch, capacity = s["weight"].shape
    budget, n = s["budget"], s["lengths"].long()[:, None]
    slot = torch.arange(capacity, device="cuda").expand(batch, capacity)
    valid, pos = slot < n, s["pos"].long()
    end = torch.where(valid, pos, -1).amax(1, keepdim=True) + 1
    safe = valid & ((pos < s["sinks"]) | (pos >= end - s["recent"]))
    by_weight = s["weight"].sort(dim=1, descending=True, stable=True).indices
    rank = (valid.long() + safe.long()).gather(1, by_weight)
    order = by_weight.gather(1, rank.sort(dim=1, descending=True, stable=True).indices)
    kept = n.clamp(max=budget)
    keep = torch.zeros_like(valid).scatter_(1, order, slot < kept)
    hole, mover = ~keep & (slot < kept), keep & (slot >= kept)
    movers = mover.sort(dim=1, descending=True, stable=True).indices         # kept tokens behind the budget, in order
    source = torch.where(hole, movers.gather(1, (hole.long().cumsum(1) - 1).clamp(min=0)), slot)
    few = min(budget, capacity)
    source = source[:, :few]
    rows = source[:, :, None, None].expand(-1, -1, s["kvh"], s["hd"])
    s["k"][:, :few] = s["k"].gather(1, rows)
    s["v"][:, :few] = s["v"].gather(1, rows)
    there = slot[:, :few] < kept
    s["weight_out"][:, :few] = torch.where(there, s["weight"].gather(1, source), s["weight_out"][:, :few])
    s["pos_out"][:, :few] = torch.where(there, s["pos"].gather(1, source), s["pos_out"][:, :few])
    s["lengths_out"].copy_(kept[:, 0])


def work(case):
    H, kvh, hd = HEADS[case["heads"]]
    n, batch = _lengths(case), case["batch"]
    row = 2 * kvh * hd * 2                                                   # K and V of a token
    if case["op"] == "evict":
        # the tables are read and the kept part of them written; how many rows move depends on the weights: of the
        # slots below the budget as many lose their token as tokens behind it are kept
        tables = sum(8 * m + 8 * min(m, case["budget"]) for m in n)
        moved = sum(min(m, case["budget"]) * max(0, m - case["budget"]) / m for m in n)
        return {"bytes": tables + 2 * moved * row, "flops": sum(n)}
    new, prefix = case["new"], case.get("prefix", 0)
    seen = sum(new * (m + prefix) + new * (new + 1) // 2 for m in n)         # (query token, key) pairs
    keys = sum(n) + prefix
    moved = keys * row + 2 * batch * new * row + 2 * batch * new * H * hd * 2
    if case["op"] == "attention":
        moved += sum(4 * m + 4 * (m + new) for m in n)
    return {"bytes": moved, "flops": 4 * seen * H * hd}


def exact(case, seed):
    s = prepare(case, seed)
    n = s["n"]
    if case["op"] == "evict":
        return _exact_evict(s)
    new, group, hd = s["new"], s["H"] // s["kvh"], s["hd"]
    o = torch.empty(case["batch"], new, s["H"], hd, dtype=torch.float64, device="cuda")
    weight = s["weight_out"].double()
    prefix = case["op"] == "prefix"
    for h in range(s["kvh"]):
        heads = slice(h * group, (h + 1) * group)
        if prefix:
            pk, pv = s["prefix_k"][:, h].double(), s["prefix_v"][:, h].double()
            qh = s["q"][:, :, heads].double() / hd ** 0.5
            zp = qh.reshape(-1, hd) @ pk.T
            ep = zp.exp()                                                    # (logits of some ten at most: no maximum needed in 64 bits)
            front = (ep @ pv).view(case["batch"], new, group, hd)
            mass = ep.sum(1).view(case["batch"], new, group)
            del zp, ep
        for b in range(case["batch"]):
            k = torch.cat([s["k"][b, :n[b], h], s["k_new"][b, :, h]]).double()
            v = torch.cat([s["v"][b, :n[b], h], s["v_new"][b, :, h]]).double()
            z = torch.einsum("tgd,jd->tgj", s["q"][b, :, heads].double(), k) / hd ** 0.5
            hidden = torch.ones(new, new, device="cuda", dtype=torch.bool).triu(1)
            z[:, :, n[b]:].masked_fill_(hidden[:, None, :], -math.inf)
            e = z.exp()
            total = e.sum(2) + (mass[b] if prefix else 0.0)
            o[b, :, heads] = (torch.einsum("tgj,jd->tgd", e, v) + (front[b] if prefix else 0.0)) / total[..., None]
            if not prefix:
                add = (e / total[..., None]).sum((0, 1)) / s["H"]
                if h == 0:
                    weight[b, :n[b]] = s["weight"][b, :n[b]].double()
                    weight[b, n[b]:n[b] + new] = 0.0
                weight[b, :n[b] + new] += add
    for b in range(case["batch"]):
        s["k"][b, n[b]:n[b] + new] = s["k_new"][b]
        s["v"][b, n[b]:n[b] + new] = s["v_new"][b]
    return {"o": o, "weight": weight, "k": s["k"], "v": s["v"]} if not prefix else {"o": o, "k": s["k"], "v": s["v"]}


def _exact_evict(s):
    weight, pos = s["weight"].cpu().numpy(), s["pos"].cpu().numpy()
    for b, m in enumerate(s["n"]):
        kept = min(m, s["budget"])
        end = int(pos[b, :m].max()) + 1
        value = weight[b, :m].astype(np.float64)
        value[(pos[b, :m] < s["sinks"]) | (pos[b, :m] >= end - s["recent"])] = np.inf
        chosen = np.sort(np.lexsort((np.arange(m), -value))[:kept])
        source = np.arange(kept)
        source[np.setdiff1d(np.arange(kept), chosen)] = chosen[chosen >= kept]
        at = torch.from_numpy(source).to("cuda")
        for name in ("k", "v"):
            s[name][b, :kept] = s[name][b, at]
        for name in ("weight", "pos"):
            s[name + "_out"][b, :kept] = s[name][b, at]
        s["lengths_out"][b] = kept
    return {"k": s["k"], "v": s["v"], "weight": s["weight_out"], "pos": s["pos_out"], "lengths": s["lengths_out"]}
