"""Cases of the operators on caller-held caches: what a program that uses them has them do.

``scored``  attention of a stream's newest queries over its cache, which also adds up the weight that every
            cached row received: one query per head while decoding, many for a prompt or a chunk of one.
``evict``   the rows of every cache that received the most weight are kept, with the first and the newest
            positions; the others make room.
``prefix``  one decode step of a batch whose sequences share a (weighted) prefix and go on with their own rows.

Sizes are those of this repository's workloads (8 KV heads of 128 dims with 4 or 5 query heads each, contexts of
8192 to 32768 tokens, caches of 2048 to 32768 rows, batches of 8 to 32 sequences, the tiny fp32 stream with 64 dims) or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_SCORED = dict(op="scored", streams=8, rows=1024, ragged=False, queries=1, scored=1, group=4, head_dim=128, dtype="bf16", decay=1.0)
_EVICT = dict(op="evict", streams=8, rows=1025, ragged=False, keep=1024, first=4, recent=64, head_dim=128, dtype="bf16")
_PREFIX = dict(op="prefix", batch=8, kv_heads=8, group=4, prefix=2048, rows=128, ragged=True, weighted=False, head_dim=128, dtype="bf16")


def listed():
    return [
        # one sequence's token on a layer with a small budget: latency
        dict(_SCORED, name="scored decode small"),
        # a batch of 32 sequences whose caches have every length from nothing to full: memory
        dict(_SCORED, name="scored decode batch", streams=256, rows=8192, ragged=True, group=5),
        # fp32 heads of 64 dims, an odd number of rows, older weight fading
        dict(_SCORED, name="scored decode fp32", streams=24, rows=4501, group=3, head_dim=64, dtype="fp32", decay=0.97),
        # the last chunk of a long prompt; its last 64 queries choose what stays
        dict(_SCORED, name="scored chunk", rows=32768, queries=2048, scored=64),
        # a whole prompt, every query counts
        dict(_SCORED, name="scored prompt", rows=8192, queries=8192, scored=8192),
        # a few tokens at once in fp32, left-padded sequences
        dict(_SCORED, name="scored tokens fp32", streams=6, rows=1000, ragged=True, queries=33, scored=33, group=2, head_dim=64, dtype="fp32"),
        # one row too many per cache, every token
        dict(_EVICT, name="evict one row"),
        # a batch's prompts of mixed lengths cut to a budget
        dict(_EVICT, name="evict batch", streams=256, rows=4096, ragged=True, keep=1024),
        # long fp32 caches cut to a quarter
        dict(_EVICT, name="evict long fp32", streams=32, rows=32768, keep=8192, recent=128, head_dim=64, dtype="fp32"),
        # a few sequences behind a short system prompt, fp32
        dict(_PREFIX, name="prefix small fp32", batch=3, group=2, prefix=1000, rows=77, head_dim=64, dtype="fp32"),
        # a batch behind a compressed document
        dict(_PREFIX, name="prefix document", batch=32, prefix=32768, rows=512, weighted=True),
        # a large batch behind a shared prompt
        dict(_PREFIX, name="prefix large batch", batch=256, group=5, prefix=8192, rows=1024),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(["scored", "scored", "evict", "prefix"])
    d, dtype, esz = rng.choice([(128, "bf16", 2), (128, "bf16", 2), (64, "bf16", 2), (128, "fp32", 4), (64, "fp32", 4)])
    group, ragged = rng.randint(1, 8), rng.random() < 0.5
    common = dict(op=op, ragged=ragged, head_dim=d, dtype=dtype)
    if op == "scored" and rng.random() < 0.5:
        streams = _log(rng, 1, 256)
        rows = _log(rng, 16, max(16, min(32768, 2 ** 30 // (streams * 2 * d * esz))))
        return dict(common, streams=streams, rows=rows, queries=1, scored=1, group=group, decay=rng.choice([1.0, 0.9]))
    if op == "scored":
        streams, queries = _log(rng, 1, 32), _log(rng, 2, 2048)
        cost = 2 ** 31 if dtype == "bf16" else 2 ** 27           # score entries: an fp32 pass has no tensor cores to run on
        rows = _log(rng, min(queries, max(16, cost // (streams * group * queries))), max(16, min(32768, cost // (streams * group * queries))))
        return dict(common, streams=streams, rows=rows, queries=queries, scored=rng.choice([queries, queries, min(queries, 64), 1]), group=group,
                    decay=rng.choice([1.0, 0.9]))
    if op == "evict":
        streams = _log(rng, 1, 256)
        rows = _log(rng, 64, min(65536, 2 ** 30 // (streams * 2 * d * esz)))
        keep = _log(rng, max(1, rows // 32), rows)
        first = rng.randint(0, min(8, keep))
        return dict(common, streams=streams, rows=rows, keep=keep, first=first, recent=rng.randint(0, min(256, keep - first)))
    batch, heads = _log(rng, 1, 256 if dtype == "bf16" else 16), rng.randint(1, 8)
    prefix = _log(rng, 1, min(32768, 2 ** (29 if dtype == "bf16" else 26) // (batch * heads * group)))
    rows = _log(rng, 1, max(1, min(2048, 2 ** 29 // (batch * heads * 2 * d * esz))))
    return dict(common, batch=batch, kv_heads=heads, group=group, prefix=prefix, rows=rows, weighted=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- sizes

def _lengths(case):
    """Rows in use of every stream (every sequence of a prefix case): all of them, or all lengths from 0 to full in mixed order."""
    n, count = case["rows"], case["streams"] if "streams" in case else case["batch"]
    return [n * ((37 * s + 11) % 64) // 63 if case["ragged"] else n for s in range(count)]


def _visible(length, queries):
    """Pairs of a query and a row that it sees: the newest `queries` rows are the queries' own."""
    seen = length - queries
    return queries * seen + queries * (queries + 1) // 2 if seen >= 0 else length * (length + 1) // 2


def work(case):
    """Every row in use, query, score and position read once, every output and score written once; both products of attention."""
    d, e, lengths = case["head_dim"], 2 if case["dtype"] == "bf16" else 4, _lengths(case)
    total = sum(lengths)
    if case["op"] == "scored":
        heads = case["streams"] * case["group"]
        return {"bytes": 2 * total * d * e + 2 * heads * case["queries"] * d * e + 8 * total,
                "flops": 4 * d * case["group"] * sum(_visible(n, case["queries"]) for n in lengths)}
    if case["op"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lengths)
        return {"bytes": 8 * total + 8 * kept + 4 * kept * d * e, "flops": 0}
    heads, rows = case["batch"] * case["kv_heads"] * case["group"], case["kv_heads"] * (case["prefix"] + total)
    weights = 4 * case["kv_heads"] * case["prefix"] if case["weighted"] else 0
    return {"bytes": 2 * rows * d * e + 2 * heads * d * e + weights, "flops": 4 * d * case["group"] * case["kv_heads"] * (case["batch"] * case["prefix"] + total)}


# ---------------------------------------------------------------------------------------------- inputs

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _keys(g, lead, n, d):
    """Keys as the 8B-shaped workload has them: a mean per head, four channels ten times the others."""
    mean = 0.5 * torch.randn(*lead, 1, d, device="cuda", generator=g)
    scale = torch.ones(*lead, 1, d, device="cuda")
    scale.scatter_(-1, torch.rand(*lead, 1, d, device="cuda", generator=g).topk(4, dim=-1).indices, 10.0)
    return (torch.randn(*lead, n, d, device="cuda", generator=g) + mean) * scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    d, n, t = case["head_dim"], case["rows"], _type(case)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if case["op"] == "prefix":
        B, H = case["batch"], case["kv_heads"]
        keys = _keys(g, (H,), case["prefix"] + n * B, d)
        state = {"prefix_k": keys[:, :case["prefix"]].to(t).contiguous(), "prefix_v": normal(H, case["prefix"], d).to(t),
                 "k": keys[:, case["prefix"]:].reshape(H, B, n, d).transpose(0, 1).to(t).contiguous(), "v": normal(B, H, n, d).to(t),
                 "q": normal(B, H * case["group"], d).to(t), "w": None, "lens": lens}
        if case["weighted"]:                                # a compressed prefix: weights 4 first, then some of 2, then 1
            age = torch.arange(case["prefix"], device="cuda") / case["prefix"]
            state["w"] = torch.where(age < 0.8, 4.0, torch.where(age < 0.9, 2.0, 1.0)).expand(H, -1).contiguous()
        return {"case": case, **state}
    S = case["streams"]
    k, v = _keys(g, (S,), n, d).to(t), normal(S, n, d).to(t)
    # weights received so far: most rows hardly any, a tenth of them none at all
    score = torch.exp(2.0 * normal(S, n)) * (torch.rand(S, n, device="cuda", generator=g) > 0.1)
    state = {"case": case, "k": k, "v": v, "score": score, "lens": lens}
    if case["op"] == "scored":                              # a few calls like this one came before
        score *= 2 * case["group"] * case["scored"] / n
        return {**state, "q": normal(S, case["group"], case["queries"], d).to(t), "score_out": torch.zeros_like(score)}
    # positions of a cache that has been cut before: older rows in any order, each once, behind them the newest
    old = torch.rand(S, n, device="cuda", generator=g).masked_fill_(torch.arange(n, device="cuda") >= n - n // 4, 2.0).argsort(dim=1, stable=True)
    out = {"k": torch.zeros(S, case["keep"], d, dtype=t, device="cuda"), "score": torch.zeros(S, case["keep"], device="cuda"),
           "pos": torch.zeros(S, case["keep"], dtype=torch.int32, device="cuda"), "lens": torch.zeros_like(lens)}
    return {**state, "pos": (3 * old).to(torch.int32), "out": {**out, "v": torch.zeros_like(out["k"])}}


# ---------------------------------------------------------------------------------------------- passes

def run(state):
    return globals()["_run_" + state["case"]["op"]](state)


def _run_scored(state):
    case, q, lens = state["case"], state["q"], state["lens"]
    m, n, scored = case["queries"], case["rows"], case["scored"]
    if own:
        import paper_2502_07861_b200 as bk

        out, score = bk.attn_scored(state["k"], state["v"], q, lens=lens, score=state["score"], score_out=state["score_out"], n_scored=scored,
                                    decay=case["decay"])
        return {"out": out, "score": score}
    S, g, _, d = q.shape
    row = torch.arange(n, device="cuda")
    limit = lens[:, None, None, None] - m + 1 + torch.arange(m, device="cuda")[:, None]            # rows that a query sees
    s = torch.matmul(q.reshape(S, g * m, d).float(), state["k"].float().transpose(1, 2)).view(S, g, m, n).mul_(1 / math.sqrt(d))
    s.masked_fill_(row >= limit, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    p.div_(p.sum(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).tiny))                    # a query that sees nothing: zeros
    out = torch.matmul(p.view(S, g * m, n), state["v"].float()).view(S, g, m, d).to(q.dtype)
    got = case["decay"] * state["score"] + p[:, :, m - scored:].sum((1, 2))
    return {"out": out, "score": torch.where(row < lens[:, None], got, state["score_out"])}


def _run_evict(state):
    case, lens, score, pos = state["case"], state["lens"], state["score"], state["pos"]
    n, keep, out = case["rows"], case["keep"], state["out"]
    if own:
        import paper_2502_07861_b200 as bk

        return bk.cache_evict(state["k"], state["v"], score, keep, lens=lens, pos=pos, n_first=case["first"], n_recent=case["recent"], out=out)
    row = torch.arange(n, device="cuda").expand_as(score)
    held = row < lens[:, None]
    newest = pos.masked_fill(~held, -1).amax(1, keepdim=True)
    safe = held & ((pos < case["first"]) | (pos > newest - case["recent"]))
    rank = held.int() + safe.int()
    order = score.masked_fill(~held | safe, 0).argsort(dim=1, descending=True, stable=True)        # by score, the lowest row first among equals,
    order = order.gather(1, rank.gather(1, order).argsort(dim=1, descending=True, stable=True))    # the safe ones ahead, the rows behind the end last
    kept = torch.zeros_like(held).scatter_(1, order[:, :keep], True) & held
    hole, moves = ~kept[:, :keep] & held[:, :keep], kept.clone()
    moves[:, :keep] = False
    movers = row.masked_fill(~moves, n).sort(dim=1).values                                         # kept rows behind the new end, in order,
    nth = (hole.cumsum(1) - 1).clamp_(min=0)                                                       # fill the holes before it, in order
    source = torch.where(hole, movers.gather(1, nth), row[:, :keep])
    new = lens.clamp(max=keep)
    there = row[:, :keep] < new[:, None]
    source = source.masked_fill(~there, 0)
    pick = lambda x: torch.where(there[..., None], x.gather(1, source[..., None].expand(-1, -1, x.shape[2])), 0)  # noqa: E731
    return {"k": pick(state["k"]), "v": pick(state["v"]), "score": pick(score[..., None])[..., 0], "pos": pick(pos[..., None])[..., 0], "lens": new}


def _run_prefix(state):
    case, q, lens, w = state["case"], state["q"], state["lens"], state["w"]
    if own:
        import paper_2502_07861_b200 as bk

        return bk.decode_attn_prefix(state["prefix_k"], state["prefix_v"], state["k"], state["v"], q, lens=lens, weight=w)
    B, H, n, d = state["k"].shape
    g, P, scale = case["group"], case["prefix"], 1 / math.sqrt(d)
    qs = q.view(B, H, g, d).float()
    ahead = torch.matmul(qs.transpose(0, 1).reshape(H, B * g, d), state["prefix_k"].float().transpose(1, 2)).mul_(scale)
    if w is not None:
        ahead.add_(w.log()[:, None])
    own_rows = torch.matmul(qs, state["k"].float().transpose(2, 3)).mul_(scale)
    own_rows.masked_fill_(torch.arange(n, device="cuda") >= lens[:, None, None, None], -math.inf)
    top = torch.maximum(ahead.amax(-1).view(H, B, g).transpose(0, 1), own_rows.amax(-1))
    ahead.sub_(top.transpose(0, 1).reshape(H, B * g, 1)).exp_()
    own_rows.sub_(top[..., None]).exp_()
    value = torch.matmul(ahead, state["prefix_v"].float()).view(H, B, g, d).transpose(0, 1) + torch.matmul(own_rows, state["v"].float())
    total = ahead.sum(-1).view(H, B, g).transpose(0, 1) + own_rows.sum(-1)
    return value.div_(total[..., None]).to(q.dtype).reshape(B, H * g, d)


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _exact_scored(case, state):
    """softmax over the rows that a query sees, head by head; zeros for one that sees none."""
    m, d, first = case["queries"], case["head_dim"], case["queries"] - case["scored"]
    out, score = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda"), state["score_out"].double()
    for s, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        k, v, got = state["k"][s, :n].double(), state["v"][s, :n].double(), case["decay"] * state["score"][s, :n].double()
        empty = max(0, m - n)                               # queries ahead of the first row
        for h in range(case["group"]):
            z = (state["q"][s, h, empty:].double() @ k.T) / math.sqrt(d)
            future = torch.ones(z.shape, dtype=torch.bool, device="cuda").triu_(diagonal=n - (m - empty) + 1)
            p = torch.softmax(z.masked_fill_(future, -math.inf), dim=-1)
            out[s, h, empty:] = p @ v
            got += p[max(0, first - empty):].sum(0)
        score[s, :n] = got
    return {"out": out, "score": score}


def _exact_evict(case, state):
    """Stream by stream on the host: rows sorted by what protects them, score and place; those that stay keep their row if they can."""
    keep, out = case["keep"], {name: x.double() if x.is_floating_point() else x.clone() for name, x in state["out"].items()}
    scores, positions = state["score"].cpu().numpy(), state["pos"].cpu().numpy()
    for s, n in enumerate(_lengths(case)):
        score, pos = scores[s, :n], positions[s, :n]
        safe = (pos < case["first"]) | (pos > (pos.max() if n else 0) - case["recent"])
        best = sorted(range(n), key=lambda i: (not safe[i], 0.0 if safe[i] else -score[i], i))[:keep]
        stay, late = {i for i in best if i < keep}, iter(sorted(i for i in best if i >= keep))
        rows = torch.tensor([i if i in stay else next(late) for i in range(min(n, keep))], dtype=torch.long, device="cuda")
        for name in ("k", "v", "score", "pos"):
            out[name][s, :len(rows)] = state[name][s][rows].to(out[name].dtype)
        out["lens"][s] = len(rows)
    return out


def _exact_prefix(case, state):
    """Sequence by sequence: the weighted mean over the prefix and the sequence's own rows."""
    H, g, d, q = case["kv_heads"], case["group"], case["head_dim"], state["q"].double()
    out, pk, pv = torch.empty_like(q), state["prefix_k"].double(), state["prefix_v"].double()
    weight = torch.ones(H, case["prefix"], dtype=torch.float64, device="cuda") if state["w"] is None else state["w"].double()
    for b, n in enumerate(_lengths(case)):
        k, v = torch.cat([pk, state["k"][b, :, :n].double()], 1), torch.cat([pv, state["v"][b, :, :n].double()], 1)
        z = torch.einsum("hgd,hnd->hgn", q[b].view(H, g, d), k) / math.sqrt(d)
        e = torch.exp(z - z.amax(-1, keepdim=True)) * torch.cat([weight, weight.new_ones(H, n)], 1)[:, None]
        out[b] = (torch.einsum("hgn,hnd->hgd", e, v) / e.sum(-1, keepdim=True)).view(H * g, d)
    return out
