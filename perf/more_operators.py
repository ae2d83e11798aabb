"""Drafts that branch, and a cache that forgets, as cases whose time can be measured.

Several stored answers are close to a query: together they are a tree of drafted tokens, which the target model reads at once.
And a long context fills the pages: positions that attention has hardly weighed are evicted.  A pass is one of

``tree``     attention of a tree's rows over the paged cache: a row sees the context and its own ancestors.
``settle``   the path of the tree that the target's probabilities (from given random numbers) or largest logits agree with,
             and the token behind it.
``keep``     a tree's keys and values are written for some layers, those of the path that stands move behind the context, and
             all of them are read back.
``weigh``    the attention weights of a batch's rows, summed over rows and the heads that share keys, are added to what each
             position has.
``evict``    the positions with the largest sums, and the newest and first ones, stay: in the same pages or in others.

Sequence ``b`` has ``length[b]`` tokens in the cache, the rows ``first[b] .. first[b + 1] - 1`` of the batch are its newest ones, and
``pages[b]`` lists its pages.  Lengths, trees and paths follow from the case alone.
"""

import math
import random

import torch

own = False

DEV = "cuda:0"
E4M3_MAX = 448.0


def listed():
    return [
        # one near hit, two or three stored answers for it: latency
        {"name": "tree_one_bf16", "op": "tree", "dtype": "bf16", "n": 1, "nodes": 16, "nodes_hi": 16, "branch": 30, "len": 2001, "len_hi": 2001,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 21},
        # a serving batch of near hits over an 8-bit cache, trees of unlike sizes
        {"name": "tree_batch_fp8", "op": "tree", "dtype": "fp8", "n": 24, "nodes": 5, "nodes_hi": 64, "branch": 40, "len": 300, "len_hi": 6000,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 32, "window": 0, "mix": 22},
        # wide trees behind long contexts under a window, heads of 96 that fill no tile
        {"name": "tree_wide_bf16", "op": "tree", "dtype": "bf16", "n": 4, "nodes": 200, "nodes_hi": 256, "branch": 60, "len": 6000, "len_hi": 15000,
         "heads": 16, "kv_heads": 4, "d": 96, "page": 16, "window": 8000, "mix": 23},
        # one tree, greedy, logits in 16 bits
        {"name": "settle_one", "op": "settle", "dtype": "bf16", "n": 1, "nodes": 25, "nodes_hi": 25, "branch": 40, "vocab": 32000, "mode": "greedy", "mix": 24},
        # a batch, drawn from probabilities, an odd vocabulary
        {"name": "settle_batch", "op": "settle", "dtype": "f32", "n": 32, "nodes": 8, "nodes_hi": 40, "branch": 40, "vocab": 128001, "mode": "drawn", "mix": 25},
        # what stands of one tree, two layers
        {"name": "keep_one_bf16", "op": "keep", "dtype": "bf16", "n": 1, "nodes": 16, "nodes_hi": 16, "branch": 30, "len": 2001, "len_hi": 2001,
         "kv_heads": 8, "d": 128, "page": 64, "layers": 2, "mix": 26},
        # of a batch of trees in 8 bits, eight layers
        {"name": "keep_batch_fp8", "op": "keep", "dtype": "fp8", "n": 48, "nodes": 5, "nodes_hi": 64, "branch": 40, "len": 100, "len_hi": 1500,
         "kv_heads": 8, "d": 128, "page": 16, "layers": 8, "mix": 27},
        # decoding: the weights of one token of each sequence are added to what there is
        {"name": "weigh_step_fp8", "op": "weigh", "dtype": "fp8", "n": 64, "new": 1, "new_hi": 1, "len": 100, "len_hi": 16000, "whole": False,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 28},
        # a prompt's last tokens weigh all of it, for what is to be kept of it
        {"name": "weigh_tail_bf16", "op": "weigh", "dtype": "bf16", "n": 2, "new": 32, "new_hi": 32, "len": 9000, "len_hi": 16001, "whole": True,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 29},
        # every token of a prompt's chunk behind a long context weighs what it sees: the largest
        {"name": "weigh_chunk_bf16", "op": "weigh", "dtype": "bf16", "n": 1, "new": 4096, "new_hi": 4096, "len": 12289, "len_hi": 12289, "whole": True,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 30},
        # prompts come down to 2,048 positions, into pages of their own (the prompts' are shared with others)
        {"name": "evict_prompts_fp8", "op": "evict", "dtype": "fp8", "n": 5, "len": 3000, "len_hi": 16000, "keep": 2048, "recent": 64, "early": 4,
         "kv_heads": 8, "d": 128, "page": 64, "place": False, "mix": 31},
        # answers that go on: written, and those that have grown beyond 1,000 positions come down to it where they stand
        {"name": "evict_steps_bf16", "op": "evict", "dtype": "bf16", "n": 33, "len": 900, "len_hi": 1064, "keep": 1000, "recent": 200, "early": 4,
         "kv_heads": 8, "d": 64, "page": 16, "place": True, "mix": 32},
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "settle", "keep", "weigh", "weigh", "evict", "evict"])
    mix = rng.randrange(100, 1 << 20)
    low = rng.choice([1, 2, 5, 16])
    if op == "settle":
        return {"op": op, "dtype": rng.choice(["f32", "bf16"]), "n": _spread(rng, 1, 32), "nodes": low, "nodes_hi": _spread(rng, low, 64),
                "branch": rng.choice([0, 20, 40, 60, 90]), "vocab": _spread(rng, 1000, 131072), "mode": rng.choice(["drawn", "greedy"]), "mix": mix}
    case = {"op": op, "dtype": rng.choice(["bf16", "fp8"]), "d": rng.choice([64, 64, 96, 128, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128]),
            "kv_heads": rng.choice([1, 2, 4, 8]), "mix": mix}
    if op == "keep":
        return {**case, "n": _spread(rng, 1, 48), "nodes": low, "nodes_hi": _spread(rng, low, 128), "branch": rng.choice([0, 20, 40, 60, 90]), "len": 1,
                "len_hi": _spread(rng, 1, 1500), "layers": rng.randrange(1, 7)}
    if op == "evict":
        hi = _spread(rng, 40, 16000)
        keep = _spread(rng, 16, hi)
        recent = rng.randrange(0, keep // 2)
        return {**case, "n": _spread(rng, 1, max(1, min(33, 60000 // hi))), "len": _spread(rng, 1, hi), "len_hi": hi, "keep": keep, "recent": recent,
                "early": rng.randrange(0, min(8, keep - recent)), "place": rng.random() < 0.5}
    case["heads"] = case["kv_heads"] * rng.choice([1, 2, 4, 5, 8] if case["kv_heads"] < 8 else [1, 2, 4])
    case["window"] = rng.choice([0, 0, 0, _spread(rng, 16, 4096)])
    top = _spread(rng, 64, 32768)
    if op == "tree":
        hi = _spread(rng, low, 256)
        return {**case, "n": _spread(rng, 1, max(1, min(32, 100000 // top, 1200 // hi))), "nodes": low, "nodes_hi": hi, "branch": rng.choice([0, 20, 40, 60, 90]),
                "len": _spread(rng, 1, top), "len_hi": top}
    hi = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 65, 1500)])
    top = _spread(rng, 64, 65536) if hi < 65 else _spread(rng, 64, 9000)
    return {**case, "n": _spread(rng, 1, max(1, min(64, 300000 // top, 8000 // hi))), "new": 1 if rng.random() < 0.5 else hi, "new_hi": hi, "len": _spread(rng, 1, top),
            "len_hi": top, "whole": rng.random() < 0.5}


def _sizes(case):
    """Per sequence the new rows and the tokens in the cache, these included."""
    rng = random.Random(case["mix"])
    new, length = [], []
    for _ in range(case["n"]):
        if case["op"] == "evict":
            m = 0
        else:
            m = _spread(rng, case["nodes"], case["nodes_hi"]) if "nodes" in case else _spread(rng, case["new"], case["new_hi"])
        new.append(m)
        if case["op"] == "settle":
            length.append(m)
        elif "nodes" in case:
            length.append(m + _spread(rng, case["len"], case["len_hi"]))
        else:
            length.append(max(m, _spread(rng, case["len"], case["len_hi"])))
    return new, length


def _parents(case):
    """Of every sequence's rows: the row before it, or, `branch` times in a hundred, another earlier one; row 0 is the root."""
    rng = random.Random(case["mix"] + 1)
    return [[-1] + [i - 1 if rng.randrange(100) >= case["branch"] else rng.randrange(i) for i in range(1, m)] for m in _sizes(case)[0]]


def _ancestors(parents):
    lists = []
    for i, p in enumerate(parents):
        lists.append((lists[p] if p >= 0 else []) + [i])
    return lists


def _paths(case):
    """Of every sequence the path that stands: from the root to some row."""
    rng = random.Random(case["mix"] + 2)
    return [_ancestors(p)[rng.randrange(len(p))] for p in _parents(case)]


def _visible(case):
    """(position, row, head) pairs of all rows of one head; positions that some row sees, of all sequences."""
    new, length = _sizes(case)
    w = case["window"] or 1 << 40
    pairs, seqs = 0, 0
    for m, l, p in zip(new, length, _parents(case) if case["op"] == "tree" else [None] * len(new)):
        if p is None:
            pairs += sum(min(w, l - m + i + 1) for i in range(m))
            seqs += min(l, w + m - 1)
        else:
            deep = [len(a) for a in _ancestors(p)]
            pairs += sum(min(w, l - m + k) for k in deep)
            seqs += min(l - m, w - 1) + m
    return pairs, seqs


def work(case):
    new, length = _sizes(case)
    t = sum(new)
    if case["op"] == "settle":
        e = 4 if case["dtype"] == "f32" else 2
        return {"bytes": case["n"] * case["vocab"] * e + t * 20 + case["n"] * 4, "flops": case["n"] * case["vocab"]}
    cell = case["d"] + 4 if case["dtype"] == "fp8" else 2 * case["d"]
    if case["op"] == "keep":
        moved = sum(sum(1 for j, r in enumerate(p) if j != r) for p in _paths(case))
        vectors = 2 * case["layers"] * case["kv_heads"]
        return {"bytes": vectors * (t * (4 * case["d"] + 2 * cell) + moved * 2 * cell), "flops": vectors * t * case["d"]}
    if case["op"] == "evict":
        stay = [min(l, case["keep"]) for l in length]
        heads = case["kv_heads"]
        if case["place"]:  # written, evicted, read back
            gone = sum(l - s for l, s in zip(length, stay))
            return {"bytes": heads * (2 * (sum(length) * (2 * case["d"] + cell) + sum(stay) * (cell + 2 * case["d"]) + gone * 2 * cell) + 8 * sum(length)),
                    "flops": heads * sum(length)}
        return {"bytes": heads * (sum(stay) * (2 * (3 * cell + 2 * case["d"]) + 16) + 8 * sum(length)), "flops": heads * sum(length)}
    pairs, seqs = _visible(case)
    if case["op"] == "tree":
        return {"bytes": 2 * seqs * case["kv_heads"] * cell + t * case["heads"] * (4 * case["d"] + 4), "flops": 4 * pairs * case["heads"] * case["d"]}
    return {"bytes": seqs * case["kv_heads"] * cell + sum(length) * case["kv_heads"] * (4 if case["whole"] else 8) + t * case["heads"] * (2 * case["d"] + 4),
            "flops": 2 * pairs * case["heads"] * case["d"]}


# ---- inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _as_int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _ends(counts):
    ends = [0]
    for c in counts:
        ends.append(ends[-1] + c)
    return _as_int(ends)


def _cache_inputs(case, seed):
    """Keys and values of every token that is in the cache (layer by layer, rows of sequence after sequence, in 16 bits), the batch,
    and what goes with the operator: queries, the weights that positions have, logarithms of the rows' sums."""
    new, length = _sizes(case)
    g = _generator(seed)
    kvh, d, page, layers = case["kv_heads"], case["d"], case["page"], case.get("layers", 1)
    total = sum(new) if case["op"] == "keep" else sum(length)  # (a path's keys and values do not go by the context's)
    # channels of different size, as projections leave them: a few large ones in the keys
    big = 1.0 + 3.0 * (torch.rand(kvh, d, generator=g, device=DEV) < 0.04)
    k = torch.empty(layers, total, kvh, d, device=DEV, dtype=torch.bfloat16)
    v = torch.empty_like(k)
    for layer in range(layers):
        k[layer] = (_normal(g, total, kvh, d) * big).to(torch.bfloat16)
        v[layer] = (_normal(g, total, kvh, d) * torch.exp2(_normal(g, total, kvh, 1))).to(torch.bfloat16)
    need = [-(-x // page) for x in length]
    spare = [-(-min(x, case["keep"]) // page) if case["op"] == "evict" and not case["place"] else 0 for x in length]
    pool = sum(need) + sum(spare) + 3
    order = torch.randperm(pool, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    tables, at = [], 0
    for counts in (need, spare):
        table = torch.zeros(case["n"], max(1, max(counts)), dtype=torch.int32, device=DEV)
        for b, c in enumerate(counts):
            table[b, :c] = order[at:at + c]
            at += c
        tables.append(table)
    a = {"op": case["op"], "new": new, "length": length, "page": page, "pool": pool, "k": k, "v": v, "pages": tables[0], "to": tables[1], "scale": 1.0 / math.sqrt(d),
         "window": case.get("window", 0), "first_dev": _ends(new), "length_dev": _as_int(length), "all_dev": _ends(length)}
    if "heads" in case:
        a["q"] = _normal(g, sum(new), case["heads"], d).to(torch.bfloat16)
    if case["op"] in ("weigh", "evict"):
        # weights of a few positions are large, those of some are zero
        shape = (1, pool, kvh, page)
        mass = torch.exp(2.0 * _normal(g, *shape) - 4.0)
        a["mass"] = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, torch.zeros_like(mass), mass)
        a["born"] = torch.zeros(shape, dtype=torch.int32, device=DEV)
    if case["op"] == "evict":
        for b, l in enumerate(length):  # true positions: some have been evicted before, and their places are others' now
            pos = torch.arange(l, device=DEV)
            places = torch.argsort(torch.rand(kvh, l, generator=g, device=DEV), 1) * 2
            a["born"][0, a["pages"][b, pos // page].long(), :, pos % page] = places.t().to(torch.int32)
    if case["op"] == "weigh":
        a["whole"] = case["whole"]
        a["newest"] = _as_int([l - 1 + 3 * b for b, l in enumerate(length)])
        a["fresh"] = _as_int([0 if case["whole"] else l - m for l, m in zip(length, new)])
        a["lse"] = torch.cat([_plain_lse(a, case, b) for b in range(case["n"])])
    return a


def _held(case, x):
    return _plain_dequantised(x) if case["dtype"] == "fp8" else x.float()


def _plain_lse(a, case, b):
    """What attention gives for a sequence's rows, and what a program has from it."""
    m, l = a["new"][b], a["length"][b]
    start, row0 = sum(a["length"][:b]), sum(a["new"][:b])
    group = case["heads"] // case["kv_heads"]
    lse = torch.empty(m, case["heads"], device=DEV)
    row, pos = torch.arange(l - m, l, device=DEV)[:, None], torch.arange(l, device=DEV)[None]
    hidden = (pos > row) | ((pos <= row - a["window"]) if a["window"] else (pos < 0))
    for h in range(case["kv_heads"]):
        kt = _held(case, a["k"][0, start:start + l, h]).t().contiguous()
        for c in range(group):
            s = torch.matmul(a["q"][row0:row0 + m, h * group + c].float(), kt) * a["scale"]
            lse[:, h * group + c] = torch.logsumexp(s.masked_fill_(hidden, -math.inf), 1)
    return lse


def _settle_inputs(case, seed):
    new, _ = _sizes(case)
    g = _generator(seed)
    t, vocab = sum(new), case["vocab"]
    logits = _normal(g, t, vocab) * 2.5  # mass on some dozens of tokens of each row, and mostly one that leads
    logits.scatter_add_(1, logits.argmax(1, keepdim=True), 6.0 * torch.rand(t, 1, generator=g, device=DEV))
    target = (logits if case["mode"] == "greedy" else torch.softmax(logits, 1)).to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
    del logits
    guess = target.float().argmax(1)
    first = _ends(new)
    parents = _as_int([p for s in _parents(case) for p in s])
    base = torch.repeat_interleave(first[:-1].long(), torch.tensor(new, device=DEV))
    above = torch.where(parents >= 0, base + parents, base)  # the row that judges each row's token
    # children of one row differ, as the branches of stored answers do: one of them is what the target would say, or none is
    other = torch.randint(0, vocab, (t,), generator=g, device=DEV)
    wrong = torch.rand(t, generator=g, device=DEV) < 0.35
    tokens = torch.where(wrong, other, guess[above])
    tokens[first[:-1].long()] = other[first[:-1].long()]
    u = torch.rand(t, generator=g, device=DEV) if case["mode"] == "drawn" else None
    return {"op": "settle", "new": new, "target": target, "tokens": tokens.to(torch.int32), "parents": parents, "above": above, "base": base, "u": u, "first_dev": first,
            "deepest": max(len(x) for p in _parents(case) for x in _ancestors(p))}


# ---- the plain forms

def _plain_quantise(x):
    """Codes and one scale per vector of the last axis, in 32 bits."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    s = top / torch.full_like(top, E4M3_MAX)
    y = torch.where(s > 0, x / s, torch.zeros_like(x))
    return y.to(torch.float8_e4m3fn), s


def _plain_dequantised(x):
    code, s = _plain_quantise(x)
    return code.float() * s


def _plain_pool(case, pool):
    shape = (case.get("layers", 1), pool, case["page"], case["kv_heads"], case["d"])
    if case["dtype"] == "bf16":
        return {n: torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for n in ("k", "v")}
    return {**{n: torch.zeros(shape, dtype=torch.uint8, device=DEV) for n in ("k", "v")}, **{n: torch.zeros(shape[:4] + (1,), device=DEV) for n in ("ks", "vs")}}


def _plain_rows(s, lo, hi):
    """Pages and slots of positions lo[b] .. hi[b] - 1 of every sequence, sequence after sequence."""
    counts = [h - l for l, h in zip(lo, hi)]
    seq = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV))
    at = torch.cat([torch.arange(l, h, device=DEV) for l, h in zip(lo, hi)])
    return s["pages"][seq, at // s["page"]].long(), at % s["page"]


def _plain_write(pool, page, slot, k, v):
    for name, x in (("k", k), ("v", v)):
        if name + "s" in pool:
            code, scale = _plain_quantise(x)
            pool[name][:, page, slot] = code.view(torch.uint8)
            pool[name + "s"][:, page, slot] = scale
        else:
            pool[name][:, page, slot] = x


def _plain_gather(pool, name, page, slot):
    if name + "s" in pool:
        return pool[name][:, page, slot].view(torch.float8_e4m3fn).float() * pool[name + "s"][:, page, slot]
    return pool[name][:, page, slot].float()


def _plain_tree(s):
    outs, lses = [], []
    at = 0
    for m, l, parents, table in zip(s["new"], s["length"], s["parents"], s["pages"]):
        q = s["q"][at:at + m].float()
        # who is whose ancestor, by doubling: `up` is where each row's known ancestors end
        sees = torch.eye(m + 1, dtype=torch.bool, device=DEV)
        up = torch.cat((torch.where(parents >= 0, parents, m), torch.full_like(parents[:1], m))).long()
        for _ in range(max(1, m.bit_length())):
            sees = sees | sees[up]
            up = up[up]
        sees = sees[:m, :m]
        at += m
        heads, d = q.shape[1:]
        pos = torch.arange(l, device=DEV)
        page, slot = table[pos // s["page"]].long(), pos % s["page"]
        k, v = _plain_gather(s["pool"], "k", page, slot)[0], _plain_gather(s["pool"], "v", page, slot)[0]
        kvh = k.shape[1]
        q = q.view(m, kvh, heads // kvh, d).permute(1, 2, 0, 3).reshape(kvh, -1, d)
        w = torch.matmul(q, k.permute(1, 2, 0).contiguous()).view(kvh, heads // kvh, m, -1) * s["scale"]
        deep = sees.long().sum(1) - 1
        place = torch.cat((pos[:l - m], l - m + deep))  # (a row stands as deep as its ancestors are many)
        seen = torch.cat((torch.ones(m, l - m, dtype=torch.bool, device=DEV), sees), 1)
        if s["window"]:
            seen = seen & (place[None] > (l - m + deep)[:, None] - s["window"])
        w.masked_fill_(~seen, -math.inf)
        top = w.amax(-1, keepdim=True)
        w = torch.exp(w - top)
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w.view(kvh, -1, l), v.permute(1, 0, 2).contiguous()).view(kvh, heads // kvh, m, d) / total
        outs.append(o.permute(2, 0, 1, 3).reshape(m, heads, d).to(torch.bfloat16))
        lses.append((top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(m, heads))
    return [torch.cat(outs), torch.cat(lses)]


def _plain_settle(s):
    """Which token is drawn must not hang on the order of a sum over the vocabulary: sums in 64 bits."""
    target, tokens, vocab = s["target"], s["tokens"].long(), s["target"].shape[1]
    first = s["first_dev"].long()
    places, rows = torch.arange(vocab, device=DEV), torch.arange(len(tokens), device=DEV)
    above = torch.where(s["parents"] >= 0, s["above"], torch.full_like(s["above"], -1))
    at, going = first[:-1].clone(), torch.ones(len(s["new"]), dtype=torch.bool, device=DEV)
    accepted = torch.zeros_like(at)
    path, out = torch.full_like(tokens, -1), torch.full((len(tokens) + 1,), -1, device=DEV)  # (an entry more: for sequences that are done)
    path[first[:-1]] = 0
    for step in range(s["deepest"]):
        if s["u"] is None:
            x = target[at].float()
            x = torch.where(x == x.amax(1, keepdim=True), places, vocab).amin(1)
        else:
            sums = target[at].double().cumsum(1)
            x = torch.where(sums > s["u"][at].double()[:, None] * sums[:, -1:], places, vocab).amin(1)
        fits = (above[None] == at[:, None]) & (tokens[None] == x[:, None])
        child = torch.where(fits, rows, len(rows)).amin(1)
        on = going & (child < len(rows))
        out[torch.where(going, first[:-1] + accepted, len(tokens))] = x
        at = torch.where(on, child, at)
        accepted = accepted + on
        spot = first[:-1] + accepted
        path[spot] = torch.where(on, child - first[:-1], path[spot])
        going = on
    return [accepted.to(torch.int32), path.to(torch.int32), out[:-1].to(torch.int32)]


def _plain_keep(s):
    pool = s["pool"]
    page, slot = _plain_rows(s, [l - m for l, m in zip(s["length"], s["new"])], s["length"])
    _plain_write(pool, page, slot, s["k"], s["v"])
    base = torch.repeat_interleave(s["first_dev"][:-1].long(), torch.tensor(s["new"], device=DEV))
    to = (s["rows"] >= 0).nonzero().squeeze(1)
    of = base[to] + s["rows"].long()[to]
    for x in pool.values():
        x[:, page[to], slot[to]] = x[:, page[of], slot[of]]
    return [_plain_gather(pool, name, page, slot).to(torch.bfloat16) for name in ("k", "v")]


def _plain_weigh(s):
    mass, born = s["mass"], s["born"]
    mass.copy_(s["mass_before"])
    at = 0
    for b, (m, l, table) in enumerate(zip(s["new"], s["length"], s["pages"])):
        pos = torch.arange(l, device=DEV)
        page, slot = table[pos // s["page"]].long(), pos % s["page"]
        k = _plain_gather(s["pool"], "k", page, slot)[0]
        kvh = k.shape[1]
        row = torch.arange(l - m, l, device=DEV)[:, None, None]
        hidden = (pos > row) | ((pos <= row - s["window"]) if s["window"] else (pos < 0))
        q, lse = s["q"][at:at + m].float().unflatten(1, (kvh, -1)), s["lse"][at:at + m].unflatten(1, (kvh, -1))
        at += m
        sums = torch.empty(l, kvh, device=DEV)
        for h in range(kvh):
            w = torch.matmul(q[:, h], k[:, h].t().contiguous()) * s["scale"] - lse[:, h, :, None]
            sums[:, h] = torch.exp(w.masked_fill_(hidden, -math.inf)).sum((0, 1))
        new = pos >= s["fresh"][b]
        mass[0, page, :, slot] = torch.where(new[:, None], sums, mass[0, page, :, slot] + sums)
        born[0, page, :, slot] = torch.where(new[:, None], (s["newest"][b] - (l - 1 - pos))[:, None], born[0, page, :, slot]).to(torch.int32)
    return [mass, born]


def _plain_evict(s):
    pool, mass, born, keep = s["pool"], s["mass"], s["born"], s["keep"]
    mass.copy_(s["mass_before"])
    born.copy_(s["born_before"])
    if s["place"]:
        _plain_write(pool, *_plain_rows(s, [0] * len(s["length"]), s["length"]), s["k"], s["v"])
    ks, vs = [], []
    for b, (l, table) in enumerate(zip(s["length"], s["pages"])):
        stay = min(l, keep)
        pos = torch.arange(l, device=DEV)
        page, slot = table[pos // s["page"]].long(), pos % s["page"]
        w, when = mass[0, page, :, slot].t(), born[0, page, :, slot].t()  # [kv heads, positions]
        safe = (when > when.amax(1, keepdim=True) - s["recent"]) | (when < s["early"])
        best = torch.sort(torch.where(safe, math.inf, w), dim=1, descending=True, stable=True)[1][:, :stay]
        kept = torch.zeros_like(safe).scatter_(1, best, True)
        free, moves = ~kept[:, :stay], kept[:, stay:]
        # the first one beyond that is kept goes to the first free place, and so on
        order = torch.zeros(len(w), stay + 1, dtype=torch.int64, device=DEV)
        order.scatter_(1, torch.where(moves, moves.long().cumsum(1) - 1, stay), pos[stay:].expand_as(moves))
        of = torch.where(free, order.gather(1, (free.long().cumsum(1) - 1).clamp_(min=0)), pos[:stay])
        into = s["pages"] if s["place"] else s["to"]
        to_page, to_slot = into[b, pos[:stay] // s["page"]].long(), pos[:stay] % s["page"]
        head = torch.arange(len(w), device=DEV)[:, None]
        for x in pool.values():
            x[0, to_page, to_slot] = x[0][page[of], slot[of], head].transpose(0, 1)
        for x, y in ((mass, w), (born, when)):
            x[0, to_page, :, to_slot] = y.gather(1, of).t()
        ks.append(_plain_gather(pool, "k", to_page, to_slot)[0].to(torch.bfloat16))
        vs.append(_plain_gather(pool, "v", to_page, to_slot)[0].to(torch.bfloat16))
    return [torch.cat(ks), torch.cat(vs), mass, born]


# ---- the cases

def prepare(case, seed):
    if case["op"] == "settle":
        s = _settle_inputs(case, seed)
        if own:
            from paper_2508_18736_amd import siso
            s["kv"] = siso.PagedKV(1, 64, 1)
            s["batch"] = s["kv"].batch(s["first_dev"], rows=sum(s["new"]), max_new=max(s["new"]))
            s["tree"] = s["kv"].tree(s["batch"], s["parents"])
        return s
    s = _cache_inputs(case, seed)
    trees = _parents(case) if "nodes" in case else None
    if case["op"] == "tree":
        s["parents"] = [_as_int(p) for p in trees]
    if case["op"] == "keep":
        s["rows"] = _as_int([r for p, m in zip(_paths(case), s["new"]) for r in p + [-1] * (m - len(p))])
    if case["op"] in ("weigh", "evict"):
        s["mass_before"], s["born_before"] = s["mass"].clone(), s["born"].clone()
    if case["op"] == "evict":
        s.update(keep=case["keep"], recent=case["recent"], early=case["early"], place=case["place"], stay=[min(l, case["keep"]) for l in s["length"]])
    if own:
        from paper_2508_18736_amd import siso
        kv = s["kv"] = siso.PagedKV(case["kv_heads"], case["d"], s["pool"], page_tokens=case["page"], layers=case.get("layers", 1),
                                    dtype=siso.FP8 if case["dtype"] == "fp8" else siso.BF16)
        most = max(s["length"])
        if case["op"] != "evict":
            s["batch"] = kv.batch(s["first_dev"], s["length_dev"], s["pages"], rows=sum(s["new"]), max_new=max(s["new"]), max_length=most)
        s["all"] = kv.batch(s["all_dev"], s["length_dev"], s["pages"], rows=sum(s["length"]), max_new=most, max_length=most)
        if case["op"] == "tree":
            s["tree"] = kv.tree(s["batch"], _as_int([p for t in trees for p in t]))
        if case["op"] == "evict":
            s["stays"] = kv.batch(_ends(s["stay"]), _as_int(s["stay"]), s["pages"] if case["place"] else s["to"], rows=sum(s["stay"]), max_new=max(s["stay"]),
                                  max_length=max(s["stay"]))
        if case["op"] in ("weigh", "evict"):
            s["weights"] = kv.weights(s["mass"], s["born"])
        if case["op"] != "keep":  # what earlier calls have written
            kv.write(s["all"], s["k"][0], s["v"][0])
    else:
        s["pool"] = _plain_pool(case, s["pool"])
        if case["op"] != "keep":
            _plain_write(s["pool"], *_plain_rows(s, [0] * len(s["length"]), s["length"]), s["k"], s["v"])
    return s


def run(s):
    if not own:
        return {"tree": _plain_tree, "settle": _plain_settle, "keep": _plain_keep, "weigh": _plain_weigh, "evict": _plain_evict}[s["op"]](s)
    kv = s["kv"]
    if s["op"] == "tree":
        return list(kv.attend(s["batch"], s["q"], scale=s["scale"], window=s["window"], with_lse=True, tree=s["tree"]))
    if s["op"] == "settle":
        return list(kv.verify_tree(s["batch"], s["tree"], s["tokens"], s["target"], s["u"]))
    if s["op"] == "keep":
        out = [torch.empty_like(s["k"]), torch.empty_like(s["v"])]
        for layer in range(kv.layers):
            kv.write(s["batch"], s["k"][layer], s["v"][layer], layer=layer)
        kv.keep(s["batch"], s["rows"])
        for layer in range(kv.layers):
            kv.read(s["batch"], layer=layer, out_k=out[0][layer], out_v=out[1][layer])
        return out
    s["mass"].copy_(s["mass_before"])
    if s["op"] == "weigh":
        kv.weigh(s["batch"], s["q"], s["lse"], s["weights"], scale=s["scale"], window=s["window"], fresh=s["fresh"], newest=s["newest"])
        return [s["mass"], s["born"]]
    s["born"].copy_(s["born_before"])
    if s["place"]:
        kv.write(s["all"], s["k"][0], s["v"][0])
    kv.evict(s["all"], s["weights"], s["keep"], recent=s["recent"], early=s["early"], to=None if s["place"] else s["to"])
    return [*kv.read(s["stays"]), s["mass"], s["born"]]


# ---- the definitions in 64 bits

def _exact_codes(x):
    """The value that each element stands for once it is held as an E4M3 code under its vector's scale.  The scale and the quotient
    are single numbers of 32 bits by definition; everything else is in 64."""
    x = x.double()
    s = (x.abs().amax(-1, keepdim=True) / 448.0).float().double()
    y = torch.where(s > 0, x / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(x)).float().double()
    a = y.abs().clamp(max=448.0)
    exponent = torch.floor(torch.log2(a.clamp(min=2.0 ** -6))).clamp(min=-6, max=8)
    exponent = torch.where(torch.exp2(exponent) > a.clamp(min=2.0 ** -6), exponent - 1, exponent)
    step = torch.exp2(exponent - 3)
    return torch.sign(y) * torch.round(a / step).mul(step).clamp(max=448.0) * s


def exact(case, seed):
    if case["op"] == "settle":
        return _exact_settle(case, seed)
    a = _cache_inputs(case, seed)
    held = _exact_codes if case["dtype"] == "fp8" else (lambda x: x.double())
    return {"tree": _exact_tree, "keep": _exact_keep, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, a, held)


def _exact_tree(case, a, held):
    outs, lses, at, start = [], [], 0, 0
    group = case["heads"] // case["kv_heads"]
    for m, l, parents in zip(a["new"], a["length"], _parents(case)):
        seen = torch.zeros(m, l, dtype=torch.bool)
        for i, chain in enumerate(_ancestors(parents)):
            w = case["window"] or 1 << 40
            here = l - m + len(chain) - 1
            seen[i, max(0, here - w + 1):l - m] = True
            for k in chain[-min(w, len(chain)):]:
                seen[i, l - m + k] = True
        seen = seen.to(DEV)
        out = torch.empty(m, case["heads"], case["d"], dtype=torch.float64, device=DEV)
        lse = torch.empty(m, case["heads"], dtype=torch.float64, device=DEV)
        for h in range(case["kv_heads"]):
            k, v = held(a["k"][0, start:start + l, h]), held(a["v"][0, start:start + l, h])
            for c in range(h * group, (h + 1) * group):
                z = (a["q"][at:at + m, c].double() @ k.t()) / math.sqrt(case["d"])
                z = torch.where(seen, z, torch.full_like(z, -math.inf))
                lse[:, c] = torch.logsumexp(z, 1)
                out[:, c] = torch.softmax(z, 1) @ v
        at, start = at + m, start + l
        outs.append(out)
        lses.append(lse)
    return [torch.cat(outs), torch.cat(lses)]


def _exact_settle(case, seed):
    """Sequence by sequence and row by row, in Python's own numbers where a token is judged."""
    s = _settle_inputs(case, seed)
    tokens = s["tokens"].tolist()
    accepted, path, out, at = [], [], [], 0
    for parents in _parents(case):
        m, r, kept, said = len(parents), 0, [0], []
        while r is not None:
            p = s["target"][at + r].double()
            if s["u"] is None:
                x = int((p == p.max()).nonzero()[0])
            else:
                sums = torch.cumsum(p, 0)
                x = int((sums > float(s["u"][at + r]) * float(sums[-1])).nonzero()[0])
            said.append(x)
            r = next((c for c in range(m) if parents[c] == r and tokens[at + c] == x), None)
            if r is not None:
                kept.append(r)
        accepted.append(len(kept) - 1)
        path += kept + [-1] * (m - len(kept))
        out += said + [-1] * (m - len(said))
        at += m
    return [torch.tensor(x, dtype=torch.int32) for x in (accepted, path, out)]


def _exact_keep(case, a, held):
    rows, at = [], 0
    for path, m in zip(_paths(case), a["new"]):
        rows += [at + (path[i] if i < len(path) else i) for i in range(m)]
        at += m
    rows = torch.tensor(rows, device=DEV)
    return [held(a[name][:, rows]) for name in ("k", "v")]


def _exact_weigh(case, a, held):
    mass, born = a["mass"].double(), a["born"].clone()
    group = case["heads"] // case["kv_heads"]
    at = start = 0
    for b, (m, l) in enumerate(zip(a["new"], a["length"])):
        begin = int(a["fresh"][b])
        j = torch.arange(l, device=DEV)
        page, slot = a["pages"][b, j // case["page"]].long(), j % case["page"]
        for h in range(case["kv_heads"]):
            k = held(a["k"][0, start:start + l, h])
            total = torch.zeros(l, dtype=torch.float64, device=DEV)
            for r in range(0, m, 1024):
                e = min(m, r + 1024)
                p = torch.arange(l - m + r, l - m + e, device=DEV)[:, None]
                seen = (j[None] <= p) & ((j[None] > p - case["window"]) if case["window"] else (j[None] >= 0))
                for c in range(h * group, (h + 1) * group):
                    z = (a["q"][at + r:at + e, c].double() @ k.t()) / math.sqrt(case["d"]) - a["lse"][at + r:at + e, c].double()[:, None]
                    total += torch.where(seen, torch.exp(z), torch.zeros_like(z)).sum(0)
            old = mass[0, page, h, slot]
            old[begin:] = 0
            mass[0, page, h, slot] = old + total
            born[0, page[begin:], h, slot[begin:]] = (int(a["newest"][b]) - (l - 1) + j[begin:]).to(torch.int32)
        at, start = at + m, start + l
    return [mass, born]


def _exact_evict(case, a, held):
    mass, born = a["mass"].double(), a["born"].clone()
    ks, vs, start = [], [], 0
    for b, l in enumerate(a["length"]):
        stay = min(l, case["keep"])
        j = torch.arange(l, device=DEV)
        page, slot = a["pages"][b, j // case["page"]].long(), j % case["page"]
        j = j[:stay]
        to_page, to_slot = (a["pages"] if case["place"] else a["to"])[b, j // case["page"]].long(), j % case["page"]
        ko, vo = [], []
        for h in range(case["kv_heads"]):
            w, when = mass[0, page, h, slot], born[0, page, h, slot]
            weight, place = w.tolist(), when.tolist()
            newest = max(place)
            order = sorted(range(l), key=lambda i: (not (place[i] > newest - case["recent"] or place[i] < case["early"]),
                                                    0.0 if place[i] > newest - case["recent"] or place[i] < case["early"] else -weight[i], i))
            kept = set(order[:stay])
            later = iter(sorted(i for i in kept if i >= stay))
            of = torch.tensor([i if i in kept else next(later) for i in range(stay)], device=DEV)
            ko.append(held(a["k"][0, start + of, h]))
            vo.append(held(a["v"][0, start + of, h]))
            mass[0, to_page, h, to_slot] = w[of]
            born[0, to_page, h, to_slot] = when[of]
        ks.append(torch.stack(ko, 1))
        vs.append(torch.stack(vo, 1))
        start += l
    return [torch.cat(ks), torch.cat(vs), mass, born]
