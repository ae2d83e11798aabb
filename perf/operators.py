"""What a query that misses the semantic cache costs behind it, as cases whose time can be measured: the paged key/value
cache that the target model writes and reads, its attention over that cache, and the verification of a near miss's
stored answer as a draft.

A pass is one of

``store``    a ragged batch of new tokens is written to the paged cache (8-bit storage: quantised as it is written) and
             read back.
``attend``   the attention of every sequence's newest tokens over its pages: one token each (decoding), a few (the last
             token and a draft), or a prompt's chunk.
``verify``   drafted tokens are judged by the target's probabilities from given random numbers, or by its largest
             logits, and the token behind the last accepted one is chosen.

Sequence ``b`` of a batch has ``length[b]`` tokens in the cache, the rows ``first[b] .. first[b + 1] - 1`` of the batch are
its newest ones, and ``pages[b]`` lists its pages.  Lengths follow from the case alone.
"""

import math
import random

import torch

own = False

DEV = "cuda:0"
E4M3_MAX = 448.0


def listed():
    return [
        # eight sequences append one token each: latency of the write, sizes of a 1,024-dimensional model with 8 heads
        {"name": "store_tokens_fp8", "op": "store", "dtype": "fp8", "n": 8, "new": 1, "new_hi": 1, "len": 100, "len_hi": 4000,
         "kv_heads": 8, "d": 128, "page": 64, "mix": 1, "out": "bf16"},
        # prompts of a few hundred to a few thousand tokens, written behind what is there; no start or end on a page
        {"name": "store_prompts_fp8", "op": "store", "dtype": "fp8", "n": 13, "new": 200, "new_hi": 5000, "len": 200, "len_hi": 9000,
         "kv_heads": 8, "d": 128, "page": 64, "mix": 2, "out": "bf16"},
        # 16-bit storage with a head size that fills no tile (768 = 8 x 96), small pages
        {"name": "store_ragged_bf16", "op": "store", "dtype": "bf16", "n": 33, "new": 1, "new_hi": 700, "len": 1, "len_hi": 3000,
         "kv_heads": 8, "d": 96, "page": 16, "mix": 3, "out": "f32"},
        # one request alone, one token: the latency of decoding
        {"name": "decode_one_bf16", "op": "attend", "dtype": "bf16", "n": 1, "new": 1, "new_hi": 1, "len": 2001, "len_hi": 2001,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 4},
        # a serving batch over an 8-bit cache, contexts of very different lengths
        {"name": "decode_batch_fp8", "op": "attend", "dtype": "fp8", "n": 64, "new": 1, "new_hi": 1, "len": 100, "len_hi": 16000,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 5},
        # two long documents, one token each: a long axis and few rows
        {"name": "decode_long_bf16", "op": "attend", "dtype": "bf16", "n": 2, "new": 1, "new_hi": 1, "len": 100000, "len_hi": 131072,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 128, "window": 0, "mix": 6},
        # near misses: the last token and up to eight drafted ones of each sequence
        {"name": "draft_batch_fp8", "op": "attend", "dtype": "fp8", "n": 24, "new": 3, "new_hi": 9, "len": 300, "len_hi": 6000,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 32, "window": 0, "mix": 7},
        # a prompt's chunk behind a long context: the largest
        {"name": "prompt_chunk_bf16", "op": "attend", "dtype": "bf16", "n": 1, "new": 4096, "new_hi": 4096, "len": 12289, "len_hi": 12289,
         "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "mix": 8},
        # prompts and single tokens in one batch, a sliding window, 12 heads of 64 (768) that share nothing, 8-bit storage
        {"name": "mixed_window_fp8", "op": "attend", "dtype": "fp8", "n": 40, "new": 1, "new_hi": 1500, "len": 1, "len_hi": 5000,
         "heads": 12, "kv_heads": 12, "d": 64, "page": 16, "window": 1000, "mix": 9},
        # one near miss, its stored answer as the draft (no probabilities of its own)
        {"name": "verify_one", "op": "verify", "dtype": "f32", "n": 1, "drafts": 4, "drafts_hi": 4, "vocab": 32000, "mode": "stored", "mix": 10},
        # a batch whose drafts come from a small model with its probabilities, an odd vocabulary
        {"name": "verify_batch", "op": "verify", "dtype": "f32", "n": 64, "drafts": 1, "drafts_hi": 8, "vocab": 128001, "mode": "drawn", "mix": 11},
        # greedy decoding: the target's logits in 16 bits, all rows are searched
        {"name": "verify_greedy", "op": "verify", "dtype": "bf16", "n": 48, "drafts": 0, "drafts_hi": 8, "vocab": 65537, "mode": "greedy", "mix": 12},
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["store", "attend", "attend", "attend", "verify"])
    mix = rng.randrange(100, 1 << 20)
    if op == "verify":
        lo = rng.choice([0, 1, 4])
        return {"op": op, "dtype": rng.choice(["f32", "bf16"]), "n": _spread(rng, 1, 64), "drafts": lo, "drafts_hi": lo + rng.randrange(0, 9 - lo),
                "vocab": _spread(rng, 30000, 131072), "mode": rng.choice(["stored", "drawn", "greedy"]), "mix": mix}
    dtype = rng.choice(["bf16", "fp8"])
    d = rng.choice([64, 64, 96, 128, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    if op == "store":
        hi = _spread(rng, 1, 3000)
        n = _spread(rng, 1, max(1, min(64, 24000 // hi)))
        return {"op": op, "dtype": dtype, "n": n, "new": _spread(rng, 1, hi), "new_hi": hi, "len": 1, "len_hi": _spread(rng, 1, 8000),
                "kv_heads": kv_heads, "d": d, "page": page, "mix": mix, "out": rng.choice(["bf16", "f32"])}
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8] if kv_heads < 8 else [1, 2, 4])
    kind = rng.choice(["one", "few", "chunk", "mixed"])
    if kind == "one" or kind == "few":
        new, hi = (1, 1) if kind == "one" else (rng.randrange(1, 4), rng.randrange(4, 18))
        top = _spread(rng, 64, 65536)
        n = _spread(rng, 1, max(1, min(64, 300000 // top)))
        low = _spread(rng, 1, top)
    elif kind == "chunk":
        new = _spread(rng, 32, 2048)
        hi = new
        top = new + _spread(rng, 1, 8000)
        n, low = rng.randrange(1, 3), top
    else:
        new, hi = 1, _spread(rng, 32, 1500)
        top = _spread(rng, 32, 5000)
        n, low = _spread(rng, 2, 24), 1
    return {"op": op, "dtype": dtype, "n": n, "new": new, "new_hi": hi, "len": low, "len_hi": top, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "window": rng.choice([0, 0, 0, _spread(rng, 16, 4096)]), "mix": mix}


def _sizes(case):
    """Per sequence the new rows and (store, attend) the tokens in the cache, these included."""
    rng = random.Random(case["mix"])
    if case["op"] == "verify":
        return [1 + rng.randint(case["drafts"], case["drafts_hi"]) for _ in range(case["n"])], None
    new, length = [], []
    for _ in range(case["n"]):
        m = _spread(rng, case["new"], case["new_hi"])
        new.append(m)
        length.append(max(m, _spread(rng, case["len"], case["len_hi"])) if case["op"] == "attend" else m + _spread(rng, case["len"], case["len_hi"]))
    return new, length


def _visible(case):
    """Per row of every sequence: how many positions it sees, summed; per sequence: how many its rows see together."""
    new, length = _sizes(case)
    w = case["window"] or 1 << 40
    rows, seqs = 0, 0
    for m, l in zip(new, length):
        rows += sum(min(w, l - m + i + 1) for i in range(m))
        seqs += min(l, w + m - 1)
    return rows, seqs


def work(case):
    new, length = _sizes(case)
    t = sum(new)
    if case["op"] == "verify":
        e = 4 if case["dtype"] == "f32" else 2
        sides = 2 if case["mode"] == "drawn" else 1
        rows = t if case["mode"] == "greedy" else case["n"]
        return {"bytes": rows * case["vocab"] * e * sides + t * 12 + case["n"] * 8, "flops": rows * case["vocab"] * sides}
    cell = case["d"] + 4 if case["dtype"] == "fp8" else 2 * case["d"]
    if case["op"] == "store":
        vectors = 2 * t * case["kv_heads"]
        back = 2 if case["out"] == "bf16" else 4
        return {"bytes": vectors * (2 * case["d"] + 2 * cell + back * case["d"]), "flops": vectors * case["d"] * (3 if case["dtype"] == "fp8" else 1)}
    rows, seqs = _visible(case)
    return {"bytes": 2 * seqs * case["kv_heads"] * cell + t * case["heads"] * (4 * case["d"] + 4), "flops": 4 * rows * case["heads"] * case["d"]}


# ---- inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _cache_inputs(case, seed):
    """Keys and values of every token that is in the cache (rows of sequence after sequence, in 16 bits), queries, and
    the batch: first, length, pages."""
    new, length = _sizes(case)
    g = _generator(seed)
    total, kvh, d = sum(length), case["kv_heads"], case["d"]
    # channels of different size, as projections leave them: a few large ones in the keys
    big = 1.0 + 3.0 * (torch.rand(kvh, d, generator=g, device=DEV) < 0.04)
    k = torch.empty(total, kvh, d, device=DEV, dtype=torch.bfloat16)
    v = torch.empty_like(k)
    for at in range(0, total, 65536):
        part = min(65536, total - at)
        k[at:at + part] = (_normal(g, part, kvh, d) * big).to(torch.bfloat16)
        v[at:at + part] = (_normal(g, part, kvh, d) * torch.exp2(_normal(g, part, kvh, 1))).to(torch.bfloat16)
    q = None
    if case["op"] == "attend":
        q = _normal(g, sum(new), case["heads"], d).to(torch.bfloat16)
    need = [-(-x // case["page"]) for x in length]
    order = torch.randperm(sum(need) + 3, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    width = max(need)
    pages = torch.zeros(case["n"], width, dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(need):
        pages[b, :c] = order[at:at + c]
        at += c
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ends = lambda x: as_int([sum(x[:i]) for i in range(len(x) + 1)])  # noqa: E731
    return {"k": k, "v": v, "q": q, "pages": pages, "pool": sum(need) + 3, "new": new, "length": length,
            "first_dev": ends(new), "length_dev": as_int(length), "all_dev": ends(length)}


def _verify_inputs(case, seed):
    new, _ = _sizes(case)
    g = _generator(seed)
    t, vocab = sum(new), case["vocab"]
    kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    logits = _normal(g, t, vocab) * 2.5  # mass on some dozens of tokens of each row, and mostly one that leads
    logits.scatter_add_(1, logits.argmax(1, keepdim=True), 6.0 * torch.rand(t, 1, generator=g, device=DEV))
    first = [sum(new[:i]) for i in range(len(new) + 1)]
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"new": new, "first_dev": as_int(first), "u_accept": None, "u_sample": None, "draft": None}
    if case["mode"] == "greedy":
        s["target"] = logits.to(kind)
        guess = s["target"].float().argmax(1)
    elif case["mode"] == "stored":
        s["target"] = torch.softmax(logits, 1).to(kind)
        guess = s["target"].float().argmax(1)
    else:
        s["target"] = torch.softmax(logits, 1).to(kind)
        near = logits + 0.7 * _normal(g, t, vocab)
        s["draft"] = torch.softmax(near, 1).to(kind)
        guess = (near - torch.log(-torch.log(torch.rand(t, vocab, generator=g, device=DEV).clamp_(1e-7, 1 - 1e-7)))).argmax(1)
    # the chunk's own tokens: the last one that stands, then the draft of each row before it; now and then some other one
    other = torch.randint(0, vocab, (t,), generator=g, device=DEV)
    wrong = torch.rand(t, generator=g, device=DEV) < (0.1 if case["mode"] != "drawn" else 0.0)
    tokens = torch.where(wrong, other, guess).roll(1)
    tokens[torch.tensor(first[:-1], device=DEV)] = other[:case["n"]]
    s["tokens"] = tokens.to(torch.int32)
    if case["mode"] != "greedy":
        s["u_accept"] = torch.rand(t, generator=g, device=DEV)
        s["u_sample"] = torch.rand(case["n"], generator=g, device=DEV)
    return s


# ---- the plain forms

def _plain_quantise(x):
    """Codes and one scale per vector of the last axis, in 32 bits."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    s = top / torch.full_like(top, E4M3_MAX)  # (a number instead of the tensor would be multiplied by its rounded reciprocal)
    y = torch.where(s > 0, x / s, torch.zeros_like(x))
    return y.to(torch.float8_e4m3fn), s


def _plain_rows(s, b):
    """Page and slot of positions lo .. hi - 1 of sequence b."""
    at = torch.arange(s["length"][b] - s["new"][b], s["length"][b], device=DEV)
    return s["pages"][b, at // s["page"]].long(), at % s["page"]


def _plain_pool(case, pool):
    shape = (pool, case["page"], case["kv_heads"], case["d"])
    if case["dtype"] == "bf16":
        return {"k": torch.zeros(shape, dtype=torch.bfloat16, device=DEV), "v": torch.zeros(shape, dtype=torch.bfloat16, device=DEV)}
    scale = shape[:3] + (1,)
    return {"k": torch.zeros(shape, dtype=torch.float8_e4m3fn, device=DEV), "v": torch.zeros(shape, dtype=torch.float8_e4m3fn, device=DEV),
            "ks": torch.zeros(scale, device=DEV), "vs": torch.zeros(scale, device=DEV)}


def _plain_write(pool, page, slot, k, v):
    for name, x in (("k", k), ("v", v)):
        if name + "s" in pool:
            code, scale = _plain_quantise(x)
            pool[name].view(torch.uint8)[page, slot] = code.view(torch.uint8)
            pool[name + "s"][page, slot] = scale
        else:
            pool[name][page, slot] = x


def _plain_gather(pool, name, page, slot):
    if name + "s" in pool:
        return pool[name].view(torch.uint8)[page, slot].view(torch.float8_e4m3fn).float() * pool[name + "s"][page, slot]
    return pool[name][page, slot].float()


def _plain_store(s):
    page, slot = zip(*[_plain_rows(s, b) for b in range(len(s["new"]))])
    page, slot = torch.cat(page), torch.cat(slot)
    _plain_write(s["pool"], page, slot, s["k"], s["v"])
    return [_plain_gather(s["pool"], name, page, slot).to(s["out"]) for name in ("k", "v")]


def _plain_attend(s):
    outs, lses = [], []
    at = 0
    for m, l, table in zip(s["new"], s["length"], s["pages"]):
        q = s["q"][at:at + m].float()
        at += m
        heads, d = q.shape[1:]
        low = max(0, l - m - s["window"] + 1) if s["window"] else 0
        pos = torch.arange(low, l, device=DEV)
        page, slot = table[pos // s["page"]].long(), pos % s["page"]
        k, v = _plain_gather(s["pool"], "k", page, slot), _plain_gather(s["pool"], "v", page, slot)
        kvh = k.shape[1]
        q = q.view(m, kvh, heads // kvh, d).permute(1, 2, 0, 3).reshape(kvh, -1, d)
        w = torch.matmul(q, k.permute(1, 2, 0).contiguous()).view(kvh, heads // kvh, m, -1) * s["scale"]
        row = torch.arange(l - m, l, device=DEV)[:, None]
        hidden = pos[None] > row
        if s["window"]:
            hidden = hidden | (pos[None] <= row - s["window"])
        w.masked_fill_(hidden, -math.inf)
        top = w.amax(-1, keepdim=True)
        w = torch.exp(w - top)
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w.view(kvh, -1, pos.shape[0]), v.permute(1, 0, 2).contiguous()).view(kvh, heads // kvh, m, d) / total
        outs.append(o.permute(2, 0, 1, 3).reshape(m, heads, d).to(torch.bfloat16))
        lses.append((top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(m, heads))
    return [torch.cat(outs), torch.cat(lses)]


def _plain_verify(s):
    """Which token is named must not hang on the order of a sum over the vocabulary: products and sums in 64 bits."""
    target, tokens, vocab = s["target"], s["tokens"].long(), s["target"].shape[1]
    first = s["first_dev"].long()
    rows = first[1:] - first[:-1]
    i = torch.arange(s["most"], device=DEV)
    row = first[:-1, None] + i[None]  # row i of each sequence judges the token of row i + 1
    judged = i[None] < rows[:, None] - 1
    row = torch.where(judged, row, first[:-1, None])
    draft = torch.where(judged, tokens[torch.where(judged, row + 1, row)], torch.zeros_like(row))
    if s["u_accept"] is None:
        x = target.float()
        best = torch.where(x == x.amax(1, keepdim=True), torch.arange(vocab, device=DEV), vocab).amin(1)
        good = best[row] == draft
    else:
        p = target[row, draft].double()
        c = s["draft"][row, draft].double() if s["draft"] is not None else torch.ones_like(p)
        good = s["u_accept"][row].double() * c < p
    accepted = (good & judged).long().cumprod(1).sum(1)
    stop = first[:-1] + accepted
    if s["u_accept"] is None:
        chosen = best[stop]
    else:
        w = target[stop].double()
        refused = accepted < rows - 1
        if s["draft"] is not None:
            w = torch.where(refused[:, None], (w - s["draft"][stop].double()).clamp_(min=0), w)
        else:
            not_this = torch.where(refused, tokens[torch.where(refused, stop + 1, stop)], torch.full_like(stop, -1))
            w = torch.where(torch.arange(vocab, device=DEV)[None] == not_this[:, None], torch.zeros_like(w), w)
        sums = w.cumsum(1)
        chosen = torch.where(sums > s["u_sample"].double()[:, None] * sums[:, -1:], torch.arange(vocab, device=DEV), vocab).amin(1)
    out = torch.full_like(tokens, -1)
    kept = judged & (i[None] < accepted[:, None])
    out[row[kept]] = draft[kept]
    out[stop] = chosen
    return [accepted.to(torch.int32), out.to(torch.int32)]


# ---- the cases

def prepare(case, seed):
    if case["op"] == "verify":
        s = _verify_inputs(case, seed)
        s["most"] = max(s["new"])
        if own:
            from paper_2508_18736_amd import siso
            s["kv"] = siso.PagedKV(1, 64, 1)
            s["batch"] = s["kv"].batch(s["first_dev"], max_new=s["most"])
        s["op"] = "verify"
        return s
    a = _cache_inputs(case, seed)
    s = {"op": case["op"], "page": case["page"], "window": case.get("window", 0), "scale": 1.0 / math.sqrt(case["d"]), "q": a["q"],
         "new": a["new"], "length": a["length"], "pages": a["pages"]}
    if case["op"] == "store":
        rows = torch.cat([torch.arange(e - m, e) for m, e in zip(a["new"], torch.tensor(a["length"]).cumsum(0).tolist())]).to(DEV)
        s["k"], s["v"] = a["k"][rows], a["v"][rows]
        s["out"] = torch.bfloat16 if case["out"] == "bf16" else torch.float32
    if own:
        from paper_2508_18736_amd import siso
        s["kv"] = siso.PagedKV(case["kv_heads"], case["d"], a["pool"], page_tokens=case["page"], dtype=siso.FP8 if case["dtype"] == "fp8" else siso.BF16)
        s["batch"] = s["kv"].batch(a["first_dev"], a["length_dev"], a["pages"], max_new=max(a["new"]), max_length=max(a["length"]))
        if case["op"] == "attend":  # what earlier calls have written
            s["kv"].write(s["kv"].batch(a["all_dev"], a["length_dev"], a["pages"]), a["k"], a["v"])
    else:
        s["pool"] = _plain_pool(case, a["pool"])
        if case["op"] == "attend":
            at = 0
            for l, table in zip(a["length"], a["pages"]):
                pos = torch.arange(l, device=DEV)
                _plain_write(s["pool"], table[pos // case["page"]].long(), pos % case["page"], a["k"][at:at + l], a["v"][at:at + l])
                at += l
    return s


def run(s):
    if not own:
        return {"store": _plain_store, "attend": _plain_attend, "verify": _plain_verify}[s["op"]](s)
    kv, batch = s["kv"], s["batch"]
    if s["op"] == "store":
        kv.write(batch, s["k"], s["v"])
        return list(kv.read(batch, dtype=s["out"]))
    if s["op"] == "attend":
        return list(kv.attend(batch, s["q"], scale=s["scale"], window=s["window"], with_lse=True))
    return list(kv.verify(batch, s["tokens"], s["target"], s["draft"], s["u_accept"], s["u_sample"]))


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
    if case["op"] == "verify":
        return _exact_verify(case, seed)
    a = _cache_inputs(case, seed)
    held = _exact_codes if case["dtype"] == "fp8" else (lambda x: x.double())
    starts = [sum(a["length"][:i]) for i in range(len(a["length"]) + 1)]
    if case["op"] == "store":
        return [torch.cat([held(x[e - m:e]) for m, e in zip(a["new"], starts[1:])]) for x in (a["k"], a["v"])]
    outs, lses, at = [], [], 0
    group = case["heads"] // case["kv_heads"]
    for b, (m, l) in enumerate(zip(a["new"], a["length"])):
        out = torch.empty(m, case["heads"], case["d"], dtype=torch.float64, device=DEV)
        lse = torch.empty(m, case["heads"], dtype=torch.float64, device=DEV)
        for h in range(case["kv_heads"]):
            k, v = held(a["k"][starts[b]:starts[b + 1], h]), held(a["v"][starts[b]:starts[b + 1], h])
            for r in range(0, m, 1024):
                e = min(m, r + 1024)
                p = torch.arange(l - m + r, l - m + e, device=DEV)[:, None]
                j = torch.arange(l, device=DEV)[None]
                seen = (j <= p) & ((j > p - case["window"]) if case["window"] else (j >= 0))
                for c in range(group):
                    z = (a["q"][at + r:at + e, h * group + c].double() @ k.t()) / math.sqrt(case["d"])
                    z = torch.where(seen, z, torch.full_like(z, -math.inf))
                    lse[r:e, h * group + c] = torch.logsumexp(z, 1)
                    out[r:e, h * group + c] = torch.softmax(z, 1) @ v
        at += m
        outs.append(out)
        lses.append(lse)
    return [torch.cat(outs), torch.cat(lses)]


def _exact_verify(case, seed):
    """Sequence by sequence and row by row, in Python's own numbers where a token is judged."""
    s = _verify_inputs(case, seed)
    tokens = s["tokens"].tolist()
    accepted, out = [], []
    at = 0
    for b, rows in enumerate(s["new"]):
        kept = 0
        while True:
            r = at + kept
            p = s["target"][r].double()
            if case["mode"] == "greedy":
                following = int((p == p.max()).nonzero()[0])
                good = kept < rows - 1 and following == tokens[r + 1]
            elif kept < rows - 1:
                x = tokens[r + 1]
                c = float(s["draft"][r, x].double()) if s["draft"] is not None else 1.0
                good = float(s["u_accept"][r]) * c < float(p[x])
            else:
                good = False
            if not good:
                break
            kept += 1
        if case["mode"] != "greedy":
            if kept < rows - 1:
                if s["draft"] is not None:
                    p = (p - s["draft"][r].double()).clamp(min=0)
                else:
                    p[tokens[r + 1]] = 0.0
            sums = torch.cumsum(p, 0)
            following = int((sums > float(s["u_sample"][b]) * float(sums[-1])).nonzero()[0])
        accepted.append(kept)
        out += tokens[at + 1:at + 1 + kept] + [following] + [-1] * (rows - 1 - kept)
        at += rows
    return [torch.tensor(accepted, dtype=torch.int32), torch.tensor(out, dtype=torch.int32)]
