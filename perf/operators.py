"""Performance cases of the operators over a paged key/value cache: rotary
positions, writing new tokens into the cache, attention of one or more new
tokens of every sequence over it, and eviction by accumulated weight.

A case is a plain dict: "op" (rotary, append, attend, evict), "dtype", the head
counts "hq" and "hkv", the head width "d", the page size "page" and the sizes of
the batch. Ragged batches follow from the case's own numbers (``_batch``), so
that every seed has the same shapes and other values. The plain forms treat a
batch as one padded block.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------ cases ---

def _rotary(dtype, tokens, heads, d, rot, interleaved, transpose=False, far=8192, scaling="none"):
    return dict(op="rotary", dtype=dtype, tokens=tokens, hq=heads, d=d, rot=rot,
                interleaved=interleaved, transpose=transpose, far=far, scaling=scaling)


def _append(dtype, seqs, new, length, hkv, d, page, interleaved=False):
    return dict(op="append", dtype=dtype, seqs=seqs, new=new, length=length, hkv=hkv, d=d,
                page=page, interleaved=interleaved)


def _attend(dtype, seqs, new, length, hq, hkv, d, page, accumulate=False, causal=True):
    return dict(op="attend", dtype=dtype, seqs=seqs, new=new, length=length, hq=hq, hkv=hkv, d=d,
                page=page, accumulate=accumulate, causal=causal)


def _evict(dtype, seqs, length, hkv, d, page, budget, recent):
    return dict(op="evict", dtype=dtype, seqs=seqs, length=length, hkv=hkv, d=d, page=page,
                budget=budget, recent=recent)


def listed():
    cases = [
        # One token's queries of a small batch: the call's latency.
        _rotary("bf16", 5, 32, 128, 128, False),
        # A long prompt's queries, a part of each head, far positions stretched.
        _rotary("bf16", 16384, 32, 128, 64, True, far=1000000, scaling="yarn"),
        # A training batch's gradient in single precision, odd sizes.
        _rotary("f32", 3001, 12, 80, 80, False, transpose=True, scaling="linear"),
        # The new token of each of many sequences goes into the cache.
        _append("bf16", 64, 1, 4096, 8, 128, 16),
        # Prompts of several users go into the cache at once.
        _append("f16", 9, 2048, 4096, 8, 128, 64, interleaved=True),
        # Single-token serving of one user: latency and the split of a short cache.
        _attend("bf16", 1, 1, 1500, 32, 8, 128, 16),
        # Single-token serving of a full batch with long caches, weights gathered.
        _attend("bf16", 64, 1, 16384, 32, 8, 128, 64, accumulate=True),
        # Chunks of long prompts over what is cached of them.
        _attend("bf16", 4, 2048, 16384, 32, 8, 128, 64),
        # Chunks of middling prompts, narrow heads, weights gathered for eviction.
        _attend("f16", 6, 700, 3001, 14, 2, 64, 16, accumulate=True),
        # Smoothing over a stored set in single precision: every key is visible.
        _attend("f32", 3, 300, 2500, 6, 6, 96, 48, causal=False),
        # A few sequences past their budget.
        _evict("bf16", 2, 1100, 4, 64, 16, 1024, 128),
        # A batch of long caches cut to half.
        _evict("bf16", 32, 12288, 8, 128, 64, 6144, 512),
    ]
    for c in cases:
        size = "x".join(str(c[k]) for k in ("tokens", "seqs", "new", "length", "budget") if k in c)
        heads = "_".join("%s%d" % (k, c[k]) for k in ("hq", "hkv", "d") if k in c)
        c["name"] = "_".join([c["op"], c["dtype"], size, heads])
    return cases


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["rotary", "append", "attend", "attend", "attend", "attend", "evict"])
    d = rng.choice([64, 128, 128, 80, 96, 72, 256])
    page = rng.choice([16, 32, 64, 128, 24, 7])
    hkv = rng.choice([1, 2, 4, 8, 5])
    while True:
        if op == "rotary":
            c = _rotary(dtype, _log_int(rng, 1, 16384), rng.randint(1, 40), d,
                        2 * rng.randint(1, d // 2), rng.random() < 0.5, rng.random() < 0.5,
                        _log_int(rng, 100, 2000000), rng.choice(["none", "linear", "ntk", "yarn"]))
        elif op == "append":
            new = rng.choice([1, _log_int(rng, 2, 2048)])
            c = _append(dtype, _log_int(rng, 1, 64), new, new + _log_int(rng, 1, 4096), hkv, d,
                        page, rng.random() < 0.5)
        elif op == "attend":
            new = rng.choice([1, _log_int(rng, 2, 2048)])
            c = _attend(dtype, _log_int(rng, 1, 64), new, new + _log_int(rng, 10, 16384),
                        hkv * rng.choice([1, 2, 4, 7, 8]), hkv, d, page, rng.random() < 0.4,
                        rng.random() < 0.8)
        else:
            length = _log_int(rng, 20, 12288)
            budget = rng.randint(1, length)
            c = _evict(dtype, _log_int(rng, 1, 32), length, hkv, d, page, budget,
                       rng.randint(0, budget))
        w = work(c)
        if w["flops"] < (1.2e11 if dtype == "f32" else 8e11) and w["bytes"] < 2e9:
            return c


def _batch(case):
    """(new tokens, length) of every sequence: up to a half shorter than the
    case's numbers; the first has the full ones."""
    rng = random.Random(case["seqs"] * 1000003 + case["length"])
    new, out = case.get("new", 0), []
    for s in range(case["seqs"]):
        if s == 0:
            out.append((new, case["length"]))
            continue
        n = new if new <= 1 else rng.randint((new + 1) // 2, new)
        out.append((n, max(n, rng.randint((case["length"] + 1) // 2, case["length"]))))
    return out


def work(case):
    """What one pass cannot do without: inputs read and outputs written once."""
    size, d = SIZES[case["dtype"]], case["d"]
    if case["op"] == "rotary":
        values = case["tokens"] * case["hq"] * d
        return {"bytes": 2 * values * size + 8 * case["tokens"] + 4 * case["rot"],
                "flops": 3 * case["tokens"] * case["hq"] * case["rot"]}
    batch = _batch(case)
    row = case["hkv"] * d * size                     # one token's keys (or values)
    if case["op"] == "append":
        tokens = sum(n for n, _ in batch)
        return {"bytes": tokens * (4 * row + 4 * case["hkv"] + 8),
                "flops": 3 * tokens * case["hkv"] * d}
    if case["op"] == "attend":
        tokens, keys = sum(n for n, _ in batch), sum(L for _, L in batch)
        seen = sum(n * L - (n * (n - 1) // 2 if case["causal"] else 0) for n, L in batch)
        weights = 8 * keys * case["hkv"] if case["accumulate"] else 0
        return {"bytes": 2 * tokens * case["hq"] * d * size + 2 * keys * row + weights
                + 4 * keys // case["page"],
                "flops": 4 * d * case["hq"] * seen}
    keys = sum(L for _, L in batch)
    left = sum(min(L, case["budget"]) for _, L in batch)
    return {"bytes": 4 * keys * case["hkv"] + left * (4 * row + 12 * case["hkv"]),
            "flops": keys * case["hkv"]}


# ----------------------------------------------------------------- inputs ---

def _frequencies(case):
    """(frequencies in fp64, factor of the values) of a rotary case, on the host."""
    n = case["rot"] if "rot" in case else case["d"]
    i = torch.arange(n // 2, dtype=torch.float64)
    scaling, factor, original, base = case.get("scaling", "none"), 8.0, 4096.0, 10000.0
    if scaling == "ntk" and n > 2:
        base = base * factor ** (n / (n - 2))
    f = base ** (-2.0 * i / n)
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        turns = original * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f / factor * (1.0 - keep) + f * keep
        return f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _pages(batch, page, g, spare=3):
    """(table, pages in the pool): every sequence's pages anywhere in the pool."""
    need = [-(-L // page) for L in batch]
    pool = sum(need) + spare
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(batch), max(max(need), 1), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, pool


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, d = DTYPES[case["dtype"]], case["d"]

    def normal(*shape, by=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(by).to(dt)

    s = {"case": case}
    if case["op"] in ("rotary", "append"):
        freqs, s["factor"] = _frequencies(case)
        s["freqs"] = freqs.cuda()
    if case["op"] == "rotary":
        s["x"] = normal(case["tokens"], case["hq"], d)
        s["positions"] = torch.randint(0, case["far"], (case["tokens"],), generator=g,
                                       device="cuda")
        return s
    batch = _batch(case)
    s["batch"], hkv, page = batch, case["hkv"], case["page"]
    table, pool = _pages([L for _, L in batch], page, g)
    lengths = _ints([L for _, L in batch])
    if case["op"] == "append":
        k = torch.zeros(pool, hkv, page, d, dtype=dt, device="cuda")
        v, weight = torch.zeros_like(k), torch.zeros(pool, hkv, page, device="cuda")
    else:
        k, v = normal(pool, hkv, page, d), normal(pool, hkv, page, d)
        if case["op"] == "evict":
            # heavy-tailed, and with tokens that no row ever looked at
            weight = torch.randn(pool, hkv, page, generator=g, device="cuda").mul_(2.0).exp_()
            weight = torch.where(weight < 0.1, torch.zeros_like(weight), weight)
        else:
            weight = torch.rand(pool, hkv, page, generator=g, device="cuda")
    s.update(k=k, v=v, weight=weight, table=table, lengths=lengths)
    if case["op"] == "evict":
        to, pool2 = _pages([min(L, case["budget"]) for _, L in batch], page, g)
        s.update(to_k=torch.zeros(pool2, hkv, page, d, dtype=dt, device="cuda"),
                 to_v=torch.zeros(pool2, hkv, page, d, dtype=dt, device="cuda"),
                 to_weight=torch.zeros(pool2, hkv, page, device="cuda"),
                 to_table=to, to_lengths=torch.zeros(len(batch), dtype=torch.int32, device="cuda"))
    else:
        new = [n for n, _ in batch]
        tokens = sum(new)
        s["offsets"] = _ints([sum(new[:i]) for i in range(len(new) + 1)])
        if case["op"] == "append":
            s["new_k"], s["new_v"] = normal(tokens, hkv, d), normal(tokens, hkv, d)
            s["positions"] = torch.cat([torch.arange(L - n, L) for n, L in batch]).cuda()
        else:
            s["q"] = normal(tokens, case["hq"], d, by=1.5)
            s["weight_out"] = torch.zeros_like(weight)
    if own:
        import paper_2202_12674_amd as P
        s["cache"] = P.PagedCache(k, v, table, lengths, weight)
        if case["op"] == "evict":
            s["target"] = P.PagedCache(s["to_k"], s["to_v"], s["to_table"], s["to_lengths"],
                                       s["to_weight"])
        elif case["op"] == "attend":
            s["workspace"] = P.alloc_workspace(
                P.attention_workspace_bytes(s["cache"], s["q"].shape[0], case["hq"],
                                            accumulate=case["accumulate"]), k.device)
    return s


# -------------------------------------------------------------------- run ---

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2202_12674_amd as P
    c = s["case"]
    if c["op"] == "rotary":
        return P.rotary(s["x"], s["positions"], s["freqs"], scale=s["factor"],
                        interleaved=c["interleaved"], transpose=c["transpose"])
    if c["op"] == "append":
        P.cache_append(s["cache"], s["new_k"], s["new_v"], s["offsets"], s["positions"],
                       s["freqs"], scale=s["factor"], interleaved=c["interleaved"])
        return s["k"], s["v"]
    if c["op"] == "attend":
        out = P.attention(s["q"], s["cache"], s["offsets"], causal=c["causal"],
                          accumulate=c["accumulate"],
                          weight_out=s["weight_out"] if c["accumulate"] else None,
                          workspace=s["workspace"])
        return (out, s["weight_out"]) if c["accumulate"] else out
    kept = P.cache_evict(s["cache"], s["target"], c["budget"], recent=c["recent"])
    return kept, s["to_lengths"], s["to_k"], s["to_v"], s["to_weight"]


def _turn(x, positions, freqs, factor, interleaved, transpose=False):
    """The rotated x (tokens x heads x d) in 32 bits, angles in 64."""
    t = positions.double()[:, None] * freqs[None, :]
    cos, sin = t.cos().float()[:, None, :] * factor, t.sin().float()[:, None, :] * factor
    if transpose:
        sin = -sin
    n, y = 2 * freqs.numel(), x.float().clone()
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2),
                                                                 slice(n // 2, n))
    p, q = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = p * cos - q * sin, q * cos + p * sin
    return y


def _tokens(s):
    """(sequence, number within it) of every new token."""
    t = torch.arange(s["new_k"].shape[0] if "new_k" in s else s["q"].shape[0], device="cuda")
    offsets = s["offsets"].long()
    seq = torch.searchsorted(offsets, t, right=True) - 1
    return seq, t - offsets[seq]


def _run_plain(s):
    c = s["case"]
    if c["op"] == "rotary":
        return _turn(s["x"], s["positions"], s["freqs"], s["factor"], c["interleaved"],
                     c["transpose"]).to(s["x"].dtype)
    if c["op"] == "append":
        return _append_plain(s)
    return _attend_plain(s) if c["op"] == "attend" else _evict_plain(s)


def _append_plain(s):
    c = s["case"]
    seq, i = _tokens(s)
    offsets = s["offsets"].long()
    j = s["lengths"].long()[seq] - (offsets[1:] - offsets[:-1])[seq] + i
    page, slot = s["table"][seq, j // c["page"]].long(), j % c["page"]
    k = _turn(s["new_k"], s["positions"], s["freqs"], s["factor"], c["interleaved"])
    s["k"][page, :, slot] = k.to(s["k"].dtype)
    s["v"][page, :, slot] = s["new_v"]
    s["weight"][page, :, slot] = 0.0
    return s["k"], s["v"]


def _attend_plain(s):
    c, q = s["case"], s["q"]
    seqs, new, hkv, group, d = c["seqs"], c["new"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    # keys and values of every sequence, padded to the longest (the first page's)
    j = torch.arange(c["length"], device="cuda")
    lengths = s["lengths"].long()[:, None]
    there = j[None, :] < lengths                                        # seqs x keys
    page = torch.where(there, s["table"][:, j // c["page"]].long(), s["table"][:, :1].long())
    slot = torch.where(there, (j % c["page"])[None, :], 0)
    heads = torch.arange(hkv, device="cuda")[None, :, None]
    at = (page[:, None, :], heads, slot[:, None, :])                    # seqs x heads x keys
    K, V = (s[x][at].float().view(seqs * hkv, -1, d) for x in ("k", "v"))
    # rows of every sequence: token by token, the group's heads of each
    seq, i = _tokens(s)
    rows = torch.zeros(seqs, new, hkv, group, d, device="cuda")
    rows[seq, i] = q.float().view(-1, hkv, group, d)
    rows = rows.transpose(1, 2).reshape(seqs * hkv, new * group, d)
    offsets = s["offsets"].long()
    count = (offsets[1:] - offsets[:-1])[:, None]
    last = lengths - 1
    if c["causal"]:
        last = lengths - count + torch.arange(new, device="cuda")[None, :]
    hidden = (j > torch.minimum(last, lengths - 1)[..., None])[:, None, :, None, :]
    p = torch.bmm(rows, K.transpose(1, 2).contiguous()).mul_(d ** -0.5)
    p.view(seqs, hkv, new, group, -1).masked_fill_(hidden, -math.inf)
    p = p.sub_(p.amax(dim=2, keepdim=True)).exp_()
    p.div_(p.sum(dim=2, keepdim=True))
    out = torch.bmm(p, V).view(seqs, hkv, new, group, d)
    out = out.transpose(1, 2)[seq, i].reshape(q.shape).to(q.dtype)
    if not c["accumulate"]:
        return out
    p = p.view(seqs, hkv, new, group, -1)
    p.masked_fill_((torch.arange(new, device="cuda") >= count)[:, None, :, None, None], 0.0)
    gained = s["weight"][at] + p.sum(dim=(2, 3))
    where = there[:, None, :].expand_as(gained)                         # only keys that are there
    flat = ((page[:, None, :] * hkv + heads) * c["page"] + slot[:, None, :])
    spill = s["weight_out"].numel()                                     # the rest behind the end
    to = torch.cat([s["weight_out"].view(-1), s["weight_out"].new_zeros(1)])
    to[torch.where(where, flat, spill)] = gained
    s["weight_out"].copy_(to[:-1].view_as(s["weight_out"]))
    return out, s["weight_out"]


def _evict_plain(s):
    c = s["case"]
    lengths = s["lengths"].long()[:, None]
    j = torch.arange(c["length"], device="cuda")
    there = j[None, :] < lengths
    page = torch.where(there, s["table"][:, j // c["page"]].long(), 0)
    slot = j % c["page"]
    heads = torch.arange(c["hkv"], device="cuda")[None, :, None]
    w = s["weight"][page[:, None, :], heads, slot]                      # seqs x heads x keys
    w = w.masked_fill((there & (j >= lengths - c["recent"]))[:, None, :], math.inf)
    w = w.masked_fill(~there[:, None, :], -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices[:, :, :c["budget"]]
    i = torch.arange(c["budget"], device="cuda")
    left = lengths.clamp(max=c["budget"])                               # kept of each sequence
    kept = (i < left)[:, None, :]
    order = torch.sort(order.masked_fill(~kept, c["length"]), dim=2).values
    # behind the last kept key its copy is written again
    i = torch.minimum(i[None, :], left - 1)
    source = order.gather(2, i[:, None, :].expand_as(order))
    from_page = page[:, None, :].expand(-1, c["hkv"], -1).gather(2, source)
    to_page = s["to_table"].long().gather(1, i // c["page"])[:, None, :]
    for x in ("k", "v", "weight"):
        s["to_" + x][to_page, heads, (i % c["page"])[:, None, :]] = \
            s[x][from_page, heads, source % c["page"]]
    s["to_lengths"].copy_(left[:, 0])
    order = order.masked_fill(~kept, -1).to(torch.int32)
    return order, s["to_lengths"], s["to_k"], s["to_v"], s["to_weight"]


# ------------------------------------------------------------------ exact ---

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turn(s["x"], s, case, case["transpose"])
    if case["op"] == "append":
        k, v, start = s["k"].double(), s["v"].double(), 0
        turned = _exact_turn(s["new_k"], s, case, False)
        for i, (n, L) in enumerate(_batch(case)):
            for first in range((L - n) // case["page"] * case["page"], L, case["page"]):
                a, b = max(first, L - n), min(first + case["page"], L)   # this page's new tokens
                page, t = int(s["table"][i, first // case["page"]]), start + a - (L - n)
                k[page, :, a - first:b - first] = turned[t:t + b - a].transpose(0, 1)
                v[page, :, a - first:b - first] = s["new_v"][t:t + b - a].double().transpose(0, 1)
            start += n
        return k, v
    return _exact_attend(s, case) if case["op"] == "attend" else _exact_evict(s, case)


def _exact_evict(s, case):
    """One head of one sequence at a time: what is heavier than the weight at the
    border, and the first of those as heavy as it."""
    budget, size = case["budget"], case["page"]
    kept = torch.full((case["seqs"], case["hkv"], budget), -1, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(case["seqs"], dtype=torch.int32, device="cuda")
    k, v, w = s["to_k"].double(), s["to_v"].double(), s["to_weight"].double()
    for i, (_, L) in enumerate(_batch(case)):
        pages, n = s["table"][i, :-(-L // size)].long(), min(L, budget)
        to = s["to_table"][i, :-(-n // size)].long()
        recent = min(n, case["recent"])
        lengths[i] = n
        for h in range(case["hkv"]):
            weight = s["weight"][pages, h].reshape(-1)[:L].double()
            keep = torch.zeros(L, dtype=torch.bool, device="cuda")
            keep[L - recent:] = True
            if n > recent:
                old = weight[:L - recent]
                border = torch.kthvalue(old, old.numel() - (n - recent) + 1).values
                over, equal = old > border, old == border
                keep[:L - recent] = over | (equal & (equal.cumsum(0) <= n - recent - over.sum()))
            index = torch.nonzero(keep)[:, 0]
            kept[i, h, :n] = index.int()
            for x, y in ((s["k"], k), (s["v"], v), (s["weight"], w)):
                rows = x[pages, h].flatten(0, 1)[index].double()
                place = y[to, h].flatten(0, 1)
                place[:n] = rows
                y[to, h] = place.view(to.numel(), size, *place.shape[1:])
    return kept, lengths, k, v, w


def _exact_turn(x, s, case, transpose):
    """Each pair as a complex number times factor * exp(i angle)."""
    n = 2 * s["freqs"].numel()
    angle = torch.outer(s["positions"].double(), s["freqs"])[:, None, :]
    if transpose:
        angle = -angle
    y = x.double()
    part = y[..., :n].unflatten(-1, (n // 2, 2) if case["interleaved"] else (2, n // 2))
    pair = part if case["interleaved"] else part.transpose(-1, -2)
    z = torch.view_as_complex(pair.contiguous()) * torch.polar(
        torch.full_like(angle, s["factor"]), angle)
    z = torch.view_as_real(z)
    z = z if case["interleaved"] else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), y[..., n:]], dim=-1)


def _exact_attend(s, case):
    """A block of query rows of one query head at a time, from log sums."""
    group, page = case["hq"] // case["hkv"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    weight = torch.zeros(s["weight"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for i, (n, L) in enumerate(_batch(case)):
        need = -(-L // page)
        pages = s["table"][i, :need].long()
        keep = torch.arange(need * page, device="cuda") < L
        for h in range(case["hq"]):
            K = s["k"][pages, h // group].reshape(need * page, -1)[keep].double()
            V = s["v"][pages, h // group].reshape(need * page, -1)[keep].double()
            total = torch.zeros(need * page, dtype=torch.float64, device="cuda")
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                z = s["q"][start + a:start + b, h].double() @ K.t() / math.sqrt(case["d"])
                if case["causal"]:
                    last = torch.arange(L - n + a, L - n + b, device="cuda")[:, None]
                    z[torch.arange(L, device="cuda")[None, :] > last] = -math.inf
                p = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True))
                out[start + a:start + b, h] = p @ V
                total[keep] += p.sum(dim=0)
            if case["accumulate"]:
                weight[pages, h // group] += total.view(need, page)
        if case["accumulate"]:
            full = torch.zeros(need * page, dtype=torch.bool, device="cuda")
            full[:L] = True
            old = s["weight"][pages].double().transpose(0, 1).reshape(case["hkv"], -1)
            new = weight[pages].transpose(0, 1).reshape(case["hkv"], -1)
            new = torch.where(full, old + new, torch.zeros_like(new))
            weight[pages] = new.view(case["hkv"], need, page).transpose(0, 1)
        start += n
    return (out, weight) if case["accumulate"] else out
