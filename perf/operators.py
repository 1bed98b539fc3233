"""Workloads of the paged cache: attention over pages for a batch that shares a long prefix, and the pages' own
operations (rows kept by a compaction, forks with their copies on write, freeing).

Every operator is here twice: in plain torch operations in 32 bits (``own`` false), and as the calls that a user makes
of ``paper_2601_07667_b200.binding`` (``own`` true).  ``exact`` is attention in 64 bits, sequence by sequence.

A cache holds, for every layer, pages of ``page`` tokens [n_pages][H_k][page][d]; a slot's row of the table names its
pages, ``len`` its tokens, ``refs`` counts the slots that hold a page.
"""
import math
import random

import torch

own = False

D = 128
HEADS = ((8, 2), (32, 8), (64, 8), (28, 4), (16, 16), (32, 1))


# ---- cases ----------------------------------------------------------------------------------------
def _attend(name, heads, prefix, groups, seqs, suffix, page, q_tokens=1, layers=1, keys="bf16"):
    return {**({"name": name} if name else {}), "op": "attend", "q_heads": heads[0], "kv_heads": heads[1], "prefix": prefix,
            "groups": groups, "seqs": seqs, "suffix": suffix, "page": page, "q_tokens": q_tokens, "layers": layers, "keys": keys}


def _store(name, kv_heads, tokens, requests, keep, page, layers, keys="bf16"):
    return {**({"name": name} if name else {}), "op": "store", "kv_heads": kv_heads, "tokens": tokens, "requests": requests,
            "keep": keep, "page": page, "layers": layers, "keys": keys}


def _prune(name, kv_heads, tokens, requests, keep, page, layers, keys="bf16"):
    return {**_store(name, kv_heads, tokens, requests, keep, page, layers, keys), "op": "prune"}


def _round(name, kv_heads, prefix, groups, children, grow, page, layers, keys="bf16"):
    return {**({"name": name} if name else {}), "op": "round", "kv_heads": kv_heads, "prefix": prefix, "groups": groups,
            "children": children, "grow": grow, "page": page, "layers": layers, "keys": keys}


def listed():
    return [
        # four samples of a short pruned prompt on the small head layout: what a single token costs at the least
        _attend("attend_small_512", (8, 2), 512, 1, 4, 16, 16),
        # the layers of one decoding step, 32 samples of a prompt pruned to a budget of 2048
        _attend("attend_8b_2k", (32, 8), 2048, 1, 32, 400, 64, layers=4),
        # a whole prompt of 128K tokens that is not pruned, 48 questions about it; its last page is half full
        _attend("attend_8b_128k", (32, 8), 130999, 1, 48, 700, 64),
        # many samples on wide groups: more than a thousand rows share every key, the arithmetic counts
        _attend("attend_wide_64k", (64, 8), 65536, 1, 130, 300, 128),
        # drafts of five tokens to be checked, four sequences on each of six prompts of odd lengths
        _attend("attend_drafts_8k", (32, 8), 8011, 6, 4, 900, 32, q_tokens=5, layers=2),
        # a quantised (E4M3) key cache, seven queries per head
        _attend("attend_7b_fp8_48k", (28, 4), 49999, 1, 24, 333, 64, keys="fp8"),
        # ordinary decoding after pruning: nothing is shared
        _attend("attend_alone_4k", (32, 8), 4096, 24, 1, 500, 64),
        # half of every prompt's rows, per head, from the prefill's K and V into pages
        _store("store_half_24k", 8, 24001, 4, 0.5, 64, 1),
        # the same for a short prompt and four layers
        _store("store_small_4k", 2, 4096, 1, 0.125, 16, 4),
        # cached prompts pruned again, from their pages into fewer
        _prune("prune_32k", 8, 32768, 2, 0.0625, 64, 8),
        # a round of sampling: children fork from prompts, grow, and are freed; the half full page is copied on write
        _round("round_8b_2k", 8, 2023, 2, 32, 24, 64, 8),
        # one token for each of a few children on small pages, a thousand pages in the pool
        _round("round_small", 2, 519, 1, 4, 1, 16, 1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("attend",) * 5 + ("store", "prune", "round", "round"))
    page, keys = rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "bf16", "fp8"))
    if op == "attend":
        heads = rng.choice(HEADS)
        groups = rng.choice((1, 1, 1, 2, 5, 16))
        return _attend(None, heads, _log_int(rng, 60, 131072), groups, _log_int(rng, 1, 128), _log_int(rng, 1, 1500), page,
                       rng.choice((1, 1, 1, 2, 5, 8)), rng.choice((1, 1, 2, 4)), keys)
    kv_heads = rng.choice((1, 2, 4, 8))
    if op == "round":
        return _round(None, kv_heads, _log_int(rng, 20, 8192), rng.choice((1, 2, 4)), _log_int(rng, 1, 64), _log_int(rng, 1, 200),
                      page, rng.choice((1, 2, 8)), keys)
    make = _store if op == "store" else _prune
    return make(None, kv_heads, _log_int(rng, 500, 65536), rng.choice((1, 2, 4)), round(math.exp(rng.uniform(math.log(0.02), math.log(0.6))), 4),
                page, rng.choice((1, 2, 4)), keys)


def _plain_scores(c):
    """Logits that the plain form of an attention case holds at once."""
    if c["op"] != "attend":
        return 0
    return c["layers"] * c["q_heads"] * c["groups"] * c["seqs"] * c["q_tokens"] * _pool_pages(c) * c["page"]


def draw(rng):
    """One more case of the ranges the listed ones stand for, no larger than the largest of them."""
    cost = lambda c: (lambda w: max(w["bytes"], w["flops"] / 250.0))(work(c))  # noqa: E731
    most, logits = max(cost(c) for c in listed()), max(_plain_scores(c) for c in listed())
    while True:
        c = _draw_one(rng)
        if cost(c) <= most and _plain_scores(c) <= logits:
            return c


# ---- shapes ---------------------------------------------------------------------------------------
def _prefixes(c):
    """Tokens of every group's prompt: ragged where there are several."""
    r = random.Random(c["prefix"] * 31 + c["groups"])
    return [c["prefix"] if c["groups"] == 1 else r.randint(max(1, c["prefix"] // 4), c["prefix"]) for _ in range(c["groups"])]


def _suffixes(c):
    """Tokens that every sequence has of its own behind its prompt, the queries' among them."""
    r = random.Random(c["suffix"] * 17 + c["seqs"])
    return [[max(c["q_tokens"], _log_int(r, 1, c["suffix"])) for _ in range(c["seqs"])] for _ in range(c["groups"])]


def _pages_of(tokens, page):
    return -(-tokens // page)


def _attend_pages(c):
    """(pages that a group shares, pages of all its sequences' own) for every group."""
    got = []
    for p, tails in zip(_prefixes(c), _suffixes(c)):
        shared = p // c["page"] if c["seqs"] > 1 else 0
        got.append((shared, sum(_pages_of(p + s, c["page"]) - shared for s in tails)))
    return got


def _lengths(c):
    if c["requests"] == 1:
        return [c["tokens"]]
    r = random.Random(c["tokens"] * 31 + c["requests"])
    return [r.randint(max(64, c["tokens"] // 3), c["tokens"]) for _ in range(c["requests"])]


def _kept(c):
    return [max(32, min(n, int(n * c["keep"]))) for n in _lengths(c)]


def _pool_pages(c):
    page = c["page"]
    if c["op"] == "attend":
        return sum(a + b for a, b in _attend_pages(c)) + 3
    if c["op"] == "store":
        return sum(_pages_of(m, page) for m in _kept(c)) + 5
    if c["op"] == "prune":
        return sum(_pages_of(n, page) + _pages_of(m, page) for n, m in zip(_lengths(c), _kept(c))) + 5
    per = sum(_pages_of(p, page) for p in _prefixes(c)) + c["groups"] * c["children"] * (2 + _pages_of(c["grow"], page))
    return max(per + 7, 1024 // max(1, c["layers"] * c["kv_heads"] // 2))


def work(case):
    """Bytes and operations of one pass: what is cached, once (a shared prefix once for its group), queries and results once;
    rows and pages that are copied read and written once, with the lists and counts that say which."""
    c, page, kb = case, case["page"], 1 if case["keys"] == "fp8" else 2
    row = c["kv_heads"] * D * (kb + 2)
    if c["op"] == "attend":
        keys = pairs = 0
        for p, tails in zip(_prefixes(c), _suffixes(c)):
            shared = p // page * page if c["seqs"] > 1 else 0
            keys += shared + sum(p + s - shared for s in tails)
            pairs += c["q_tokens"] * sum(p + s - (c["q_tokens"] - 1) / 2.0 for s in tails)
        tokens = c["groups"] * c["seqs"] * c["q_tokens"]
        return {"bytes": c["layers"] * (keys * row + tokens * c["q_heads"] * (4 * D + 4)) + 4 * _pool_pages(c),
                "flops": c["layers"] * 4.0 * D * c["q_heads"] * pairs}
    if c["op"] in ("store", "prune"):
        m = sum(_kept(c))
        return {"bytes": c["layers"] * m * (2 * row + 4 * c["kv_heads"]) + 4 * _pool_pages(c), "flops": 0}
    copies = sum(c["children"] for p in _prefixes(c) if p % page)
    rest = sum(c["children"] * (p % page) for p in _prefixes(c))          # tokens on the pages that are copied
    grown = c["groups"] * c["children"] * c["grow"]
    return {"bytes": c["layers"] * 2 * row * (rest + grown) + 4 * _pool_pages(c) + 4 * copies, "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _rows(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pool(c, g, n_pages, slots, max_pages):
    """A cache's buffers: random rows everywhere, an empty table."""
    L, Hk, page = c["layers"], c["kv_heads"], c["page"]
    s = {"case": c, "k": _rows(g, L, n_pages, Hk, page, D), "v": _rows(g, L, n_pages, Hk, page, D),
         "table": torch.zeros((slots, max_pages), dtype=torch.int32, device="cuda"),
         "len": torch.zeros(slots, dtype=torch.int32, device="cuda"), "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
         "k_scale": None}
    return s


def _quantise(c, s):
    """E4M3 codes of the pool's keys and a scale for each layer's kv head (the head's largest magnitude is 448)."""
    if c["keys"] == "fp8":
        most = torch.maximum(s["k"].amax(dim=(1, 3, 4)), -s["k"].amin(dim=(1, 3, 4))).float()          # [L][H_k]
        s["k_scale"] = (most / 448.0).contiguous()
        s["k"] = torch.stack([_codes(x, sc) for x, sc in zip(s["k"], s["k_scale"])])


def _codes(x, scale):
    """[..][H_k][page][d] rows as codes of the heads' scales."""
    return (x.float() / scale[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _prepare_attend(c, seed):
    g, r = _generator(seed), random.Random(seed)
    L, Hq, Hk, page, nq = c["layers"], c["q_heads"], c["kv_heads"], c["page"], c["q_tokens"]
    n_pages, ids = _pool_pages(c), list(range(_pool_pages(c)))
    r.shuffle(ids)
    rows, lens, refs, of_group, at = [], [], [0] * n_pages, [], 0
    first = []                                                     # a group's shared pages
    for i, (p, tails) in enumerate(zip(_prefixes(c), _suffixes(c))):
        shared = p // page if c["seqs"] > 1 else 0
        head = ids[at:at + shared]
        at += shared
        first.append(head or None)
        for t in tails:
            m = _pages_of(p + t, page) - shared
            rows.append(head + ids[at:at + m])
            at += m
            lens.append(p + t)
            of_group.append(i)
    for row in rows:
        for x in row:
            refs[x] += 1
    most = max(len(x) for x in rows) + 1
    n = len(rows)
    s = _pool(c, g, n_pages, n + 1, most)
    order = list(range(n + 1))[1:]                                 # slot 0 stays free; sequences in the order of their groups
    s["table"][1:] = _int([row + [0] * (most - len(row)) for row in rows])
    s["len"][1:] = _int(lens)
    s["refs"] = _int(refs)
    s["slots"], s["cu_q"] = _int(order), _int([i * nq for i in range(n + 1)])
    # queries lean towards a direction of their group and head; a few keys of the prompt lie far along it
    u = torch.randn((c["groups"], L, Hk, D), generator=g, device="cuda")
    u = u / u.norm(dim=-1, keepdim=True)
    for i, row in enumerate(rows):
        if i == 0 or of_group[i] != of_group[i - 1]:
            for j in range(8):
                x = row[(j * 997) % max(1, lens[i] // page)]
                s["k"][:, x, :, (j * 5) % page] = (3.0 * math.sqrt(D) * u[of_group[i]]).to(torch.bfloat16)
    lean = math.sqrt(D / 3.0) * u[torch.tensor(of_group, device="cuda")]             # [n][L][H_k][d]
    lean = lean.transpose(0, 1).repeat_interleave(Hq // Hk, dim=2).repeat_interleave(nq, dim=1)
    s["q"] = (torch.randn((L, n * nq, Hq, D), generator=g, device="cuda") + lean).to(torch.bfloat16)
    _quantise(c, s)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((L, n * nq, Hq), dtype=torch.float32, device="cuda")
    return s


def _keep_lists(g, L, Hk, lengths, kept):
    """Ascending token indices per layer and head, every request's behind one another: [L][H_k][sum kept]."""
    parts = []
    for n, m in zip(lengths, kept):
        x = torch.rand((L, Hk, n), generator=g, device="cuda").topk(m, dim=-1).indices
        parts.append(x.sort(dim=-1).values.to(torch.int32))
    return torch.cat(parts, dim=-1).contiguous()


def _prepare_store(c, seed):
    g = _generator(seed)
    lengths, kept = _lengths(c), _kept(c)
    B, page, L, Hk = len(lengths), c["page"], c["layers"], c["kv_heads"]
    s = _pool(c, g, _pool_pages(c), B, _pages_of(max(kept), page))
    s["k"].zero_(), s["v"].zero_()
    if c["keys"] == "fp8":
        s["k"], s["k_scale"] = s["k"].view(torch.uint8)[..., :D].contiguous(), torch.ones((L, Hk), device="cuda")
    src = _rows(g, L, sum(lengths), Hk, D)
    s["src_k"] = src if c["keys"] != "fp8" else (src.float() * 40.0).to(torch.float8_e4m3fn).view(torch.uint8)
    s["src_v"] = _rows(g, L, sum(lengths), Hk, D)
    s["idx"], s["slots"] = _keep_lists(g, L, Hk, lengths, kept), _int(list(range(B))[::-1])
    s["none"], s["want"] = _int([0] * B), _int(kept[::-1])
    s["cu"], s["off"] = _int(_cum(lengths)), _int(_cum(kept))
    s["host"] = {"lengths": lengths, "kept": kept}
    return s


def _prepare_prune(c, seed):
    g, r = _generator(seed), random.Random(seed)
    lengths, kept = _lengths(c), _kept(c)
    B, page = len(lengths), c["page"]
    n_pages = _pool_pages(c)
    s = _pool(c, g, n_pages, 2 * B, _pages_of(max(lengths), page))
    ids = list(range(n_pages))
    r.shuffle(ids)
    refs, at, rows = [0] * n_pages, 0, []
    for n in lengths:
        m = _pages_of(n, page)
        rows.append(ids[at:at + m] + [0] * (s["table"].shape[1] - m))
        for x in ids[at:at + m]:
            refs[x] = 1
        at += m
    s["table"][:B], s["len"][:B], s["refs"] = _int(rows), _int(lengths), _int(refs)
    _quantise(c, s)
    s["idx"] = _keep_lists(g, c["layers"], c["kv_heads"], lengths, kept)
    s["src"], s["dst"], s["off"] = _int(list(range(B))), _int(list(range(B, 2 * B))), _int(_cum(kept))
    s["none"], s["want"] = _int([-1] * B + [0] * B), _int([-1] * B + kept)
    s["host"] = {"kept": kept}
    return s


def _prepare_round(c, seed):
    g, r = _generator(seed), random.Random(seed)
    prefixes, page, nc = _prefixes(c), c["page"], c["children"]
    P, n_pages = len(prefixes), _pool_pages(c)
    s = _pool(c, g, n_pages, P + P * nc, _pages_of(max(prefixes) + c["grow"], page))
    ids = list(range(n_pages))
    r.shuffle(ids)
    refs, at, rows = [0] * n_pages, 0, []
    for p in prefixes:
        m = _pages_of(p, page)
        rows.append(ids[at:at + m] + [0] * (s["table"].shape[1] - m))
        for x in ids[at:at + m]:
            refs[x] = 1
        at += m
    s["table"][:P], s["len"][:P], s["refs"] = _int(rows), _int(prefixes), _int(refs)
    _quantise(c, s)
    parent = [i for i in range(P) for _ in range(nc)]
    n = len(parent)
    s["parent"] = _int([-1] * P + parent)
    s["want"] = _int([-1] * P + [prefixes[p] + c["grow"] for p in parent])
    s["free"] = _int([-1] * P + [0] * n)
    s["slots"], s["cu_q"] = _int(list(range(P, P + n))), _int([i * c["grow"] for i in range(n + 1)])
    new = _rows(g, c["layers"], n * c["grow"], c["kv_heads"], D)
    s["new_k"] = new if c["keys"] != "fp8" else torch.stack(
        [(x.float() / sc[:, None]).to(torch.float8_e4m3fn).view(torch.uint8) for x, sc in zip(new, s["k_scale"])])
    s["new_v"] = _rows(g, c["layers"], n * c["grow"], c["kv_heads"], D)
    return s


def _cum(x):
    got = [0]
    for v in x:
        got.append(got[-1] + v)
    return got


def prepare(case, seed):
    s = {"attend": _prepare_attend, "store": _prepare_store, "prune": _prepare_prune, "round": _prepare_round}[case["op"]](case, seed)
    s["handle"] = _handle(s) if own else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------
def _keys32(s):
    """The pool's keys as the values they stand for, [L][H_k][n_pages * page][d] in 32 bits."""
    k = s["k"]
    if s["k_scale"] is not None:
        k = k.view(torch.float8_e4m3fn).float() * s["k_scale"][:, None, :, None, None]
    return k.float().transpose(1, 2).flatten(2, 3)


def _attend_plain(s):
    c = s["case"]
    L, Hk, page, nq = c["layers"], c["kv_heads"], c["page"], c["q_tokens"]
    G, n_pages = c["q_heads"] // Hk, s["refs"].shape[0]
    slots = s["slots"].long()
    lens, table = s["len"][slots].long(), s["table"][slots].long()
    # where a page of the pool stands in each sequence (-1: nowhere); column n_pages takes what lies behind a sequence's end
    j = torch.arange(table.shape[1], device="cuda")
    place = torch.full((table.shape[0], n_pages + 1), -1, dtype=torch.long, device="cuda")
    place.scatter_(1, torch.where(j * page < lens[:, None], table, n_pages), j.expand_as(table))
    place = place[:, :n_pages, None]
    at = torch.where(place >= 0, place * page + torch.arange(page, device="cuda"), -1).flatten(1)          # [n][pool tokens]
    pos = (lens[:, None] - nq + torch.arange(nq, device="cuda")).flatten()                                  # of every query token
    seen = at.repeat_interleave(nq, dim=0)
    seen = ((seen >= 0) & (seen <= pos[:, None])).repeat_interleave(G, dim=0)                               # [tokens * G][pool tokens]
    q = s["q"].float().unflatten(2, (Hk, G)).transpose(1, 2).flatten(2, 3)                                  # [L][H_k][tokens * G][d]
    x = (q @ _keys32(s).transpose(-1, -2)).mul_(1.0 / math.sqrt(D))
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    e = x.sub_(top).exp_()
    total = e.sum(dim=-1, keepdim=True)
    out = (e @ s["v"].float().transpose(1, 2).flatten(2, 3)) / total
    lse = top + torch.log(total)
    back = lambda y: y.unflatten(2, (-1, G)).transpose(1, 2).flatten(2, 3)                                  # noqa: E731
    s["out"].copy_(back(out))
    s["lse"].copy_(back(lse)[..., 0])
    return s["out"], s["lse"]


def _reserve_plain(s, want):
    """Slots grow to `want` tokens: the lowest free pages, slot after slot; of a shared page that is half full the tokens are copied first."""
    page, table, n = s["case"]["page"], s["table"], s["len"]
    free = torch.argsort((s["refs"] != 0).to(torch.int32), stable=True)
    j = torch.arange(table.shape[1], device="cuda")
    have, grows = (n + page - 1) // page, want > n
    last = table.gather(1, (n // page).clamp(max=table.shape[1] - 1).long()[:, None])[:, 0].long()
    own_page = grows & (n % page != 0) & (s["refs"][last] > 1)
    fresh = grows[:, None] & (j >= have[:, None]) & (j < ((want + page - 1) // page)[:, None])
    fresh |= own_page[:, None] & (j == (n // page)[:, None])
    ids = free[(torch.cumsum(fresh.flatten(), 0) - 1).clamp(min=0).unflatten(0, fresh.shape)]
    s["refs"].index_add_(0, last[own_page], torch.full_like(last[own_page], -1, dtype=torch.int32))
    table[fresh] = ids[fresh].to(torch.int32)
    s["refs"][ids[fresh]] = 1
    new = table.gather(1, (n // page).clamp(max=table.shape[1] - 1).long()[:, None])[:, 0].long()
    held = (torch.arange(page, device="cuda") < (n % page)[own_page][:, None])[None, :, None, :, None]
    for pool in (s["k"], s["v"]):
        pool[:, new[own_page]] = torch.where(held, pool[:, last[own_page]], pool[:, new[own_page]])
    n.copy_(torch.where(grows, want, n))


def _trim_plain(s, to):
    page, table, n = s["case"]["page"], s["table"], s["len"]
    j = torch.arange(table.shape[1], device="cuda")
    cut = (to >= 0) & (to < n)
    gone = cut[:, None] & (j >= ((to + page - 1) // page)[:, None]) & (j < ((n + page - 1) // page)[:, None])
    gone = table[gone].long()
    s["refs"].index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    n.copy_(torch.where(cut, to, n))


def _fork_plain(s, parent):
    page, table, n = s["case"]["page"], s["table"], s["len"]
    j = torch.arange(table.shape[1], device="cuda")
    child, of = parent >= 0, parent.clamp(min=0).long()
    held = child[:, None] & (j < ((n[of] + page - 1) // page)[:, None])
    ids = table[of][held]
    table[held] = ids
    s["refs"].index_add_(0, ids.long(), torch.ones_like(ids))
    n.copy_(torch.where(child, n[of], n))


def _put(s, slot, pos, k, v):
    """Rows k, v [L][rows][H_k][d] (pos and slot [rows]) to their places in the pages."""
    page = s["case"]["page"]
    at = s["table"][slot.long(), (pos // page).long()].long()
    s["k"][:, at, :, (pos % page).long()] = k.transpose(0, 1)
    s["v"][:, at, :, (pos % page).long()] = v.transpose(0, 1)


def _store_plain(s):
    _trim_plain(s, s["none"])
    _reserve_plain(s, s["want"])
    off, n = s["off"].long(), s["idx"].shape[-1]
    r = torch.arange(n, device="cuda")
    b = torch.bucketize(r, off[1:], right=True)
    rows = (s["idx"].long() + s["cu"].long()[b])[..., None].expand(-1, -1, -1, D).transpose(1, 2)
    _put(s, s["slots"][b], r - off[b], torch.gather(s["src_k"], 1, rows), torch.gather(s["src_v"], 1, rows))
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


def _prune_plain(s):
    page = s["case"]["page"]
    _trim_plain(s, s["none"])
    _reserve_plain(s, s["want"])
    off, n = s["off"].long(), s["idx"].shape[-1]
    r = torch.arange(n, device="cuda")
    b = torch.bucketize(r, off[1:], right=True)
    idx = s["idx"].long().transpose(1, 2)                                                    # [L][rows][H_k]
    at = s["table"][s["src"][b].long()[:, None], idx // page].long()                         # [L][rows][H_k]
    layer = torch.arange(idx.shape[0], device="cuda")[:, None, None]
    head = torch.arange(idx.shape[2], device="cuda")
    _put(s, s["dst"][b], r - off[b], s["k"][layer, at, head, idx % page], s["v"][layer, at, head, idx % page])
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


def _round_plain(s):
    grow = s["case"]["grow"]
    _fork_plain(s, s["parent"])
    _reserve_plain(s, s["want"])
    slot = s["slots"].repeat_interleave(grow)
    pos = s["len"][s["slots"].long()].repeat_interleave(grow) - grow + torch.arange(grow, device="cuda").repeat(s["slots"].shape[0])
    _put(s, slot, pos, s["new_k"], s["new_v"])
    _trim_plain(s, s["free"])
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


# ---- the framework's calls ------------------------------------------------------------------------
def _handle(s):
    """What a user's program keeps: the cache over its buffers, the batch's descriptor, the prefill's plan."""
    from paper_2601_07667_b200 import binding as B
    c = s["case"]
    cache = B.PagedCache(page_size=c["page"], k=s["k"], v=s["v"], table=s["table"], length=s["len"], refs=s["refs"], k_scale=s["k_scale"])
    h = {"cache": cache}
    if c["op"] == "attend":
        h["batch"] = cache.batch(s["slots"], s["cu_q"], n_tokens=s["q"].shape[1], n_q_heads=c["q_heads"])
    if c["op"] == "round":
        h["batch"] = cache.batch(s["slots"], s["cu_q"], n_tokens=s["new_v"].shape[1])
    if c["op"] == "store":
        h["path"] = B.LayerPath(n_q_heads=c["kv_heads"], n_kv_heads=c["kv_heads"], head_dim=D, window=32, pool_kernel=7,
                                pool_mode=B.ASL_POOL_AVG, seqlens=s["host"]["lengths"], budgets=s["host"]["kept"], l_min=1, l_obs=2, tau=0.3,
                                k_dtype=B.ASL_K_FP8_E4M3 if c["keys"] == "fp8" else B.ASL_K_BF16,
                                k_scale=[1.0] * c["kv_heads"] if c["keys"] == "fp8" else None)
    return h


def _attend_own(s):
    cache, batch = s["handle"]["cache"], s["handle"]["batch"]
    cache.plan(batch)
    for layer in range(s["case"]["layers"]):
        cache.attend(layer, batch, s["q"][layer], s["out"][layer], s["lse"][layer])
    return s["out"], s["lse"]


def _store_own(s):
    cache, path = s["handle"]["cache"], s["handle"]["path"]
    cache.trim(s["none"])
    cache.reserve(s["want"])
    for layer in range(s["case"]["layers"]):
        cache.store(layer, path, s["src_k"][layer], s["src_v"][layer], s["idx"][layer], s["slots"])
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


def _prune_own(s):
    cache = s["handle"]["cache"]
    cache.trim(s["none"])
    cache.reserve(s["want"])
    for layer in range(s["case"]["layers"]):
        cache.compact(layer, s["src"], s["dst"], s["off"], s["idx"][layer], max_kept=max(s["host"]["kept"]))
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


def _round_own(s):
    cache, batch = s["handle"]["cache"], s["handle"]["batch"]
    cache.fork(s["parent"])
    cache.reserve(s["want"])
    for layer in range(s["case"]["layers"]):
        cache.append(layer, batch, s["new_k"][layer], s["new_v"][layer])
    cache.trim(s["free"])
    return s["k"], s["v"], s["table"], s["len"], s["refs"]


def run(state):
    """One pass: a decoding step's attention (its plan and every layer), or a round of the pages' operations that ends in
    the state it began with."""
    op = state["case"]["op"]
    if own:
        return {"attend": _attend_own, "store": _store_own, "prune": _prune_own, "round": _round_own}[op](state)
    return {"attend": _attend_plain, "store": _store_plain, "prune": _prune_plain, "round": _round_plain}[op](state)


# ---- the definition in 64 bits --------------------------------------------------------------------
def exact(case, seed):
    """Attention of every sequence over its own tokens in 64 bits; the other operators copy rows and count."""
    if case["op"] != "attend":
        return None
    s = prepare(case, seed)
    page, nq, Hk = case["page"], case["q_tokens"], case["kv_heads"]
    G = case["q_heads"] // Hk
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    table, lens = s["table"].tolist(), s["len"].tolist()
    for i, slot in enumerate(s["slots"].tolist()):
        n = lens[slot]
        ids = torch.tensor(table[slot][:_pages_of(n, page)], device="cuda")
        for layer in range(case["layers"]):
            for h in range(Hk):
                k, v = s["k"][layer, ids, h], s["v"][layer, ids, h].double().reshape(-1, D)[:n]
                k = k.double() if s["k_scale"] is None else k.view(torch.float8_e4m3fn).double() * s["k_scale"][layer, h].double()
                k = k.reshape(-1, D)[:n]
                q = s["q"][layer, i * nq:(i + 1) * nq, h * G:(h + 1) * G].double()
                x = torch.einsum("tgd,nd->tgn", q, k) / math.sqrt(D)
                for t in range(nq):
                    y = x[t, :, :n - nq + t + 1]
                    z = torch.logsumexp(y, dim=-1, keepdim=True)
                    out[layer, i * nq + t, h * G:(h + 1) * G] = torch.exp(y - z) @ v[:n - nq + t + 1]
                    lse[layer, i * nq + t, h * G:(h + 1) * G] = z[:, 0]
    return out, lse
