"""Operators of beam search and of long contexts over the paged int8 cache, measured one at a time.

A serving program that searches with beams picks the best continuations of each sequence, forks the page tables of the beams that
go on (full pages are shared, a page that two beams would write is copied), releases what nobody holds, and now and then moves the
pages together; where contexts are long, a bound of the keys of each page says which pages a query has to read.  Five kinds of case:

  beam     logits [batch x beams, vocabulary] and the beams' scores -> the best (score, beam, token) of each sequence
  fork     page tables of the beams that go on, with room for their next tokens, and the pages that have to be copied, copied
  compact  the pages in use moved to the front of the cache
  bounds   for the pages that new tokens filled, the largest and smallest key in each channel, in 8 bits
  sparse   new tokens against the pages whose bounds promise most (the first and the last ones among them)
"""
import math

import torch

own = False

FP16, BF16, FP32 = "fp16", "bf16", "fp32"
TYPES = {FP16: torch.float16, BF16: torch.bfloat16, FP32: torch.float32}
INF = math.inf


def _beam(name, batch, beams, vocab, keep, dtype):
    return {"name": name, "kind": "beam", "batch": batch, "beams": beams, "vocab": vocab, "keep": keep, "dtype": dtype}


def _fork(name, batch, beams, shortest, longest, grown, kv_heads, dim, page, new):
    """Prompts of shortest to longest tokens that a sequence's beams share, then `grown` tokens of each beam's own."""
    return {"name": name, "kind": "fork", "batch": batch, "beams": beams, "shortest": shortest, "longest": longest, "grown": grown,
            "kv_heads": kv_heads, "dim": dim, "page": page, "new": new}


def _compact(name, pages, used, rows, kv_heads, dim, page):
    """`used` of `pages` pages are held, at random places, by `rows` sequences."""
    return {"name": name, "kind": "compact", "pages": pages, "used": used, "rows": rows, "kv_heads": kv_heads, "dim": dim, "page": page}


def _bounds(name, batch, shortest, longest, kv_heads, dim, page, new):
    return {"name": name, "kind": "bounds", "batch": batch, "shortest": shortest, "longest": longest, "kv_heads": kv_heads, "dim": dim, "page": page, "new": new}


def _sparse(name, batch, shortest, longest, heads, kv_heads, dim, page, keep, dtype, new=1):
    """keep: pages that a key head's queries read, the first and the last `recent` among them (new tokens touch no others)."""
    return {"name": name, "kind": "sparse", "batch": batch, "shortest": shortest, "longest": longest, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page": page, "keep": keep, "recent": (new + page - 2) // page + 1, "dtype": dtype, "new": new}


def listed():
    return [
        # one user, four beams, the vocabulary of a BERT-base checkpoint: latency
        _beam("beam 1x4x21128", 1, 4, 21128, 4, FP16),
        # an odd batch and an odd vocabulary, twice as many candidates as beams (some of them may end); logits added up in 32 bits
        _beam("beam 7x5x50265", 7, 5, 50265, 10, FP32),
        # a loaded server with a large vocabulary
        _beam("beam 64x8x128256", 64, 8, 128256, 16, BF16),
        # a decode step of one user's beams: latency
        _fork("fork 1x4", 1, 4, 150, 150, 41, 12, 64, 16, 1),
        # a decode step of a loaded server: 256 beams, prompts up to 1500 tokens, 300 tokens on
        _fork("fork 32x8", 32, 8, 200, 1500, 300, 8, 128, 64, 1),
        # a small cache
        _compact("compact 301 pages", 301, 170, 6, 12, 64, 16),
        # half a gigabyte of pages, in use at random places
        _compact("compact 4096 pages", 4096, 2458, 60, 8, 128, 64),
        # a few tokens on for each of some sequences: few pages become full
        _bounds("bounds 5x3", 5, 200, 1003, 12, 64, 16, 3),
        # prompts that have just been written
        _bounds("bounds prompts 16x8192", 16, 2000, 8192, 8, 128, 64, 8192),
        # a decode step of one long document: latency
        _sparse("sparse 1x100000", 1, 100000, 100000, 32, 8, 128, 64, 32, FP16),
        # drafted tokens of a few sequences, a head of its own for each query head
        _sparse("sparse 6x5 drafts", 6, 150, 5001, 12, 12, 64, 32, 20, FP16, new=5),
        # the decode step of a loaded server with long contexts, some of them shorter than what is kept
        _sparse("sparse 64x32768", 64, 900, 32768, 32, 8, 128, 64, 32, BF16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges that costs no more than the largest of its kind."""
    while True:
        kind = rng.choice(("beam", "fork", "compact", "bounds", "sparse"))
        dim, kv, page = rng.choice((64, 128)), rng.choice((1, 2, 4, 8, 12)), rng.choice((16, 32, 64, 128))
        if kind == "beam":
            beams = rng.choice((1, 2, 3, 4, 5, 8, 16))
            c = _beam("", _log(rng, 1, 64), beams, _log(rng, 1000, 152000), beams * rng.choice((1, 2)), rng.choice((FP16, BF16, FP32)))
        elif kind == "fork":
            longest = _log(rng, 20, 4000)
            c = _fork("", _log(rng, 1, 64), rng.choice((1, 2, 4, 5, 8)), max(1, int(longest * rng.random())), longest, _log(rng, 1, 600), kv, dim, page,
                      rng.choice((1, 1, 1, 4, 20)))
        elif kind == "compact":
            pages = _log(rng, 40, 16384)
            c = _compact("", pages, max(1, int(pages * rng.uniform(0.1, 0.9))), _log(rng, 1, 100), kv, dim, page)
        else:
            batch, longest = _log(rng, 1, 64), _log(rng, 100, 120000)
            shortest = max(1, int(longest * rng.random()))
            if kind == "bounds":
                c = _bounds("", batch, shortest, longest, kv, dim, page, _log(rng, 1, longest))
            else:
                c = _sparse("", batch, shortest, longest, kv * rng.choice((1, 2, 4, 7, 8)), kv, dim, page, _log(rng, 8, 100), rng.choice((FP16, BF16)),
                            rng.choice((1, 1, 1, 2, 5, 8)))
        del c["name"]
        if _cost(c) > max(_cost(x) for x in listed() if x["kind"] == kind) or c.get("heads", 1) > 64:
            continue
        if kind != "bounds" or _full_pages(c):                        # (tokens that fill no page leave nothing to do)
            return c


def _spread(lo, hi, n):
    return [hi] if n == 1 else [lo + round((hi - lo) * i / (n - 1)) for i in range(n)]


def _lengths(case):
    return _spread(case["shortest"], case["longest"], case["batch"])


def _ended(case):
    """The sequences of a fork that have come to their end: their beams are released."""
    return [g for g in range(case["batch"]) if g % 16 == 15]


def _fork_sizes(case):
    """Pages that the beams of each sequence share, pages of a beam alone, the table's width, and the cache's pages."""
    L = _lengths(case)
    page, beams = case["page"], case["beams"]
    shared = [n // page for n in L]
    alone = [-(-(n + case["grown"]) // page) - s for n, s in zip(L, shared)]
    width = max(s + a for s, a in zip(shared, alone)) + -(-case["new"] // page) + 3
    held = sum(s + beams * a for s, a in zip(shared, alone))
    return shared, alone, width, held + held // 8 + case["batch"] * beams * (1 + -(-case["new"] // page))


def _full_pages(case):
    return sum(n // case["page"] - (n - min(n, case["new"])) // case["page"] for n in _lengths(case))


def work(case):
    if case["kind"] == "beam":
        n = case["batch"] * case["beams"]
        size = 4 if case["dtype"] == FP32 else 2
        return {"bytes": float(n) * case["vocab"] * size + 4.0 * n + 12.0 * case["batch"] * case["keep"], "flops": 4.0 * n * case["vocab"]}
    G, D, page = case["kv_heads"], case["dim"], case["page"]
    token = 2.0 * G * (D + 4)                                         # a token's keys and values in the cache
    if case["kind"] == "fork":
        _, _, width, pages = _fork_sizes(case)
        W, rows = case["beams"], case["batch"] * case["beams"]
        again = W * (1 - 1 / W) ** W                                  # beams of a sequence that are not the first child of theirs, on average
        held = [(n + case["grown"]) % page for g, n in enumerate(_lengths(case)) if g not in _ended(case)]
        return {"bytes": 8.0 * rows * width + 8.0 * pages + 24.0 * rows + 2 * token * again * sum(held), "flops": 1.0 * rows * width}
    if case["kind"] == "compact":
        moved = case["used"] * (case["pages"] - case["used"]) / case["pages"]
        return {"bytes": 8.0 * case["pages"] + 8.0 * case["used"] + 2 * moved * page * token, "flops": 1.0 * case["pages"]}
    if case["kind"] == "bounds":
        full = _full_pages(case)
        return {"bytes": full * G * (page * (D + 4.0) + 2.0 * D + 4) + 8.0 * case["batch"], "flops": 3.0 * full * G * page * D + 1.0}
    L, H, new = _lengths(case), case["heads"], case["new"]
    pages = [-(-n // page) for n in L]
    looked = sum(p for p in pages if p > case["keep"])
    kept = sum(min(n, case["keep"] * page) for n in L)
    n = sum(min(new, x) for x in L)
    return {"bytes": looked * (G * (2.0 * D + 4) + 4) + kept * token + 4.0 * n * H * D, "flops": 4.0 * D * H * new * (looked + kept)}


def _cost(case):
    """Seconds, roughly, that a pass of the plain form is worth: it limits the drawn cases."""
    w = work(case)
    if case["kind"] == "beam":
        return 1.0 * case["batch"] * case["beams"] * case["vocab"]
    G, D, page = case["kv_heads"], case["dim"], case["page"]
    if case["kind"] == "fork":
        return _fork_sizes(case)[3] * page * G * D * 1e-12 + w["bytes"] / 4e12
    if case["kind"] == "compact":
        return case["pages"] * page * G * D * 1e-12 + w["bytes"] / 4e12
    tokens = sum(_lengths(case)) * G * D * 1e-12
    if case["kind"] == "bounds":
        return tokens + w["bytes"] / 1e12
    padded = case["batch"] * case["heads"] * case["new"] * min(case["longest"], case["keep"] * page) * 4.0
    return tokens + w["bytes"] / 1e12 + 8 * padded / 4e12 + case["batch"] * case["longest"] // page * case["heads"] * case["new"] * 16.0 / 4e12


# ---- inputs ------------------------------------------------------------------------------------------

def _store(g, pages, G, page, D, s):
    """Codes and steps of a cache's pages, any values."""
    for name in "kv":
        s[name] = torch.randint(-127, 128, (pages, G, page, D), generator=g, device="cuda", dtype=torch.int8)
        s[name + "_step"] = torch.rand((pages, G, page), generator=g, device="cuda") * 0.02 + 0.01


def _quantised(x):
    step = x.abs().amax(-1) / 127
    return (x / step[..., None]).round().to(torch.int8), step


def _inputs(case, seed):
    """The tensors of a case, made on the GPU from the seed."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    if case["kind"] == "beam":
        B, W, V = case["batch"], case["beams"], case["vocab"]
        x = rand(B * W, V) * 2
        x[:, : max(1, V // 200)] += 4                                 # some tokens are likely everywhere
        x[torch.rand((B * W, V), generator=g, device="cuda") < 0.02] = -INF               # tokens that the program bans
        scores = -20 * torch.rand(B * W, generator=g, device="cuda")
        at = torch.arange(B * W, device="cuda")
        scores[(at // W % 5 == 3) & (at % W > 0)] = -INF              # sequences at their first step: one beam is alive
        finished = (torch.rand(B * W, generator=g, device="cuda") < 0.1)
        return {"logits": x.to(TYPES[case["dtype"]]), "scores": scores, "finished": finished.to(torch.uint8), "end": 2}
    G, D, page = case["kv_heads"], case["dim"], case["page"]
    if case["kind"] == "fork":
        B, W = case["batch"], case["beams"]
        shared, alone, width, pages = _fork_sizes(case)
        L = _lengths(case)
        own_first, ids = [], 0
        group_first = []
        for s, a in zip(shared, alone):
            group_first += [ids] * W
            own_first += [ids + s + w * a for w in range(W)]
            ids += s + W * a
        each = lambda v: torch.tensor(v, device="cuda").repeat_interleave(W)[:, None]
        at, s, n = torch.arange(width, device="cuda")[None, :], each(shared), each([s + a for s, a in zip(shared, alone)])
        number = torch.where(at < s, torch.tensor(group_first, device="cuda")[:, None] + at, torch.tensor(own_first, device="cuda")[:, None] + at - s)
        order = torch.randperm(pages, generator=g, device="cuda")
        table = torch.where(at < n, order[number.clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
        parents = torch.randint(0, W, (B, W), generator=g, device="cuda") + W * torch.arange(B, device="cuda")[:, None]
        ended = _ended(case)
        if ended:
            parents[ended] = -1
        state = {"table": table, "refs": torch.bincount(table[table >= 0], minlength=pages).to(torch.int32), "parents": parents.flatten().to(torch.int32),
                 "lens": ints([n + case["grown"] for n in L for _ in range(W)])}
        _store(g, pages, G, page, D, state)
        return state
    if case["kind"] == "compact":
        P, U, R = case["pages"], case["used"], min(case["rows"], case["used"])
        held = torch.randperm(P, generator=g, device="cuda")[:U]
        width = -(-U // R)
        table = torch.full((R * width,), -1, dtype=torch.int32, device="cuda")
        table[:U] = held.to(torch.int32)
        refs = torch.zeros(P, dtype=torch.int32, device="cuda")
        refs[held] = torch.randint(1, 4, (U,), generator=g, device="cuda", dtype=torch.int32)     # other tables hold some of them too
        state = {"table": table.reshape(R, width), "refs": refs}
        _store(g, P, G, page, D, state)
        return state
    order = torch.randperm(case["batch"], generator=g, device="cuda").tolist()
    L = [_lengths(case)[i] for i in order]
    new = [min(case["new"], n) for n in L]
    per = [-(-n // page) for n in L]
    total, width = sum(per) + 3, max(per)
    free = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(width, device="cuda")[None, :]
    start, count = (torch.tensor(v, device="cuda")[:, None] for v in ([sum(per[:i]) for i in range(len(per))], per))
    state = {"table": torch.where(at < count, free[(start + at).clamp(max=total - 1)], -1).to(torch.int32).contiguous(), "cu": _offsets(new), "lens": ints(L),
             "max_new": max(new), "max_len": max(L), "lengths": L, "new": new}
    # what a page is about: its keys lie around a direction of their own
    state["k"], state["k_step"] = _quantised(rand(total, G, page, D).add_(rand(total, G, 1, D)))
    state["b_codes"] = torch.zeros(total, G, 2, D, dtype=torch.int8, device="cuda")
    state["b_steps"] = torch.zeros(total, G, device="cuda")
    if case["kind"] == "bounds":
        state["v"], state["v_step"] = torch.zeros_like(state["k"]), torch.zeros_like(state["k_step"])
        return state
    state["v"], state["v_step"] = _quantised(rand(total, G, page, D))
    for i in range(0, total, 4096):
        state["b_codes"][i:i + 4096], state["b_steps"][i:i + 4096] = _page_bounds(state["k"][i:i + 4096], state["k_step"][i:i + 4096])
    state["q"] = (rand(sum(new), case["heads"], D) * 1.5).to(TYPES[case["dtype"]])
    return state


def _offsets(lengths):
    return torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2209_09130_amd as P
        s["P"] = P
        if case["kind"] != "beam":
            s["cache"] = P.KVCache(s["k"], s["v"], s["k_step"], s["v_step"])
        if "b_codes" in s:
            s["bounds"] = P.KeyBounds(s["b_codes"], s["b_steps"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        P = s["P"]
        if kind == "beam":
            return P.beam_select(s["logits"], s["scores"], c["beams"], c["keep"], finished=s["finished"], end=s["end"])
        if kind == "fork":
            refs, table, lens, copies, lacking = P.pages_fork(s["refs"], s["table"], s["lens"], c["page"], s["parents"], None, c["new"])
            P.cache_copy(s["cache"], copies)
            return refs, table, lens, copies, lacking, s["k"], s["v"], s["k_step"], s["v_step"]
        if kind == "compact":
            refs, table, copies, used = P.pages_compact(s["refs"], s["table"], c["page"])
            P.cache_copy(s["cache"], copies)
            return refs, table, copies, used, s["k"], s["v"], s["k_step"], s["v_step"]
        if kind == "bounds":
            P.cache_bounds(s["cache"], s["bounds"], s["table"], s["cu"], s["lens"], s["max_new"])
            return s["b_codes"], s["b_steps"]
        return P.attention_sparse(s["q"], s["cache"], s["bounds"], s["table"], s["cu"], s["lens"], s["max_new"], c["keep"], recent=c["recent"], max_len=s["max_len"])
    return {"beam": _plain_beam, "fork": _plain_fork, "compact": _plain_compact, "bounds": _plain_bounds, "sparse": _plain_sparse}[kind](s)


def _plain_beam(s):
    B, W, V, keep = (s["case"][n] for n in ("batch", "beams", "vocab", "keep"))
    x = s["logits"].double()                                          # candidates of different beams may lie close together
    top = x.amax(1, keepdim=True)
    x -= top + (x - top).exp().sum(1, keepdim=True).log()
    x += s["scores"].double()[:, None]
    done = s["finished"].bool()
    x.masked_fill_(done[:, None], -INF)
    x[:, s["end"]] = torch.where(done, s["scores"].double(), x[:, s["end"]])
    x = x.reshape(B, W * V)
    # the best `keep`, the lowest place first among equals
    least = x.topk(keep, 1).values[:, -1:]
    more, equal = x > least, x == least
    chosen = more | (equal & (equal.cumsum(1, dtype=torch.int32) <= keep - more.sum(1, keepdim=True)))
    at = W * V - torch.where(chosen, W * V - torch.arange(W * V, device="cuda", dtype=torch.int32), 0).topk(keep, 1).values.long()
    scores, order = x.gather(1, at).sort(dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    there = scores > -INF
    parents = torch.where(there, at // V + W * torch.arange(B, device="cuda")[:, None], -1)
    return scores.float(), parents.to(torch.int32), torch.where(there, at % V, -1).to(torch.int32)


def _count(pages, there, total):
    """How many of the entries that are there name each page."""
    return torch.zeros(total, dtype=torch.int32, device="cuda").index_add_(0, pages.clamp(0, total - 1).flatten().long(), there.flatten().to(torch.int32))


def _listed_first(mask):
    """The places where a mask is set, in order, then the others."""
    return torch.sort(mask, descending=True, stable=True).indices


def _copy(s, copies):
    there = copies[1] >= 0
    src, dst, n = copies[:, there].long()
    seen = torch.arange(s["case"]["page"], device="cuda") < n[:, None, None]
    for name in ("k", "v", "k_step", "v_step"):
        x = s[name]
        x[dst] = torch.where(seen if x.dim() == 3 else seen[..., None], x[src], x[dst])


def _plain_fork(s):
    page, new = s["case"]["page"], s["case"]["new"]
    table, refs = s["table"], s["refs"]
    P, width = refs.numel(), table.shape[1]
    alive = s["parents"] >= 0
    parent = s["parents"].clamp(min=0).long()
    held = torch.where(alive, s["lens"][parent], 0)
    lens = torch.where(alive, held + new, 0)
    first, end = held // page, (lens + page - 1) // page              # the pages that will be written, and behind the last
    at = torch.arange(width, device="cuda")
    child = torch.where(alive[:, None] & (at < end[:, None]), table[parent], -1)
    there = (child >= 0) & (child < P)
    refs = refs - _count(table, (table >= 0) & (table < P), P) + _count(child, there, P)
    written = alive[:, None] & (at >= first[:, None]) & (at < end[:, None])
    writer = written & there
    page_of = child.clamp(0, P - 1).long()
    place = torch.arange(child.numel(), device="cuda").reshape(child.shape)
    lowest = torch.full((P,), child.numel(), device="cuda").scatter_reduce(0, page_of[writer], place[writer], "amin")
    # a page is written in place by its only holder, or by the first if all its holders are about to write it
    stays = writer & (_count(child, writer, P)[page_of] == refs[page_of]) & (lowest[page_of] == place)
    needs, shared = written & ~stays, writer & ~stays
    free = refs == 0
    rank = needs.flatten().cumsum(0).reshape(needs.shape) - 1
    has = needs & (rank < free.sum())
    fresh = _listed_first(free)[rank.clamp(0, P - 1)]
    out = torch.where(has, fresh, torch.where(needs, -1, child)).to(torch.int32)
    refs = refs - _count(child, shared, P) + _count(out, has, P)
    copied = (shared & has & (at == first[:, None]) & (held % page != 0)[:, None])
    pick = lambda v: torch.where(copied, v, 0).sum(1)
    gone = copied.any(1)
    copies = torch.stack([torch.where(gone, pick(child), -1), torch.where(gone, pick(out), -1), torch.where(gone, held % page, 0)]).to(torch.int32)
    lacking = (needs & ~has).sum() + (end - torch.maximum(first, torch.full_like(first, width))).clamp(min=0).sum()
    _copy(s, copies)
    return refs, out, lens.to(torch.int32), copies, lacking.to(torch.int32).reshape(1), s["k"], s["v"], s["k_step"], s["v_step"]


def _plain_compact(s):
    refs, table, page = s["refs"], s["table"], s["case"]["page"]
    P = refs.numel()
    used = refs > 0
    count = used.sum()
    at = torch.arange(P, device="cuda")
    moves, hole = used & (at >= count), ~used & (at < count)
    holes, movers = _listed_first(hole), _listed_first(moves)
    where = torch.where(used, torch.where(moves, holes[(moves.cumsum(0) - 1).clamp(min=0)], at), -1)
    out = torch.where((table >= 0) & (table < P), where[table.clamp(0, P - 1).long()], -1).to(torch.int32)
    listed_at = at[: max(1, P // 2)]
    there = listed_at < moves.sum()
    copies = torch.stack([torch.where(there, movers[listed_at], -1), torch.where(there, holes[listed_at], -1), torch.where(there, page, 0)]).to(torch.int32)
    moved = torch.zeros_like(refs).index_add_(0, where.clamp(min=0), torch.where(used, refs, 0))
    _copy(s, copies)
    return moved, out, copies, count.to(torch.int32).reshape(1), s["k"], s["v"], s["k_step"], s["v_step"]


def _page_bounds(codes, steps):
    """Codes [pages, G, 2, D] (largest, smallest) and steps [pages, G] of whole pages: the codes rounded outwards."""
    x = codes.float() * steps[..., None]
    high, low = x.amax(2), x.amin(2)
    top = torch.maximum(high.abs(), low.abs()).amax(-1)
    step = torch.where(top > 0, top / 127, 1)
    high, low = (high / step[..., None]).ceil().clamp(max=127), (low / step[..., None]).floor().clamp(min=-127)
    return torch.stack([high, low], 2).to(torch.int8), step


def _plain_bounds(s):
    page = s["case"]["page"]
    at = torch.arange(s["table"].shape[1], device="cuda")
    new = s["cu"][1:] - s["cu"][:-1]
    full = (at >= ((s["lens"] - new) // page)[:, None]) & (at < (s["lens"] // page)[:, None])
    pages = s["table"][full].long()
    s["b_codes"][pages], s["b_steps"][pages] = _page_bounds(s["k"][pages], s["k_step"][pages])
    return s["b_codes"], s["b_steps"]


def _plain_sparse(s):
    c = s["case"]
    B, H, G, D, page, keep, n = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["page"], c["keep"], s["max_new"]
    width = s["table"].shape[1]
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    new = (s["cu"][1:] - s["cu"][:-1])[:, None]
    there = row[None, :] < new
    q = s["q"].float()[(s["cu"][:-1, None] + row).clamp(max=s["q"].shape[0] - 1)].masked_fill(~there[..., None, None], 0)    # [B, n, H, D]
    q = q.reshape(B, n, G, H // G, D).permute(0, 2, 1, 3, 4).reshape(B, G, n * (H // G), D).contiguous()
    # what a page promises: the largest score that a key inside its bounds could have, in 8 bits
    top = q.abs().amax(-1)
    step = torch.where(top > 0, top / 127, 1)
    codes = (q * 127 / torch.where(top > 0, top, 1)[..., None]).round()
    table = s["table"].clamp(min=0).long()
    high, low = s["b_codes"][table].permute(3, 0, 2, 4, 1).float().reshape(2, B * G, D, width).contiguous()
    flat = codes.reshape(B * G, -1, D)
    sums = (torch.bmm(flat.clamp(min=0), high) + torch.bmm(flat.clamp(max=0), low)).reshape(B, G, -1, width)
    score = sums * (step[..., None] * s["b_steps"][table].permute(0, 2, 1)[:, :, None])
    rows = there[:, None, :, None].expand(B, 1, n, H // G).reshape(B, 1, -1, 1)
    score = score.masked_fill(~rows, -INF).amax(2)                    # [B, G, width]
    at = torch.arange(width, device="cuda")
    pages = ((s["lens"] + page - 1) // page)[:, None]
    exists = (at < pages)[:, None]
    score = torch.where(((at < 1) | (at >= pages - c["recent"]))[:, None], INF, score).masked_fill(~exists, -INF)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    chosen = torch.where(exists.expand(B, G, width).gather(2, best), best, width).sort(-1).values        # [B, G, keep or fewer]
    number = torch.where(chosen < width, s["table"][torch.arange(B, device="cuda")[:, None, None], chosen.clamp(max=width - 1)], 0).long()
    head = torch.arange(G, device="cuda")[None, :, None]
    k, v = ((s[x][number, head].float() * s[x + "_step"][number, head][..., None]).flatten(2, 3) for x in "kv")            # [B, G, keys, D]
    pos = (chosen[..., None] * page + torch.arange(page, device="cuda")).flatten(2)
    last = (s["lens"][:, None] - new + row).repeat_interleave(H // G, 1)                                 # a row's own position
    seen = (pos[:, :, None, :] <= last[:, None, :, None]) & (chosen < width).repeat_interleave(page, 2)[:, :, None, :]
    m = k.shape[2]
    scores = torch.bmm(q.reshape(B * G, -1, D), k.reshape(B * G, m, D).transpose(1, 2).contiguous()).reshape(B, G, -1, m)
    scores = (scores / math.sqrt(D)).masked_fill_(~seen, -INF)
    p = scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.reshape(B * G, -1, m), v.reshape(B * G, m, D)).reshape(B, G, -1, D) / torch.where(total > 0, total, 1)
    return o.reshape(B, G, n, H // G, D).permute(0, 2, 1, 3, 4).reshape(B, n, H, D)[there].to(s["q"].dtype)


# ---- the definition in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "compact"):
        s = _inputs(case, seed)
        unchanged = s["k_step"].double(), s["v_step"].double()        # steps are copied: a page that took a copy has its source's
        moved = _exact_fork(case, s) if kind == "fork" else _exact_compact(case, s)
        for src, dst, n in moved:
            for x in unchanged:
                x[dst, :, :n] = x[src, :, :n]
        return (None,) * (7 if kind == "fork" else 6) + unchanged
    s = _inputs(case, seed)
    if kind == "beam":
        B, W, keep = case["batch"], case["beams"], case["keep"]
        out = []
        for b in range(B):
            rows = slice(b * W, b * W + W)
            total = torch.log_softmax(s["logits"][rows].double(), -1) + s["scores"][rows].double()[:, None]
            for w in range(W):
                if s["finished"][b * W + w]:
                    total[w] = -INF
                    total[w, s["end"]] = s["scores"][b * W + w].double()
            out.append(total.flatten().sort(descending=True).values[:keep])
        return torch.stack(out), None, None
    page, G, D = case["page"], case["kv_heads"], case["dim"]
    if kind == "bounds":
        steps = s["b_steps"].double()
        tables = s["table"].tolist()
        full = [tables[b][j] for b, (n, m) in enumerate(zip(s["lengths"], s["new"])) for j in range((n - m) // page, n // page)]
        for i in range(0, len(full), 512):
            ids = torch.tensor(full[i:i + 512], device="cuda")
            steps[ids] = (s["k"][ids].double().abs() * s["k_step"][ids].double()[..., None]).amax((2, 3)) / 127
        return None, steps
    H, share = case["heads"], case["heads"] // G
    out = torch.empty(sum(s["new"]), H, D, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(s["lengths"], s["new"])):
        count = -(-n // page)
        ids = s["table"][b, :count].long()
        q = s["q"][at:at + m].double()
        pos = torch.arange(count * page, device="cuda").reshape(count, page)
        for g in range(G):
            heads = slice(g * share, g * share + share)
            chosen = torch.arange(count, device="cuda")
            if count > case["keep"]:
                top = q[:, heads].abs().amax(-1, keepdim=True)
                codes = torch.round(127 * q[:, heads] / top).reshape(-1, 1, D)
                high, low = s["b_codes"][ids, g].double().unbind(1)
                sums = torch.cat([torch.maximum(r * high, r * low).sum(-1)[None] for r in codes])
                # (scores are defined in 32 bits: whole numbers times a product of two steps)
                score = (sums.float() * ((top.float() / 127).reshape(-1, 1) * s["b_steps"][ids, g])).amax(0).double()
                score[0], score[count - case["recent"]:] = INF, INF
                chosen = torch.argsort(-score, stable=True)[: case["keep"]].sort().values
            k, v = (s[x][ids[chosen], g].double() * s[x + "_step"][ids[chosen], g].double()[..., None] for x in "kv")
            where = pos[chosen].flatten()
            for i in range(m):
                w = q[i, heads] @ k.reshape(-1, D).t().contiguous() / math.sqrt(D)
                w[:, where > n - m + i] = -INF
                out[at + i, heads] = torch.softmax(w, -1) @ v.reshape(-1, D)
        at += m
    return out


def _exact_fork(case, s):
    """The copies, by taking one beam after the other."""
    page, new = case["page"], case["new"]
    table, refs, lens, parents = (s[n].tolist() for n in ("table", "refs", "lens", "parents"))
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    children = []
    for p in parents:
        end = -(-(lens[p] + new) // page) if p >= 0 else 0
        children.append([x for x in (table[p] if p >= 0 else [])[:end] if x >= 0])
        for x in children[-1]:
            refs[x] += 1
    free = iter([i for i, r in enumerate(refs) if r == 0])
    moved = []
    ready = {}                                                        # page -> beams that are about to write it
    for p, row in zip(parents, children):
        if p >= 0:
            for x in row[lens[p] // page:]:
                ready[x] = ready.get(x, 0) + 1
    kept = set()
    for p, row in zip(parents, children):
        if p < 0:
            continue
        first, end = lens[p] // page, -(-(lens[p] + new) // page)
        for j in range(first, end):
            x = row[j] if j < len(row) else -1
            if x >= 0 and ready[x] == refs[x] and x not in kept:
                kept.add(x)
                continue
            to = next(free)
            if x >= 0 and j == first and lens[p] % page:
                moved.append((x, to, lens[p] % page))
    return moved


def _exact_compact(case, s):
    refs = s["refs"].tolist()
    count = sum(r > 0 for r in refs)
    holes = [i for i in range(count) if refs[i] <= 0]
    return [(src, dst, case["page"]) for src, dst in zip([i for i in range(count, len(refs)) if refs[i] > 0], holes)]
