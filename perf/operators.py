"""Operators of an 8-bit decoder's attention block, measured one at a time.

A serving program quantises the rows of a projection as they come (a step for each token) and multiplies the codes by int8
weights (a step for each output channel); keys and values go to a paged cache of int8 codes, with a step for each token and
head; a prompt attends to itself causally in 16 bits, and later tokens, one or a few drafted ones at a time, attend to the
cache.  Four kinds of case, one for each of those:

  linear   x [M, K] in 16 bits -> y [M, N], rows quantised on the way in
  cache    new keys and values are written to the cache, then the sequences' whole contexts are read back in 16 bits
  cached   queries of the new tokens against the cache (after their keys and values were written)
  causal   packed prompts of different lengths, grouped heads
"""
import math

import torch

own = False

FP16, BF16 = "fp16", "bf16"
TYPES = {FP16: torch.float16, BF16: torch.bfloat16}


def _linear(name, rows, k, n, dtype, bias=False, gelu=False):
    return {"name": name, "kind": "linear", "rows": rows, "k": k, "n": n, "dtype": dtype, "bias": bias, "gelu": gelu}


def _heads(name, kind, batch, shortest, longest, heads, kv_heads, dim, dtype, new=0, page=0, tree=False):
    """Lengths spread evenly over [shortest, longest] in random order; new: tokens of each sequence that are new (at most its
    length); tree: the new tokens are drafts, each seeing its ancestors among them."""
    return {"name": name, "kind": kind, "batch": batch, "shortest": shortest, "longest": longest, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "dtype": dtype, "new": new, "page": page, "tree": tree}


def listed():
    return [
        # the fused projection of one decoded token: 25 MB of weights for one row
        _linear("linear 1x4096x6144", 1, 4096, 6144, FP16),
        # a small odd batch of prompt rows, widths that no tile divides, the feed-forward's activation behind it
        _linear("linear 533x1600x2512 gelu", 533, 1600, 2512, BF16, bias=True, gelu=True),
        # a prompt batch at full rate
        _linear("linear 8192x4096x4096", 8192, 4096, 4096, FP16, bias=True),
        # a decode step of a few short chats: latency
        _heads("cache 4 tokens", "cache", 4, 20, 150, 12, 12, 64, FP16, new=1, page=16),
        # a chunk of prompt appended to contexts of some thousand tokens, which its attention then reads
        _heads("cache chunk 4x512", "cache", 4, 700, 4500, 32, 8, 128, BF16, new=512, page=64),
        # whole prompts written and read back
        _heads("cache prompts 16x2048", "cache", 16, 900, 2048, 32, 8, 128, FP16, new=2048, page=128),
        # one user, one token, a medium context: latency
        _heads("cached 1x4000", "cached", 1, 4000, 4000, 32, 8, 128, FP16, new=1, page=64),
        # sixteen drafted tokens in a tree for each of eight sequences, a head of its own for each query head
        _heads("cached tree 8x16", "cached", 8, 300, 2100, 16, 16, 64, BF16, new=16, page=32, tree=True),
        # the decode step of a loaded server: ragged contexts up to 8192 tokens
        _heads("cached 64x8192", "cached", 64, 17, 8192, 32, 8, 128, BF16, new=1, page=64),
        # short texts as they come to a classifier, packed
        _heads("causal 7x61", "causal", 7, 5, 61, 12, 12, 64, FP16),
        # a batch of ragged prompts, four query heads to a key head
        _heads("causal 8x2048", "causal", 8, 300, 2048, 32, 8, 128, BF16),
        # two long documents
        _heads("causal 2x8192", "causal", 2, 8100, 8192, 32, 8, 128, FP16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges that costs no more than the largest of its kind."""
    while True:
        kind, dtype = rng.choice(("linear", "cache", "cached", "causal")), rng.choice((FP16, BF16))
        if kind == "linear":
            c = _linear("", _log(rng, 1, 16384), 64 * _log(rng, 4, 128), 16 * _log(rng, 16, 512), dtype, rng.random() < 0.5, rng.random() < 0.3)
        else:
            dim = rng.choice((64, 128))
            kv = rng.choice((1, 2, 4, 8, 12))
            batch, longest = _log(rng, 1, 64), _log(rng, 1, 8192)
            shortest = max(1, int(longest * rng.uniform(0.0, 1.0)))
            new, page, tree = 0, 0, False
            if kind != "causal":
                page = rng.choice((16, 32, 64, 128, 256))
                tree = kind == "cached" and rng.random() < 0.3
                new = _log(rng, 1, longest) if kind == "cache" else _log(rng, 2, 32) if tree else rng.choice((1, 1, 1, 2, 5, 8))
            c = _heads("", kind, batch, shortest, longest, kv * rng.choice((1, 2, 4, 7, 8)), kv, dim, dtype, new, page, tree)
        del c["name"]
        if _cost(c) <= max(_cost(x) for x in listed() if x["kind"] == kind) and c.get("heads", 1) <= 64:
            return c


def _lengths(case):
    B, lo, hi = case["batch"], case["shortest"], case["longest"]
    return [hi] if B == 1 else [lo + round((hi - lo) * i / (B - 1)) for i in range(B)]


def _new(case, lengths):
    return [min(case["new"], n) for n in lengths]


def work(case):
    if case["kind"] == "linear":
        m, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": 2.0 * m * k + n * k + 2.0 * m * n + 4.0 * n * (2 if case["bias"] else 1), "flops": 2.0 * m * n * k}
    L, H, G, D = _lengths(case), case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "causal":
        return {"bytes": 4.0 * sum(L) * D * (H + G), "flops": 4.0 * D * H * sum(n * (n + 1) / 2 for n in L)}
    new = _new(case, L)
    row = 2.0 * G * (D + 4)                                           # a token's keys and values in the cache
    if case["kind"] == "cache":
        return {"bytes": sum(new) * (4.0 * G * D + row) + sum(L) * (row + 4.0 * G * D), "flops": 4.0 * G * D * (sum(new) + sum(L))}
    return {"bytes": sum(L) * row + 4.0 * sum(new) * H * D, "flops": 4.0 * D * H * sum(n * m for n, m in zip(L, new))}


def _cost(case):
    """Seconds, roughly, that a pass of the plain form is worth: it limits the drawn cases."""
    w = work(case)
    if case["kind"] == "linear":
        return w["bytes"] / 4e12 + w["flops"] / 1e14
    L = case["longest"]
    padded = case["batch"] * case["heads"] * (case["new"] or L) * L * 4.0 if case["kind"] != "cache" else 0.0   # one copy of the scores
    return w["bytes"] / 4e12 + w["flops"] / 1e14 + 8 * padded / 4e12 + case["batch"] * L * case["kv_heads"] * case["dim"] * 16.0 / 4e12


# ---- inputs ------------------------------------------------------------------------------------------

def _inputs(case, seed):
    """The tensors of a case, made on the GPU from the seed."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    if case["kind"] == "linear":
        m, k, n = case["rows"], case["k"], case["n"]
        x = rand(m, k)
        x[:, : max(1, k // 100)] *= 8                                 # a few channels are larger, as after a LayerNorm
        w = rand(n, k) * 0.02
        s_w = w.abs().amax(1) / 127
        return {"x": x.to(t), "w": (w / s_w[:, None]).round().clamp(-127, 127).to(torch.int8), "s_w": s_w,
                "bias": rand(n) * 0.1 if case["bias"] else None}
    order = torch.randperm(case["batch"], generator=g, device="cuda").tolist()
    L = [_lengths(case)[i] for i in order]
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "causal":
        qkv = rand(sum(L), (H + 2 * G) * D).to(t)                     # the fused projection's output, read in place
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split((H * D, G * D, G * D), 1))
        return {"q": q, "k": k, "v": v, "cu": _offsets(L), "max_len": max(L), "lengths": L}
    new, page = _new(case, L), case["page"]
    pages = [-(-n // page) for n in L]
    total = sum(pages) + 3
    free = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    width = max(pages)
    at = torch.arange(width, device="cuda")[None, :]
    start, count = (torch.tensor(v, device="cuda")[:, None] for v in ([sum(pages[:i]) for i in range(len(pages))], pages))
    table = torch.where(at < count, free[(start + at).clamp(max=total - 1)], -1).to(torch.int32).contiguous()
    store = {}
    for name in "kv":
        x = rand(total, G, page, D)
        s = x.abs().amax(-1) / 127
        store[name], store[name + "_step"] = (x / s[..., None]).round().to(torch.int8), s
        del x
    state = {**store, "table": table, "cu": _offsets(new), "lens": torch.tensor(L, dtype=torch.int32, device="cuda"), "max_new": max(new),
             "max_len": max(L), "lengths": L, "new": new}
    if case["kind"] == "cache":
        state.update(new_k=rand(sum(new), G, D).to(t), new_v=rand(sum(new), G, D).to(t), cu_all=_offsets(L), rows=sum(L))
    else:
        state.update(q=(rand(sum(new), H, D) * 1.5).to(t), tree=_tree(new, g) if case["tree"] else None)
    return state


def _offsets(lengths):
    return torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)


def _tree(new, g):
    """Bit j of a draft's word: it sees draft j of its sequence.  Draft i's parent is a random earlier one; draft 0 is the root."""
    words, pick = [], torch.rand(sum(new), generator=g, device="cuda").tolist()
    for n in new:
        seen = []
        for i in range(n):
            seen.append((seen[int(pick.pop() * i)] if i else 0) | 1 << i)
        words += seen
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2209_09130_amd as P
        s["P"] = P
        if case["kind"] == "linear":
            s["w_packed"] = P.pack_weight_i8(s["w"])                  # weights are laid out once
        elif case["kind"] != "causal":
            s["cache"] = P.KVCache(s["k"], s["v"], s["k_step"], s["v_step"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        P = s["P"]
        if kind == "linear":
            return P.linear_i8_tokens(s["x"], s["w_packed"], s["s_w"], s["bias"], s["case"]["gelu"])
        if kind == "causal":
            return P.attention_causal(s["q"], s["k"], s["v"], s["cu"], s["max_len"])
        if kind == "cached":
            return P.attention_cache(s["q"], s["cache"], s["table"], s["cu"], s["lens"], s["max_new"], max_len=s["max_len"], tree=s["tree"])
        P.cache_write(s["cache"], s["new_k"], s["new_v"], s["table"], s["cu"], s["lens"], s["max_new"])
        return P.cache_read(s["cache"], s["table"], s["cu_all"], s["lens"], s["max_len"], s["rows"], s["new_k"].dtype)
    return {"linear": _plain_linear, "cache": _plain_cache, "cached": _plain_cached, "causal": _plain_causal}[kind](s)


def _codes(x):
    """(codes, steps) over the last axis: step = absmax / 127, code = 127 x / absmax rounded half to even."""
    x = x.float()
    top = x.abs().amax(-1)
    ok = top > 0
    return (x * 127 / torch.where(ok, top, 1)[..., None]).round(), torch.where(ok, top / 127, 1)


def _plain_linear(s):
    codes, step = _codes(s["x"])
    y = codes @ s["w"].float().T * (step[:, None] * s["s_w"])
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["case"]["gelu"]:
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["x"].dtype)


def _places(s, cu, rows):
    """For packed rows, of which sequence b has the last cu[b + 1] - cu[b] of its positions: their pages and offsets in them."""
    row = torch.arange(rows, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(cu, row, right=True) - 1
    pos = s["lens"][b] - (cu[b + 1] - row)
    page = s["k"].shape[2]
    return s["table"][b, pos // page].long(), (pos % page).long()


def _plain_cache(s):
    page, at = _places(s, s["cu"], s["new_k"].shape[0])
    out = []
    for name, x in (("k", s["new_k"]), ("v", s["new_v"])):
        codes, step = _codes(x)
        s[name][page, :, at] = codes.to(torch.int8)
        s[name + "_step"][page, :, at] = step
    page, at = _places(s, s["cu_all"], s["rows"])
    for name in "kv":
        out.append((s[name][page, :, at].float() * s[name + "_step"][page, :, at][..., None]).to(s["new_k"].dtype))
    return tuple(out)


def _attend(q, k, v, seen):
    """q [B, H, n, D], k and v [B, G, m, D] and seen [B, 1, n, m], in 32 bits; rows that see nothing are zeros."""
    B, H, n, D = q.shape
    G, m = k.shape[1:3]
    scores = (q.reshape(B * G, H // G * n, D) @ k.reshape(B * G, m, D).transpose(1, 2).contiguous()).reshape(B, H, n, m)
    scores = (scores / math.sqrt(D)).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(B * G, H // G * n, m) @ v.reshape(B * G, m, D)).reshape(B, H, n, D)
    return o / torch.where(total > 0, total, 1)


def _padded(x, cu, longest):
    """Packed rows x [T, H, D] as [B, H, longest, D] in 32 bits, and which of them are there."""
    at = torch.arange(longest, device="cuda", dtype=torch.int32)[None, :]
    there = at < (cu[1:] - cu[:-1])[:, None]
    return x.float()[(cu[:-1, None] + at).clamp(max=x.shape[0] - 1)].masked_fill(~there[..., None, None], 0).transpose(1, 2).contiguous(), there


def _plain_causal(s):
    (q, there), (k, _), (v, _) = (_padded(s[n], s["cu"], s["max_len"]) for n in "qkv")
    at = torch.arange(s["max_len"], device="cuda")
    seen = (at[None, :] <= at[:, None])[None, None]
    return _attend(q, k, v, seen).transpose(1, 2)[there].to(s["q"].dtype)


def _plain_cached(s):
    pages = s["table"].clamp(min=0).long()
    B, width = pages.shape
    k, v = ((s[n][pages].float() * s[n + "_step"][pages][..., None]).transpose(1, 2).flatten(2, 3) for n in "kv")
    q, there = _padded(s["q"], s["cu"], s["max_new"])
    n, m = q.shape[2], k.shape[2]
    new = (s["cu"][1:] - s["cu"][:-1])[:, None, None]
    first = s["lens"][:, None, None] - new                             # position of the first new token
    row, at = torch.arange(n, device="cuda")[None, :, None], torch.arange(m, device="cuda")[None, None, :]
    if s["tree"] is None:
        seen = at <= first + row
    else:
        words = s["tree"][(s["cu"][:-1, None] + row[..., 0]).clamp(max=s["tree"].shape[0] - 1)][..., None]
        seen = (at < first) | ((words >> (at - first).clamp(0, 63)) & 1).bool()
    seen = seen & (at < s["lens"][:, None, None])
    return _attend(q, k, v, seen[:, None]).transpose(1, 2)[there].to(s["q"].dtype)


# ---- the definition in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    D = case.get("dim")
    if case["kind"] == "linear":
        x = s["x"].double()
        top = x.abs().max(1).values.clamp(min=1e-300)
        y = torch.round(127 * x / top[:, None]) @ s["w"].double().t().contiguous()
        y = y * (top / 127)[:, None] * s["s_w"].double()[None, :]
        y = y if s["bias"] is None else y + s["bias"].double()
        return y * torch.special.ndtr(y) if case["gelu"] else y
    starts = lambda counts: [sum(counts[:i]) for i in range(len(counts))]
    if case["kind"] == "causal":
        out = []
        for at, n in zip(starts(s["lengths"]), s["lengths"]):
            part = {c: s[c][at:at + n].double().transpose(0, 1).contiguous() for c in "qkv"}
            out.append(_exact_heads(part["q"], part["k"], part["v"], torch.ones(n, n, dtype=torch.bool, device="cuda").tril()))
        return torch.cat(out)
    page = case["page"]
    tables = s["table"].tolist()

    def context(name, b):
        n = s["lengths"][b]
        ids = torch.tensor(tables[b][: -(-n // page)], device="cuda")
        whole = s[name][ids].double() * s[name + "_step"][ids].double().unsqueeze(-1)      # [pages, G, page, D]
        return whole.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, D)[:, :n]

    out = ([], []) if case["kind"] == "cache" else []
    for b, (at, n) in enumerate(zip(starts(s["new"]), s["new"])):
        if case["kind"] == "cache":
            for name, to in zip("kv", out):
                fresh = s["new_" + name][at:at + n].double()
                top = fresh.abs().max(-1, keepdim=True).values.clamp(min=1e-300)
                old = context(name, b)[:, : s["lengths"][b] - n].transpose(0, 1)
                to.append(torch.cat([old, torch.round(fresh * 127 / top) * (top / 127)]))
            continue
        m = s["lengths"][b]
        seen = torch.ones(n, m, dtype=torch.bool, device="cuda").tril(m - n)
        if s["tree"] is not None:
            words = s["tree"][at:at + n].tolist()
            seen[:, m - n:] = torch.tensor([[w >> j & 1 == 1 for j in range(n)] for w in words], device="cuda")
        out.append(_exact_heads(s["q"][at:at + n].double().transpose(0, 1), context("k", b), context("v", b), seen))
    return tuple(torch.cat(o) for o in out) if case["kind"] == "cache" else torch.cat(out)


def _exact_heads(q, k, v, seen):
    """[n, H, D] from q [H, n, D] and k, v [G, m, D] in 64 bits, one key head at a time."""
    share = q.shape[0] // k.shape[0]
    out = torch.empty(q.shape[1], q.shape[0], q.shape[2], dtype=torch.float64, device="cuda")
    for h in range(q.shape[0]):
        scores = (q[h] @ k[h // share].t().contiguous()) * q.shape[2] ** -0.5
        scores[~seen] = -math.inf
        out[:, h] = torch.softmax(scores, -1) @ v[h // share]
    return out
