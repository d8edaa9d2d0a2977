"""Bounds of a page's keys, the choice of pages by them, and attention over the chosen ones, against their definitions.

Bounds and scores are defined in binary32 operations on whole numbers, so codes, steps and the chosen pages are compared for equality; the attention with the tolerances of
test_gpu_decoder.py.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from test_gpu_decoder import BF16, F16, P, Plan, attend, check_attention, gen, offsets, quantised, run_cached, signed, tree_words  # noqa: E402,F401


INV_127 = torch.tensor(1.0) / torch.tensor(127.0)


def bounds_definition(codes, steps):
    """codes int8 [page_len, D] and steps float32 [page_len] of one page and head -> (int8 [2, D], float32)."""
    if not torch.isfinite(steps).all():
        return torch.zeros(2, codes.shape[1], dtype=torch.int8), torch.tensor(math.nan)
    x = codes.float() * steps[:, None]
    high, low = x.amax(0), x.amin(0)
    top = torch.maximum(high.abs(), low.abs()).max()
    if top == 0:
        return torch.zeros(2, codes.shape[1], dtype=torch.int8), torch.tensor(1.0)
    step = top * INV_127
    return torch.stack([(high / step).ceil().clamp(max=127), (low / step).floor().clamp(min=-127)]).to(torch.int8), step


def same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("D,G,page", [(64, 12, 16), (128, 8, 64), (128, 1, 256), (64, 3, 32), (128, 2, 1024), (64, 1, 128)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([40, 7, 0, 129, 16], [3, 7, 0, 1, 16]), ([300, 257, 64], [300, 1, 20]), ([2048, 2047], [1, 2047])])
def test_bounds_of_the_pages_that_new_positions_fill(P, D, G, page, lens, new):
    plan = Plan(P, lens, new, G, D, page, seed=D + G)
    plan.fill(P, F16, 4)
    bounds = P.KeyBounds(torch.full((plan.cache.pages, G, 2, D), 77, dtype=torch.int8, device="cuda"), torch.full((plan.cache.pages, G), 7.0, device="cuda"))
    P.cache_bounds(plan.cache, bounds, *plan.args, max(new))
    k, steps = plan.cache.k.cpu(), plan.cache.k_step.cpu()
    want, want_s = torch.full((plan.cache.pages, G, 2, D), 77, dtype=torch.int8), torch.full((plan.cache.pages, G), 7.0)
    for b, (n, m) in enumerate(zip(lens, new)):
        for j in range((n - m) // page, n // page):
            p = plan.tables[b][j]
            for g in range(G):
                want[p, g], want_s[p, g] = bounds_definition(k[p, g], steps[p, g])
    assert torch.equal(bounds.codes.cpu(), want) and torch.equal(bounds.steps.cpu(), want_s)
    again = P.KeyBounds(bounds.codes.clone(), bounds.steps.clone())
    P.cache_bounds(plan.cache, again, *plan.args, 1 << 20, rows=sum(new))              # a larger batch's maximum
    assert torch.equal(again.codes, bounds.codes) and torch.equal(again.steps, bounds.steps)


def test_bounds_of_zeros_of_keys_that_are_not_finite_and_of_bad_pages(P):
    plan = Plan(P, [16 * 7], [16 * 7], 2, 64, 16)
    k, v = (torch.randn(112, 2, 64, generator=gen(i)).bfloat16() for i in (1, 2))
    k[0:16] = 0
    k[16:32] = 2.0 ** -70
    k[32:48, :, 5] = 3e38
    k[50, 0, 3] = math.inf
    k[70, 1, 3] = math.nan
    k[80:96] *= 2.0 ** -50
    k[81] = 0
    table = plan.args[0].clone()
    P.cache_write(plan.cache, k.cuda(), v.cuda(), *plan.args, 112)
    table[0, 6] = 10 ** 6
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, table, None, plan.args[2], 112)
    codes, steps = bounds.codes.cpu(), bounds.steps.cpu()
    for j in range(6):
        p = plan.tables[0][j]
        for g in range(2):
            want, s = bounds_definition(plan.cache.k[p, g].cpu(), plan.cache.k_step[p, g].cpu())
            assert torch.equal(codes[p, g], want) and same(steps[p, g], s), (j, g)
    assert not codes[plan.tables[0][6]].any() and not steps[plan.tables[0][6]].any()
    assert steps[plan.tables[0][0]].tolist() == [1.0, 1.0] and torch.isnan(steps[plan.tables[0][3], 0]) and torch.isnan(steps[plan.tables[0][4], 1])
    # more positions than the table has room for, and more new ones than positions
    long = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, long, plan.args[0], None, torch.tensor([400], dtype=torch.int32, device="cuda"), 300)
    assert not long.codes[plan.tables[0][5]].any() and long.codes[plan.tables[0][6]].any()
    P.cache_bounds(plan.cache, long, plan.args[0], None, torch.tensor([64], dtype=torch.int32, device="cuda"), 300)
    assert long.codes[plan.tables[0][3]].any() and not long.codes[plan.tables[0][4]].any()


def choose_definition(q, codes, steps, table, pages, keep, sinks, recent, heads, G):
    """q [m, heads, D] of one sequence in its type; codes, steps and the sequence's row of the table on the CPU -> per key head the entries of the table that are kept."""
    m, _, D = q.shape
    group, out = heads // G, []
    ok = [0 <= int(table[j]) < codes.shape[0] for j in range(pages)]
    for g in range(G):
        if pages <= keep:
            out.append(list(range(pages)))
            continue
        c, s = quantised(q[:, g * group:(g + 1) * group].reshape(-1, D))
        bad = ~torch.isfinite(q[:, g * group:(g + 1) * group].reshape(-1, D).double()).all(1)
        top = q[:, g * group:(g + 1) * group].reshape(-1, D).float().abs().amax(-1)
        s = torch.where(top >= 2.0 ** -60, top * INV_127, 1.0)
        c[bad], s[bad] = 0, math.nan
        at = torch.tensor([int(table[j]) if ok[j] else 0 for j in range(pages)])
        high, low = codes[at, g].double().unbind(1)                    # [pages, D]
        sums = torch.maximum(c[:, None] * high, c[:, None] * low).sum(-1)
        score = sums.float() * (s[:, None] * steps[at, g][None])
        score = torch.where(torch.isnan(score), math.inf, score)
        score = score.amax(0) if len(score) else torch.full((pages,), -math.inf)
        score[~torch.tensor(ok)] = -math.inf
        always = [j for j in range(pages) if j < sinks or j >= pages - recent]
        rest = sorted((j for j in range(pages) if j not in always), key=lambda j: (-score[j].item(), j))
        out.append(sorted(always + rest[: keep - len(always)]))
    return out


def run_sparse(P, lens, new, H, G, D, page, keep, sinks, recent, dtype, words=None, seed=0, spoil=None, topic=1.0):
    plan = Plan(P, lens, new, G, D, page, seed)
    k, v = (torch.randn(sum(lens), G, D, generator=gen(seed + i)) for i in (0, 1))
    at = 0
    for n in lens:                                           # a page's keys lie around a direction of their own
        for j in range(0, n, page):
            k[at + j:at + min(j + page, n)] += topic * torch.randn(1, G, D, generator=gen(seed + 3 + j))
        at += n
    k, v = k.to(dtype), v.to(dtype)
    q = (torch.randn(plan.total, H, D, generator=gen(seed + 20)) * 1.5).to(dtype)
    if spoil:
        spoil(k, v, q)
    P.cache_write(plan.cache, k.cuda(), v.cuda(), plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens))
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens))
    tables, short = P.cache_select(q.cuda(), plan.cache, bounds, *plan.args, max(new), keep, sinks, recent)
    got = P.attention_sparse(q.cuda(), plan.cache, bounds, *plan.args, max(new), keep, sinks, recent, max_len=max(lens), tree=None if words is None else signed(words).cuda())
    codes, steps = bounds.codes.cpu(), bounds.steps.cpu()
    start = offsets(lens).tolist()
    for b, (n, m) in enumerate(zip(lens, new)):
        at, pages = int(plan.cu[b]), -(-n // page)
        chosen = choose_definition(q[at:at + m], codes, steps, plan.table[b], pages, keep, sinks, recent, H, G)
        assert int(short[b]) == n - (pages - min(pages, keep)) * page
        for g in range(G):
            want = [int(plan.table[b, j]) for j in chosen[g]]
            assert tables[b, g].tolist() == want + [-1] * (keep - len(want)), (b, g)
        if not m:
            continue
        pos, row = torch.arange(n)[None, :], torch.arange(m)[:, None]
        seen = pos <= n - m + row
        if words is not None:
            seen[:, n - m:] = torch.tensor([[bool(w >> j & 1) for j in range(m)] for w in words[at:at + m]])
        held = [(lambda c, s: c * s[..., None])(*quantised(x[start[b]:start[b] + n])) for x in (k, v)]
        for g in range(G):
            of = torch.zeros(n, dtype=torch.bool)
            for j in chosen[g]:
                of[j * page:(j + 1) * page] = True
            heads = slice(g * H // G, (g + 1) * H // G)
            want = attend(q[at:at + m, heads].double(), held[0][:, g:g + 1], held[1][:, g:g + 1], seen & of, D ** -0.5)
            check_attention(got[at:at + m, heads], *want, dtype, F16, n, held[1].abs().max().item())
    return plan, bounds, q, got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,G,D,page", [(4, 4, 64, 16), (8, 2, 128, 64), (7, 1, 128, 32), (32, 8, 128, 16), (20, 1, 64, 16)])
@pytest.mark.parametrize("lens,new,keep,sinks,recent", [([1], [1], 2, 1, 1), ([700, 33, 5, 1000], [1, 1, 1, 1], 4, 1, 1), ([1000, 64, 999], [5, 0, 9], 9, 2, 3),
                                                        ([1500], [1], 5, 0, 2), ([600, 900], [3, 3], 3, 0, 3)])
def test_attention_sparse(P, lens, new, keep, sinks, recent, H, G, D, page, dtype):
    run_sparse(P, lens, new, H, G, D, page, keep, sinks, recent, dtype, seed=len(lens) + H)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_sparse_of_long_contexts(P, dtype):
    run_sparse(P, [9000, 70, 20000], [1, 1, 1], 8, 2, 128, 16, 300, 1, 1, dtype, seed=1)
    run_sparse(P, [16 * 1500 + 3], [2], 4, 1, 64, 16, 40, 1, 2, dtype, seed=2, topic=0.0)
    run_sparse(P, [5000, 4000], [40, 1], 8, 2, 64, 32, 20, 2, 3, dtype, seed=3)        # more rows than one product has columns
    run_sparse(P, [16 * 300, 16 * 299 + 1, 30], [1, 1, 1], 4, 2, 64, 16, 3, 1, 2, dtype, seed=4)              # none but those that are always kept
    run_sparse(P, [16 * 600], [1], 4, 2, 64, 16, 599, 0, 1, dtype, seed=5)             # all but one


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_sparse_of_drafts_in_a_tree(P, dtype):
    for lens, new, keep in (([400, 900, 65], [16, 3, 1], 6), ([2000], [64], 20)):
        run_sparse(P, lens, new, 8, 2, 64, 16, keep, 1, (max(new) + 14) // 16 + 1, dtype, tree_words(new, 3), seed=5)


def test_whole_contexts_are_what_attention_cache_computes(P):
    for lens, keep in (([300, 17, 64], 10), ([5000, 100], 160)):
        plan, bounds, q, got = run_sparse(P, lens, [1] * len(lens), 8, 2, 128, 32, keep, 1, 1, F16, seed=4)
        assert torch.equal(got, P.attention_cache(q.cuda(), plan.cache, *plan.args, 1, max_len=min(max(lens), keep * 32)))


def test_pages_of_one_score_and_scores_that_are_not_numbers(P):
    """Keys that repeat give equal scores: the earlier pages are kept.  A key that is not finite makes its page count as the highest, a query that is not all of them."""
    def repeat(k, v, q):
        k[16:] = k[16:32].repeat(len(k) // 16 - 1, 1, 1)

    run_sparse(P, [640], [1], 4, 2, 64, 16, 7, 1, 1, F16, seed=1, spoil=repeat)

    def zeros(k, v, q):
        k[:] = 0

    run_sparse(P, [640], [1], 4, 2, 64, 16, 7, 1, 2, F16, seed=1, spoil=zeros)
    lens, page, G, D = [800], 16, 2, 64
    plan = Plan(P, lens, [2], G, D, page)
    plan.fill(P, F16, 3)
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], None, plan.args[2], 800)
    bounds.steps[plan.tables[0][20], 1] = math.nan
    bounds.steps[plan.tables[0][30], 0] = math.inf
    table = plan.args[0].clone()
    table[0, 25] = -5
    for bad in (False, True):
        q = torch.randn(2, 4, D, generator=gen(5)).half()
        if bad:
            q[1, 3, 7] = math.nan
        tables, _ = P.cache_select(q.cuda(), plan.cache, bounds, table, None, plan.args[2], 2, 6, 1, 2)
        want = choose_definition(q, bounds.codes.cpu(), bounds.steps.cpu(), table[0].cpu(), 50, 6, 1, 2, 4, G)
        for g in range(G):
            assert tables[0, g].tolist() == [int(table[0, j]) for j in want[g]]
        assert want[1] == [0, 1, 2, 3, 48, 49] if bad else 20 in want[1]               # (all of them the highest: the first ones)


def test_caches_and_bounds_past_32_bits(P):
    """The same pages at the two ends of a cache whose bounds are past 2^31 bytes: what is written there, chosen and read is the same."""
    G, H, D, page, pages = 8, 16, 128, 16, (1 << 20) + 600
    cache = P.KVCache.empty(pages, G, page, D)
    bounds = P.KeyBounds.empty(cache)
    assert bounds.codes.numel() > 1 << 31
    for n in (20, 290):                                      # pages of a sequence: scores formed by the block that chooses, and apart
        low = torch.arange(n, dtype=torch.int32, device="cuda")
        table, lens = torch.stack([low, pages - 1 - low]), torch.tensor([16 * n, 16 * n], dtype=torch.int32, device="cuda")
        k, v = (torch.randn(16 * n, G, D, generator=gen(n + i)).half().cuda().repeat(2, 1, 1) for i in (0, 1))
        P.cache_write(cache, k, v, table, None, lens, 16 * n)
        P.cache_bounds(cache, bounds, table, None, lens, 16 * n)
        assert torch.equal(bounds.codes[table[0]], bounds.codes[table[1]]) and torch.equal(bounds.steps[table[0]], bounds.steps[table[1]]) and bounds.codes[pages - n].any()
        q = torch.randn(1, H, D, generator=gen(n)).half().cuda().repeat(2, 1, 1)
        chosen, _ = P.cache_select(q, cache, bounds, table, None, lens, 1, 7)
        assert torch.equal(chosen[0], pages - 1 - chosen[1]) and (chosen[0].sort().values == chosen[0]).all()
        o = P.attention_sparse(q, cache, bounds, table, None, lens, 1, 7)
        assert torch.equal(o[0], o[1]) and o.abs().sum() > 0


def test_sequences_without_positions_or_new_tokens(P):
    plan = Plan(P, [0, 700, 3], [0, 0, 3], 2, 64, 16)
    plan.fill(P, F16, 3)
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], offsets([0, 700, 3]).cuda(), plan.args[2], 700)
    q = torch.randn(5, 4, 64, generator=gen(1)).half().cuda()
    out = torch.full((5, 4, 64), 7.0, dtype=F16, device="cuda")
    P.attention_sparse(q, plan.cache, bounds, *plan.args, 3, 5, out=out)
    assert (out[3:] == 7).all() and torch.equal(out[:3], P.attention_cache(q, plan.cache, *plan.args, 3)[:3])
    tables, lens = P.cache_select(q, plan.cache, bounds, *plan.args, 3, 5)
    assert tables[0].tolist() == [[-1] * 5] * 2 and lens.tolist() == [0, 5 * 16 - 4, 3]
    assert all(len(set(t)) == 5 and set(t) <= set(plan.tables[1]) for t in tables[1].tolist())
    # lengths that the table has no room for, and negative ones
    for n in (20000, -3):
        lens = torch.tensor([n, 700, 3], dtype=torch.int32, device="cuda")
        assert torch.isfinite(P.attention_sparse(q, plan.cache, bounds, plan.args[0], plan.args[1], lens, 3, 5)[:3]).all()
    none = P.cache_select(q[:0], plan.cache, bounds, *plan.args, 3, 5)
    assert (none[0] == -1).all() and not none[1].any()


def test_refusals(P):
    cache = P.KVCache.empty(8, 2, 16, 64)
    bounds = P.KeyBounds.empty(cache)
    q = torch.zeros(2, 4, 64, dtype=F16, device="cuda")
    table, lens = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    other = P.KeyBounds.empty(P.KVCache.empty(8, 2, 16, 128))
    wide = torch.zeros(2, 32769, dtype=torch.int32, device="cuda")
    for f in (P.cache_select, P.attention_sparse):
        for args, why in (((q, cache, other, table, None, lens, 1, 4), "bounds"), ((q, cache, bounds, table, None, lens, 1, 1), "keep"), ((q, cache, bounds, table, None, lens, 1, 4, -1), "sinks"),
                          ((q, cache, bounds, table, None, lens, 1, 4, 1, 0), "recent"), ((q, cache, bounds, table, None, lens, 1, 4, 3, 2), "keep"),
                          ((q, cache, bounds, table, None, lens, 1, 0), "keep"), ((q, cache, bounds, table, None, lens, 1, 40000), "keep"), ((q, cache, bounds, wide, None, lens, 1, 4), "32768"),
                          ((q.float(), cache, bounds, table, None, lens, 1, 4), "bfloat16"), ((q, cache, bounds, table.long(), None, lens, 1, 4), "int32"),
                          ((q[:, :3], cache, bounds, table, None, lens, 1, 4), "multiple|aligned|next to"), ((q[..., :32], cache, bounds, table, None, lens, 1, 4), "next to each other"),
                          ((q[..., :32].contiguous(), cache, bounds, table, None, lens, 1, 4), "heads of 32")):
            with pytest.raises(P.SampError, match=why):
                f(*args)
    with pytest.raises(P.SampError, match="scale"):
        P.attention_sparse(q, cache, bounds, table, None, lens, 1, 4, scale=-1.0)
    for args in ((bounds.codes[:, :, :1], bounds.steps), (bounds.codes, bounds.steps[:4]), (bounds.codes.float(), bounds.steps)):
        with pytest.raises(P.SampError):
            P.KeyBounds(*args)
    with pytest.raises(P.SampError, match="bounds"):
        P.cache_bounds(cache, other, table, None, lens, 1)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_beams_of_a_long_context(P, dtype):
    """The operators in turn: a prompt's pages and bounds, then beams that fork it, write, bound the pages they fill and read the pages that promise most."""
    G, H, D, page, W, keep, prompt, steps = 2, 8, 64, 16, 3, 6, 490, 40
    pages = 120
    cache = P.KVCache.empty(pages, G, page, D)
    bounds = P.KeyBounds.empty(cache)
    width = -(-(prompt + steps) // page)
    refs, lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (pages, 1))
    refs, table, lens, _, _ = P.pages_fork(refs, torch.full((1, width), -1, dtype=torch.int32, device="cuda"), lens, page, None, None, prompt)
    k, v = (torch.randn(prompt, G, D, generator=gen(i)).to(dtype) for i in (1, 2))
    P.cache_write(cache, k.cuda(), v.cuda(), table, None, lens, prompt)
    P.cache_bounds(cache, bounds, table, None, lens, prompt)
    held = [[k, v]] * W
    parents = torch.zeros(W, dtype=torch.int32, device="cuda")
    scores = torch.tensor([0.0, -math.inf, -math.inf], device="cuda")
    for step in range(steps):
        refs, table, lens, copies, lacking = P.pages_fork(refs, table, lens, page, parents, None, 1)
        P.cache_copy(cache, copies)
        held = [held[p] if step else held[0] for p in parents.tolist()]
        k, v = (torch.randn(W, G, D, generator=gen(50 + 2 * step + i)).to(dtype) for i in (0, 1))
        P.cache_write(cache, k.cuda(), v.cuda(), table, None, lens, 1)
        P.cache_bounds(cache, bounds, table, None, lens, 1)
        held = [[torch.cat([a, x[i:i + 1]]) for a, x in zip(h, (k, v))] for i, h in enumerate(held)]
        if step == 21:                                       # bounds move with their pages
            refs, table, copies, _ = P.pages_compact(refs, table, page)
            P.cache_copy(cache, copies, bounds)
        q = (torch.randn(W, H, D, generator=gen(step)) * 2).to(dtype)
        o = P.attention_sparse(q.cuda(), cache, bounds, table, None, lens, 1, keep)
        codes, bsteps = bounds.codes.cpu(), bounds.steps.cpu()
        n = prompt + step + 1
        for i, h in enumerate(held):
            dequantised = [(lambda c, s: c * s[..., None])(*quantised(x)) for x in h]
            for j in range(n // page):                       # the page's own bounds, whoever wrote it
                p = int(table[i, j])
                want, s = bounds_definition(cache.k[p, 0].cpu(), cache.k_step[p, 0].cpu()) if step % 13 == 0 else (codes[p, 0], bsteps[p, 0])
                assert torch.equal(codes[p, 0], want) and bsteps[p, 0] == s
            chosen = choose_definition(q[i:i + 1], codes, bsteps, table[i].cpu(), -(-n // page), keep, 1, 1, H, G)
            for g in range(G):
                seen = torch.zeros(1, n, dtype=torch.bool)
                for j in chosen[g]:
                    seen[:, j * page:(j + 1) * page] = True
                heads = slice(g * H // G, (g + 1) * H // G)
                want = attend(q[i:i + 1, heads].double(), dequantised[0][:, g:g + 1], dequantised[1][:, g:g + 1], seen, D ** -0.5)
                check_attention(o[i:i + 1, heads], *want, dtype, F16, n, dequantised[1].abs().max().item())
        scores, parents, _ = (t.flatten() for t in P.beam_select(torch.randn(W, 300, generator=gen(400 + step)).cuda() * 2, scores, W))


def test_sparse_calls_in_graphs_and_on_streams(P):
    plan, bounds, q, _ = run_sparse(P, [3000, 900, 5000], [1, 1, 1], 8, 2, 128, 32, 24, 1, 1, F16, seed=7)
    q = q.cuda()
    call = lambda: P.attention_sparse(q, plan.cache, bounds, plan.args[0], None, plan.args[2], 1, 24)
    call()
    torch.cuda.synchronize()
    graphs, side = [], [torch.cuda.Stream() for _ in range(2)]
    for st in side:
        with torch.cuda.stream(st):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                out = call()
        graphs.append((g, out))
    for seed in range(3):
        q.copy_(torch.randn(3, 8, 128, generator=gen(seed)).half())
        plan.args[2].copy_(torch.tensor([3000 - 700 * seed, 900 - seed, 5000 - 33 * seed], dtype=torch.int32))
        torch.cuda.synchronize()
        for (g, _), st in zip(graphs, side):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        want = call()
        for _, out in graphs:
            assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,G,D,page", [(8, 2, 64, 16), (4, 4, 128, 32), (7, 1, 64, 16)])
@pytest.mark.parametrize("lens,new,most,keep", [([700, 900, 40, 330], [100, 7, 3, 300], 4, 5), ([300], [100], 1, 2), ([9000, 500], [200, 1], 3, 20), ([16 * 400, 600], [16 * 390, 2], 2, 14)])
def test_more_new_tokens_than_the_maximum(P, lens, new, most, keep, H, G, D, page, dtype):
    """Of a sequence with more new tokens than max_new the first max_new rows are computed: they choose among the pages up to their own and see what attention_cache's rows see of them."""
    plan = Plan(P, lens, new, G, D, page, seed=H)
    k, v = (torch.randn(sum(lens), G, D, generator=gen(i)).to(dtype) for i in (1, 2))
    q = (torch.randn(plan.total, H, D, generator=gen(3)) * 1.5).to(dtype)
    start = offsets(lens)
    P.cache_write(plan.cache, k.cuda(), v.cuda(), plan.args[0], start.cuda(), plan.args[2], max(lens))
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], start.cuda(), plan.args[2], max(lens))
    sinks, recent = 0 if keep == 2 else 1, (most + page - 2) // page + 1
    tables, short = P.cache_select(q.cuda(), plan.cache, bounds, *plan.args, most, keep, sinks, recent)
    out = torch.full((plan.total, H, D), 7.0, dtype=dtype, device="cuda")
    P.attention_sparse(q.cuda(), plan.cache, bounds, *plan.args, most, keep, sinks, recent, out=out)
    whole = P.attention_cache(q.cuda(), plan.cache, *plan.args, most)
    codes, steps = bounds.codes.cpu(), bounds.steps.cpu()
    for b, (n, m) in enumerate(zip(lens, new)):
        at, todo, pages = int(plan.cu[b]), min(m, most), -(-n // page)
        if pages > keep:
            pages = -(-(n - m + todo) // page)
        chosen = choose_definition(q[at:at + todo], codes, steps, plan.table[b], pages, keep, sinks, recent, H, G)
        assert int(short[b]) == n - (pages - min(pages, keep)) * page
        for g in range(G):
            want = [int(plan.table[b, j]) for j in chosen[g]]
            assert tables[b, g].tolist() == want + [-1] * (keep - len(want)), (b, g)
        assert (out[at + todo:at + m] == 7).all()
        held = [(lambda c, s: c * s[..., None])(*quantised(x[int(start[b]):int(start[b]) + n])) for x in (k, v)]
        seen = torch.arange(n)[None, :] <= n - m + torch.arange(todo)[:, None]
        for g in range(G):
            of = torch.zeros(n, dtype=torch.bool)
            for j in chosen[g]:
                of[j * page:(j + 1) * page] = True
            heads = slice(g * H // G, (g + 1) * H // G)
            want = attend(q[at:at + todo, heads].double(), held[0][:, g:g + 1], held[1][:, g:g + 1], seen & of, D ** -0.5)
            check_attention(out[at:at + todo, heads], *want, dtype, F16, n, held[1].abs().max().item())
            if pages <= keep:
                check_attention(whole[at:at + todo, heads], *want, dtype, F16, n, held[1].abs().max().item())


@pytest.mark.parametrize("pages", [40, 256, 257, 600])
def test_holes_of_a_sequence_without_new_tokens(P, pages):
    """Without new tokens all pages score minus infinity, those that are none of the cache's too: the earlier ones are kept, however many pages there are."""
    page, G, D, keep = 16, 2, 64, 9
    plan = Plan(P, [16 * pages, 16 * pages - 5], [0, 1], G, D, page)
    plan.fill(P, F16, 3)
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], None, plan.args[2], 16 * pages)
    table = plan.args[0].clone()
    holes = [3, 7, pages // 2, pages - 9]
    table[:, holes] = -1
    q = torch.randn(1, 4, D, generator=gen(5)).half()
    tables, lens = P.cache_select(q.cuda(), plan.cache, bounds, table, *plan.args[1:], 1, keep, 1, 2)
    for b in range(2):
        want = choose_definition(q[:b], bounds.codes.cpu(), bounds.steps.cpu(), table[b].cpu(), pages, keep, 1, 2, 4, G)
        assert int(lens[b]) == 16 * pages - 5 * b - (pages - keep) * page
        for g in range(G):
            assert tables[b, g].tolist() == [int(table[b, j]) for j in want[g]], (b, g)
        if b == 0:
            assert want[0] == [0, 1, 2, 3, 4, 5, 6, pages - 2, pages - 1]


@pytest.mark.parametrize("pages", [40, 300])
def test_scores_that_are_zeros_of_either_sign_are_equal(P, pages):
    """Steps so small that the products of some pages are zeros, some of them negative ones: equal scores, of which the earlier pages are kept."""
    page, G, D, keep = 16, 2, 64, 9
    plan = Plan(P, [16 * pages], [1], G, D, page)
    plan.fill(P, BF16, 3)
    bounds = P.KeyBounds(torch.randint(-127, 128, (plan.cache.pages, G, 2, D), generator=gen(1), dtype=torch.int8).cuda(), torch.full((plan.cache.pages, G), 1e-38, device="cuda"))
    q = (torch.randn(1, 4, D, generator=gen(5)) * 1e-15).bfloat16()
    tables, _ = P.cache_select(q.cuda(), plan.cache, bounds, *plan.args, 1, keep, 1, 2)
    want = choose_definition(q, bounds.codes.cpu(), bounds.steps.cpu(), plan.table[0], pages, keep, 1, 2, 4, G)
    assert want == [[0, 1, 2, 3, 4, 5, 6, pages - 2, pages - 1]] * G
    assert tables[0].tolist() == [[int(plan.table[0, j]) for j in want[g]] for g in range(G)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,new,page,keep", [([9000, 70, 20000, 4000], [1, 1, 1, 1], 16, 100), ([30000] * 3 + [900, 2000], [1] * 5, 64, 32), ([5001, 700, 1500], [5, 5, 2], 32, 20)])
def test_calls_repeat_themselves(P, lens, new, page, keep, dtype):
    """The same inputs give the same bits: again, after other memory's use for the workspace, beside another stream's work, and from a copy of all tensors."""
    H, G, D = 16, 4, 128
    plan = Plan(P, lens, new, G, D, page, 3)
    k, v = (torch.randn(sum(lens), G, D, generator=gen(i)).to(dtype).cuda() for i in (1, 2))
    q = (torch.randn(plan.total, H, D, generator=gen(3)) * 1.5).to(dtype).cuda()
    P.cache_write(plan.cache, k, v, plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens))
    bounds = P.KeyBounds.empty(plan.cache)
    P.cache_bounds(plan.cache, bounds, plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens))
    copy = P.KVCache(*(t.clone() for t in (plan.cache.k, plan.cache.v, plan.cache.k_step, plan.cache.v_step)))
    both = P.KeyBounds(bounds.codes.clone(), bounds.steps.clone())
    call = lambda c=plan.cache, b=bounds, x=q: P.attention_sparse(x, c, b, *plan.args, max(new), keep)
    want, chosen = call(), P.cache_select(q, plan.cache, bounds, *plan.args, max(new), keep)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(6):
        junk = torch.full((1 << 22,), math.nan, device="cuda")
        del junk
        with torch.cuda.stream(side):
            other = [call(copy, both) for _ in range(3)]
        got = [call(), call(copy, both, q.clone()), call()]
        again = P.cache_select(q, copy, both, *plan.args, max(new), keep)
        torch.cuda.synchronize()
        assert all(torch.equal(x, want) for x in got + other) and all(torch.equal(a, b) for a, b in zip(chosen, again)), i
