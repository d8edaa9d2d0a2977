"""The bookkeeping of pages (fork, compact, copies) against its definition, one entry after the other on the CPU.  Everything is whole numbers and copies: equal to the bit."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from test_gpu_decoder import F16, P, attend, check_attention, gen, offsets, quantised  # noqa: E402,F401


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def fork_definition(refs, table, lens, page_len, parents, new):
    """samp.h's text, sequentially: refs list, table list of lists, parents and new lists."""
    refs, pages, width = list(refs), len(refs), len(table[0])
    ok = lambda p: 0 <= p < pages
    for row in table:
        for p in row:
            if ok(p):
                refs[p] -= 1
    plans, out = [], []
    for p, n in zip(parents, new):
        alive = 0 <= p < len(table)
        held = max(lens[p], 0) if alive else 0
        n = max(n, 0) if alive else 0
        end = -(-(held + n) // page_len)
        first = held // page_len if n else end
        row = [table[p][j] if alive and j < end and ok(table[p][j]) else -1 for j in range(width)]
        for x in row:
            if x >= 0:
                refs[x] += 1
        plans.append((held, n, first, end))
        out.append(row)
    writers = {}
    for i, (held, n, first, end) in enumerate(plans):
        for j in range(first, min(end, width)):
            if out[i][j] >= 0:
                writers.setdefault(out[i][j], []).append((i, j))
    free = [p for p in range(pages) if refs[p] == 0]
    copies, lacking = [[-1] * len(parents), [-1] * len(parents), [0] * len(parents)], 0
    total = {p: refs[p] for p in writers}
    for i, (held, n, first, end) in enumerate(plans):
        lacking += max(0, end - max(first, width)) if n else 0
        for j in range(first, min(end, width)):
            x = out[i][j]
            if x >= 0 and len(writers[x]) == total[x] and writers[x][0] == (i, j):
                continue
            if x >= 0:
                refs[x] -= 1
            if free:
                to = free.pop(0)
                refs[to] = 1
                if x >= 0 and j == first and held % page_len:
                    copies[0][i], copies[1][i], copies[2][i] = x, to, held % page_len
            else:
                to = -1
                lacking += 1
            out[i][j] = to
    return refs, out, [held + n for held, n, _, _ in plans], copies, [lacking]


def check_fork(P, refs, table, lens, page_len, parents, new):
    """parents None or a list; new a number or a list."""
    who = list(range(len(table))) if parents is None else parents
    each = [new] * len(who) if isinstance(new, int) else new
    want = fork_definition(refs, table, lens, page_len, who, each)
    cu = None if isinstance(new, int) else offsets(new).cuda()
    got = P.pages_fork(ints(refs).cuda(), ints(table).cuda(), ints(lens).cuda(), page_len, None if parents is None else ints(parents).cuda(), cu,
                       new if isinstance(new, int) else 0)
    for name, a, b in zip(("refs", "table", "lens", "copies", "lacking"), got, want):
        assert torch.equal(a.cpu(), ints(b)), (name, a.cpu(), ints(b))
    return got


def state(rows, width, page_len, pages, seed, shared=0.5, spare=0):
    """Rows of different lengths: pages of a row before it at random, then its own; refs count them."""
    g = gen(seed)
    rand = lambda n: int(torch.randint(0, n, (1,), generator=g))
    order = torch.randperm(pages, generator=g).tolist()
    table, lens = [], []
    for i in range(rows):
        n = rand((width - spare) * page_len + 1)
        need = -(-n // page_len)
        row = []
        if i and torch.rand(1, generator=g) < shared:
            row = table[rand(i)][: rand(need + 1)]
            row = [p for p in row if p >= 0]
        while len(row) < need and order:
            row.append(order.pop())
        n = min(n, len(row) * page_len)
        table.append(row + [-1] * (width - len(row)))
        lens.append(n)
    refs = [0] * pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    return refs, table, lens


SIZES = [(1, 1, 16, 1), (4, 3, 16, 9), (7, 5, 32, 40), (33, 9, 16, 300), (130, 17, 64, 2000), (300, 6, 16, 1000)]
LARGE = [(5, 4, 16, 40000), (150, 40, 16, 30000), (8192, 2, 16, 17000), (1000, 70, 16, 9000)]


@pytest.mark.parametrize("rows,width,page_len,pages", SIZES + LARGE)
def test_pages_fork(P, rows, width, page_len, pages):
    for seed in range(2 if pages > 10000 else 5):
        g = gen(100 + seed)
        refs, table, lens = state(rows, width, page_len, pages, seed, spare=seed % 2)
        parents = torch.randint(-1, rows, (rows,), generator=g).tolist()
        check_fork(P, refs, table, lens, page_len, parents, 1)
        check_fork(P, refs, table, lens, page_len, None, 1)
        check_fork(P, refs, table, lens, page_len, parents, 0)
        more = torch.randint(-1, rows + 3, (min(2 * rows, 8192),), generator=g).tolist()      # more rows than there were, some from none
        check_fork(P, refs, table, lens, page_len, more, torch.randint(0, 3 * page_len, (len(more),), generator=g).tolist())
        check_fork(P, refs, table, lens, page_len, parents[: max(1, rows // 3)], page_len + 1)


@pytest.mark.parametrize("pages", [60, 40000])
def test_fork_of_tables_with_holes_and_pages_behind_the_end(P, pages):
    """Positions that were taken back leave pages behind the end, which a row keeps if it is the only one; numbers that are no pages count as holes."""
    table = [[5, 6, 7, 8, -1, -1], [5, 6, 9, 10 ** 6, 11, -1], [-7, 12, -1, 13, 14, 15], [-1] * 6]
    refs = [0] * pages
    for row in table:
        for p in row:
            if 0 <= p < pages:
                refs[p] += 1
    for lens in ([20, 33, 40, 0], [64, 80, 96, 0], [0, 1, 16, 5], [-4, 1000, 50, 0]):
        for parents in (None, [0, 0, 1, 1], [3, 2, 2, -1], [1], [-1, -1], [2, 0, 1, 3, 0, 9]):
            n = 4 if parents is None else len(parents)
            for new in (0, 1, 17, 60, [(7 * i) % 40 for i in range(n)]):
                check_fork(P, refs, table, lens, 16, parents, new)
    # other holders than the table's: a page of theirs is copied before it is written, and none is ever free
    for p in (7, 30):
        refs[p] += 1
    check_fork(P, refs, table, [40, 33, 40, 0], 16, None, 1)
    check_fork(P, refs, table, [40, 33, 40, 0], 16, [0, 0, 0, -1], 20)


@pytest.mark.parametrize("pages", [4000, 30000])
@pytest.mark.parametrize("rows", [1, 17, 70, 1100])
def test_fork_of_rows_that_write_few_and_many_entries(P, rows, pages):
    """Rows of one wave go on by nothing, one token, a few pages and most of a table, over pages that others name too."""
    width, page_len = 40, 16
    held = [(13 * i) % 90 for i in range(rows)]
    table, refs = [], [0] * pages
    for i in range(rows):
        table.append([(7 * (i // 3) + j) % pages if j < 8 and (i + j) % 11 else -1 for j in range(width)])
        for p in table[-1]:
            if p >= 0:
                refs[p] += 1
    parents = [min(rows - 1, i // 8 * 8 + (5 * i) % 8) for i in range(rows)]
    for new in (20, 100, [(0, 1, 20, 70, 500, 3)[(i + i // 16) % 6] for i in range(rows)], [500 if i % 64 == 5 else i % 2 for i in range(rows)]):
        check_fork(P, refs, table, held, page_len, parents, new)
        check_fork(P, refs, table, held, page_len, None, new)


@pytest.mark.parametrize("pages,rows", [(50, 6), (20000, 6)])
def test_fork_says_how_many_pages_are_lacking(P, pages, rows):
    refs, table, lens = state(rows, 4, 16, pages, 1)
    taken = [max(r, 1) for r in refs]                        # nothing is free
    _, out, _, _, lacking = check_fork(P, taken, table, lens, 16, [0, 0, 1, 2, 3, 4], 5)
    check_fork(P, taken[:-3] + refs[-3:], table, lens, 16, [0, 0, 1, 2, 3, 4], 40)
    assert int(lacking) > 0 and (out == -1).any()
    check_fork(P, refs, table, [64] * rows, 16, None, 100)   # the table is too narrow
    # the largest numbers that an int32 holds
    got = P.pages_fork(ints(refs).cuda(), ints(table).cuda(), ints([2 ** 31 - 1] * rows).cuda(), 16, None, offsets([2 ** 31 - 1] + [0] * (rows - 1)).cuda())
    assert got[2].tolist() == [2 ** 31 - 1] * rows and int(got[4]) > 0
    # sums of such numbers, and one past an int32
    width = 5
    for n in (1, 15, 16, 40):
        got = P.pages_fork(ints([0] * pages).cuda(), torch.full((n, width), -1, dtype=torch.int32, device="cuda"), ints([0] * n).cuda(), 16, None, None, 2 ** 31 - 1)
        assert int(got[4]) == min(2 ** 31 - 1, max(n * width - pages, 0) + n * (2 ** 27 - width)) and got[2].tolist() == [2 ** 31 - 1] * n
    # counts that are not the tables': no access outside the buffers, every entry a page or -1
    got = P.pages_fork(ints([0] * pages).cuda(), ints(table).cuda(), ints(lens).cuda(), 16, ints([0] * rows).cuda(), None, 33)
    assert ((got[1] >= -1) & (got[1] < pages)).all()


def compact_definition(refs, table, page_len):
    pages = len(refs)
    used = sum(r > 0 for r in refs)
    moves = list(zip([p for p in range(used, pages) if refs[p] > 0], [p for p in range(used) if refs[p] <= 0]))
    where = {p: p for p in range(used) if refs[p] > 0}
    where.update(moves)
    out = [0] * pages
    for p, to in where.items():
        out[to] = refs[p]
    n = max(1, pages // 2)
    copies = [[a for a, _ in moves] + [-1] * (n - len(moves)), [b for _, b in moves] + [-1] * (n - len(moves)), [page_len] * len(moves) + [0] * (n - len(moves))]
    return out, [where.get(p, -1) for p in table], copies, [used]


@pytest.mark.parametrize("pages", [1, 2, 63, 64, 65, 128, 301, 5000, 65536, 65537, 200000])
def test_pages_compact(P, pages):
    for seed, share in enumerate((0.0, 0.1, 0.5, 0.9, 1.0)):
        g = gen(pages + seed)
        refs = torch.where(torch.rand(pages, generator=g) < share, torch.randint(1, 5, (pages,), generator=g), 0)
        refs[torch.rand(pages, generator=g) < 0.02] = -3     # counts that no table gives
        table = torch.randint(-2, pages + 2, (7, 13), generator=g).to(torch.int32)
        want = compact_definition(refs.tolist(), table.flatten().tolist(), 32)
        got = P.pages_compact(refs.to(torch.int32).cuda(), table.cuda(), 32)
        for name, a, b in zip(("refs", "table", "copies", "used"), got, want):
            assert torch.equal(a.cpu().flatten(), ints(b).flatten()), name
        assert got[1].shape == table.shape and got[2].shape == (3, max(1, pages // 2))
    assert P.pages_compact(refs.to(torch.int32).cuda(), table[:0].cuda(), 32)[1].shape == (0, 13)
    big = torch.randint(0, pages, (70001,), generator=g).to(torch.int32)               # more entries than one block takes
    want = compact_definition(refs.tolist(), big.tolist(), 32)
    for a, b in zip(P.pages_compact(refs.to(torch.int32).cuda(), big.cuda(), 32), want):
        assert torch.equal(a.cpu().flatten(), ints(b).flatten())


def test_bookkeeping_of_the_most_pages(P):
    pages = 1 << 26
    refs = (torch.rand(pages, device="cuda") < 0.3).int() * torch.randint(1, 5, (pages,), dtype=torch.int32, device="cuda")
    used = refs.nonzero().flatten().int()
    n = used.numel()
    refs_out, table_out, copies, count = P.pages_compact(refs, used, 16)
    stay = int((used < n).sum())
    assert int(count) == n and not refs_out[n:].any() and torch.equal(refs_out[table_out.long()], refs[used.long()])
    assert torch.equal(table_out[:stay], used[:stay]) and torch.equal(copies[0, : n - stay], used[stay:]) and torch.equal(copies[1, : n - stay], table_out[stay:])
    assert torch.equal(copies[1, : n - stay], (refs[:n] == 0).nonzero().flatten().int()) and (copies[:2, n - stay:] == -1).all() and not copies[2, n - stay:].any()
    # two rows of 3 million entries, which go on into as many free pages
    width = 3_000_000
    table = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    fresh, out, lens, _, lacking = P.pages_fork(refs, table, ints([0, 0]).cuda(), 16, None, None, 16 * width)
    assert torch.equal(out.flatten(), (refs == 0).nonzero().flatten()[: 2 * width].int()) and lens.tolist() == [16 * width] * 2 and int(lacking) == 0
    want = refs.clone()
    want[out.flatten().long()] = 1
    assert torch.equal(fresh, want)


@pytest.mark.parametrize("G,D,page", [(1, 64, 16), (12, 64, 32), (8, 128, 64), (3, 128, 1024), (2, 64, 256)])
def test_cache_copy(P, G, D, page):
    pages, g = 21, gen(D + page)
    data = [torch.randint(-127, 128, (pages, G, page, D), generator=g, dtype=torch.int8) for _ in range(2)] + [torch.rand(pages, G, page, generator=g) for _ in range(2)]
    kb = torch.randint(-127, 128, (pages, G, 2, D), generator=g, dtype=torch.int8), torch.rand(pages, G, generator=g)
    copies = torch.tensor([[3, 4, 3, -1, 2, 25, 7, 8, 9, 0], [10, 11, 12, 13, -1, 14, 40, 15, 9, 20], [page, 1, page - 1, 5, 5, 5, 5, 0, 3, 2 ** 31 - 1]], dtype=torch.int32)
    for with_bounds in (False, True):
        cache = P.KVCache(*(t.cuda() for t in data))
        bounds = P.KeyBounds(*(t.cuda() for t in kb))
        P.cache_copy(cache, copies.cuda(), bounds if with_bounds else None)
        want, want_b = [t.clone() for t in data], [t.clone() for t in kb]
        for a, b, n in ((3, 10, page), (4, 11, 1), (3, 12, page - 1), (0, 20, page)):
            for t in want:
                t[b, :, :n] = t[a, :, :n]
            if with_bounds:
                for t in want_b:
                    t[b] = t[a]
        for got, t in zip((cache.k, cache.v, cache.k_step, cache.v_step, bounds.codes, bounds.steps), want + want_b):
            assert torch.equal(got.cpu(), t)
    P.cache_copy(cache, copies[:, :0].cuda())


def test_copies_pass_32_bits(P):
    """Pages whose codes lie more than 2^31 bytes apart, and more copies than there are waves."""
    G, D, page = 8, 128, 256
    pages = (1 << 31) // (G * page * D) + 20
    cache = P.KVCache(*(torch.zeros((pages, G, page, D), dtype=torch.int8, device="cuda") for _ in range(2)),
                      *(torch.zeros((pages, G, page), device="cuda") for _ in range(2)))
    cache.k[1], cache.v_step[1] = 7, 2.5
    copies = torch.full((3, 70000), -1, dtype=torch.int32)
    copies[:, 0], copies[:, 69999] = ints([1, pages - 1, page]), ints([1, pages - 2, 9])
    P.cache_copy(cache, copies.cuda())
    assert (cache.k[pages - 1] == 7).all() and (cache.v_step[pages - 1] == 2.5).all()
    assert (cache.k[pages - 2, :, :9] == 7).all() and not cache.k[pages - 2, :, 9:].any() and not cache.k[2: pages - 2].any()


def test_refusals(P):
    t = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    r, n = torch.zeros(10, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for args, why in (((r.long(), t, n, 16), "int32"), ((r, t.t(), n, 16), "contiguous"), ((r, t[0], n, 16), "page table"), ((r, t, r, 16), "elements"), ((r, t, n, 20), "power of two"),
                      ((r, t, n, 16, r[:0]), "rows"), ((r, t, n, 16, torch.zeros(9000, dtype=torch.int32, device="cuda")), "8192"), ((r, t, n, 16, None, n), "elements"),
                      ((r, t, n, 16, None, None, -1), "max_new"), ((r[:0], t, n, 16), "pages")):
        with pytest.raises(P.SampError, match=why):
            P.pages_fork(*args)
    for args, why in (((r.float(), t, 16), "int32"), ((r, t.float(), 16), "int32"), ((r, t, 0), "power of two"), ((r[:0], t, 16), "pages")):
        with pytest.raises(P.SampError, match=why):
            P.pages_compact(*args)
    cache = P.KVCache.empty(10, 2, 16, 64)
    for args, why in (((cache, t), "3, n"), ((cache, torch.zeros(3, 4, device="cuda")), "int32"), ((cache, torch.zeros(3, 4, dtype=torch.int32, device="cuda"),
                       P.KeyBounds.empty(P.KVCache.empty(9, 2, 16, 64))), "bounds")):
        with pytest.raises(P.SampError, match=why):
            P.cache_copy(*args)


# ---- as they are used --------------------------------------------------------------------------------
@pytest.mark.parametrize("D,G,H,page", [(64, 2, 4, 16), (128, 1, 8, 32)])
def test_beam_search_over_a_paged_cache(P, D, G, H, page):
    """Prompts, then steps of beam search with random logits: after each step every beam's context is what its ancestors wrote, pages are counted right, and nothing leaks; in
    between the pages are moved together."""
    lens0, W, V, steps, pages = [37, 5, page * 2], 4, 500, 2 * page + 5, 80
    B = len(lens0)
    cache = P.KVCache.empty(pages, G, page, D)
    width = -(-(max(lens0) + steps) // page) + 1
    refs, table, lens = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((pages,), (B, width), (B,)))
    table.fill_(-1)
    refs, table, lens, copies, lacking = P.pages_fork(refs, table, lens, page, None, offsets(lens0).cuda())
    assert lens.tolist() == lens0 and int(lacking) == 0 and (copies[1] == -1).all()
    k, v = (torch.randn(sum(lens0), G, D, generator=gen(i)).half() for i in (1, 2))
    P.cache_write(cache, k.cuda(), v.cuda(), table, offsets(lens0).cuda(), lens, max(lens0))
    held = [[a[i:j] for a in (k, v)] for i, j in zip(offsets(lens0).tolist(), offsets(lens0).tolist()[1:])]
    held = [h for h in held for _ in range(W)]                         # per beam: its keys and values so far
    parents = torch.arange(B * W, dtype=torch.int32, device="cuda") // W
    scores = torch.where(torch.arange(B * W) % W == 0, 0.0, -float("inf")).cuda()
    finished = torch.zeros(B * W, dtype=torch.uint8, device="cuda")
    for step in range(steps):
        refs, table, lens, copies, lacking = P.pages_fork(refs, table, lens, page, parents, None, 1)
        assert int(lacking) == 0
        P.cache_copy(cache, copies)
        if step:
            held = [held[p] for p in parents.tolist()]
        k, v = (torch.randn(B * W, G, D, generator=gen(10 + 2 * step + i)).half() for i in (0, 1))
        P.cache_write(cache, k.cuda(), v.cuda(), table, None, lens, 1)
        held = [[torch.cat([a, x[i:i + 1]]) for a, x in zip(h, (k, v))] for i, h in enumerate(held)]
        if step % 7 == 3:
            refs, table, copies, used = P.pages_compact(refs, table, page)
            P.cache_copy(cache, copies)
            assert (refs[: int(used)] > 0).all() and not refs[int(used):].any()
        names = torch.bincount(table[table >= 0].long(), minlength=pages)
        assert torch.equal(names.to(torch.int32), refs)
        assert (table >= 0).sum(1).tolist() == [-(-h[0].shape[0] // page) for h in held]
        last = [(n - 1) // page for n in lens.tolist()]
        assert len({int(table[i, j]) for i, j in enumerate(last)}) == B * W             # nobody writes a page that another holds
        rows = [h[0].shape[0] for h in held]
        got = P.cache_read(cache, table, offsets(rows).cuda(), lens, max(rows), sum(rows), F16)
        for a, i in zip(got, (0, 1)):
            c, s = quantised(torch.cat([h[i] for h in held]))
            assert torch.equal(a.cpu(), (c * s[..., None]).float().half())
        if step % 10 == 0:
            q = torch.randn(B * W, H, D, generator=gen(step)).half()
            o = P.attention_cache(q.cuda(), cache, table, None, lens, 1)
            for i, h in enumerate(held):
                kk, vv = ((lambda c, s: c * s[..., None])(*quantised(x)) for x in h)
                check_attention(o[i:i + 1], *attend(q[i:i + 1].double(), kk, vv, torch.ones(1, rows[i], dtype=torch.bool), D ** -0.5), F16, F16, rows[i], vv.abs().max().item())
        logits = torch.randn(B * W, V, generator=gen(1000 + step)).cuda() * 3
        scores, parents, tokens = (t.flatten() for t in P.beam_select(logits, scores, W, finished=finished, end=3))
        finished = (finished[parents.long()].bool() | (tokens == 3)).to(torch.uint8)
    # the sequences are released
    refs, table, lens, copies, lacking = P.pages_fork(refs, table, lens, page, torch.full((B * W,), -1, dtype=torch.int32, device="cuda"))
    assert not refs.any() and (table == -1).all() and not lens.any() and (copies[:2] == -1).all()


def test_bookkeeping_in_graphs(P):
    """Captured once, replayed on new inputs: counts and tables come out as from the calls."""
    refs, table, lens = state(60, 8, 16, 700, 3)
    for pages in (700, 8000, 30000):                         # one block, with more LDS than a launch has by itself, several kernels
        dev = [ints(refs + [0] * (pages - 700)).cuda(), ints(table).cuda(), ints(lens).cuda(), torch.zeros(60, dtype=torch.int32, device="cuda")]

        def step():
            out = P.pages_fork(*dev[:3], 16, dev[3], None, 3)
            return out + P.pages_compact(out[0], out[1], 16)

        step()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = step()
        for seed in range(3):
            dev[3].copy_(torch.randint(-1, 60, (60,), generator=gen(seed)))
            torch.cuda.synchronize()
            g.replay()
            want = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
