"""Beam search's selection against its definition in binary64, on the CPU.

A total is a score plus a logit less the row's log-sum-exp, formed in binary64 from sums of exponentials in binary32.  In units of 2^-24, relative to a sum: an exponential has a step (2); its argument
t, in powers of two, is rounded, |t| ln 2 with a mean under the softmax of at most log2(vocabulary) <= 19 (13.2), and log2(e) in it is 1.34e-8 off (3); a thread adds 16 in a row (15), then
there are two additions, six over the wave and three over the waves (11), and a wave's sum is scaled by a power with a step of its own (3).  So a log-sum-exp is off by less than 48 * 2^-24, and the result
is rounded to binary32 once.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from test_gpu_decoder import F16, BF16, P, gen  # noqa: E402,F401

F32 = torch.float32
LSE = 48 * 2.0 ** -24


def totals(logits, scores, finished, end):
    """Per row {token: total} as a float64 tensor over the vocabulary (a finished row: its score at place 0), minus infinity for no candidate."""
    x, s = logits.double(), scores.double()
    t = s[:, None] + (x - torch.logsumexp(x, 1, keepdim=True))
    bad = ~torch.isfinite(s) | torch.isnan(x).any(1) | (x == math.inf).any(1)
    t[bad] = -math.inf
    t[torch.isnan(t)] = -math.inf                            # (a row of minus infinities)
    if finished is not None:
        for r in finished.nonzero().flatten().tolist():
            t[r] = -math.inf
            t[r, 0] = s[r] if math.isfinite(s[r]) else -math.inf
    return t


def check(P, logits, scores, beams, keep=None, finished=None, end=7, device=None):
    """Everything that the definition says: the tokens of a row in the row's order without a gap, the list in order, nothing better left out."""
    x = (logits if device is None else device)
    got = P.beam_select(x.cuda(), scores.cuda(), beams, keep, None if finished is None else finished.cuda(), end)
    best, parents, tokens = (t.cpu() for t in got)
    keep = keep or beams
    t = totals(logits, scores, finished, end)
    B = logits.shape[0] // beams
    assert best.shape == parents.shape == tokens.shape == (B, keep)
    for b in range(B):
        mine = t[b * beams:(b + 1) * beams]
        n = min(keep, int((mine > -math.inf).sum()))
        assert (parents[b, n:] == -1).all() and (tokens[b, n:] == -1).all() and (best[b, n:] == -math.inf).all()
        used = {}
        for i in range(n):
            r, v = int(parents[b, i]), int(tokens[b, i])
            assert b * beams <= r < (b + 1) * beams
            if finished is not None and finished[r]:
                assert v == end and best[b, i] == scores[r]
                v = 0
            row = used.setdefault(r, [])
            row.append(v)
            off = abs(best[b, i].double() - t[r, v]).item()
            assert off <= LSE + 2.0 ** -24 * abs(t[r, v].item()) * 1.01, (b, i, r, v, off)
        left = mine.clone()
        for r, row in used.items():
            order = torch.sort(logits[r].double(), descending=True, stable=True).indices if finished is None or not finished[r] else torch.tensor([0])
            assert order[: len(row)].tolist() == row, (b, r)
            left[r - b * beams, row] = -math.inf
        if n:
            assert (best[b, : n - 1] >= best[b, 1:n]).all()
            assert left.max() <= best[b, n - 1].double() + LSE * 2 + 2.0 ** -24 * abs(best[b, n - 1].item())
    return best, parents, tokens


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("B,W,V,keep", [(1, 1, 1, 1), (1, 1, 5, 3), (2, 3, 7, 10), (1, 4, 1000, 4), (3, 2, 4095, 64), (2, 5, 4096, 5), (1, 1, 4097, 2), (3, 4, 21128, 8), (40, 4, 32000, 8),
                                        (2, 64, 300, 64), (130, 3, 17001, 6), (1, 2, 1 << 19, 4), (65, 8, 33001, 16),
                                        (1, 13, 1 << 19, 64), (1, 30, 1 << 19, 64), (2, 16, 128256, 32)])                   # long lists in the join, of more LDS than a launch has by itself
def test_beam_select(P, B, W, V, keep, dtype):
    g = gen(B + W + V)
    x = (torch.randn(B * W, V, generator=g) * 3).to(dtype)
    scores = -10 * torch.rand(B * W, generator=g)
    check(P, x, scores, W, keep)
    finished = torch.rand(B * W, generator=g) < 0.3
    x[torch.rand(B * W, V, generator=g) < 0.1] = -math.inf
    if W > 1:
        scores[1::W] = -math.inf
    check(P, x, scores, W, keep, finished)
    check(P, x, scores, W, keep, finished.to(torch.uint8), end=-3)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_equal_logits_take_the_lowest_row_then_token(P, dtype):
    """Rows of one value, in all pieces of a row; and the two zeros, which are equal."""
    x = torch.zeros(4, 40000, dtype=dtype)
    best, parents, tokens = check(P, x, torch.zeros(4), 2, 5)
    assert parents.tolist() == [[0] * 5, [2] * 5] and tokens.tolist() == [[0, 1, 2, 3, 4]] * 2
    x[:, ::2] = -0.0
    best, parents, tokens = check(P, x, torch.zeros(4), 2, 5)
    assert parents.tolist() == [[0] * 5, [2] * 5] and tokens.tolist() == [[0, 1, 2, 3, 4]] * 2
    x = (torch.randn(1, 30000, generator=gen(3)) * 2).to(dtype).repeat(3, 1)              # beams that are alike
    best, parents, tokens = check(P, x, torch.tensor([-1.0, -1.0, -1.0]), 3, 9)
    order = torch.sort(x[0].double(), descending=True, stable=True).indices
    want, i = [], 0
    while len(want) < 9:                                     # equal logits of a row count as equal totals: all of the first row, then of the next
        same = [v for v in order[:64].tolist() if x[0, v] == x[0, order[i]]]
        want += [(r, v) for r in range(3) for v in same]
        i += len(same)
    assert list(zip(parents[0].tolist(), tokens[0].tolist())) == want[:9]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,V", [(4, 1000), (4, 33001), (260, 45003)])
def test_few_tokens_above_many_of_one_value(P, dtype, rows, V):
    """Masks that leave some tokens and set the others to one finite value: those behind the best are the first of the masked ones.  And few values in all."""
    g = gen(V)
    mask = {F16: torch.finfo(F16).min, BF16: -1e4, F32: torch.finfo(F32).min}[dtype]
    x = torch.full((rows, V), mask, dtype=dtype)
    for r in range(rows):
        allowed = torch.randint(0, V, (r % 12,), generator=g)
        x[r, allowed] = torch.randn(len(allowed), generator=g).to(dtype)
    check(P, x, -torch.rand(rows, generator=g), 4, 8)
    check(P, x, -torch.rand(rows, generator=g), 2, 64)
    check(P, torch.randint(-2, 3, (rows, V), generator=g).to(dtype), -torch.rand(rows, generator=g), 4, 16)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_logits_that_rise_or_fall_all_along(P, dtype):
    """The best of a row lie next to each other: in one thread's registers, or in one after the other's."""
    for V in (900, 16384, 33001):
        x = torch.arange(V).double()
        x = torch.stack([x, x.flip(0), (x / 8).floor() * 8, x % 97]) * (60.0 / V)
        check(P, x.to(dtype), torch.tensor([0.0, -0.1, -0.2, -0.3]), 4, 64)
        check(P, x.to(dtype), torch.tensor([0.0, -0.1, -0.2, -0.3]), 1, 17)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_rows_without_candidates_and_values_at_the_ends(P, dtype):
    V = 5000
    low, top = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.randn(12, V, generator=gen(1)).to(dtype)
    x[0, 77] = math.nan
    x[1, 4999] = -math.nan
    x[2, 0] = math.inf
    x[3] = -math.inf
    x[4] = -math.inf
    x[4, 4321] = 0.5                                         # one token is left
    x[5] = low                                               # all of them masked by the type's lowest value
    x[6, 10:] = low
    x[7] = 2.0 ** -14
    x[8, 17] = top
    scores = torch.linspace(-3, -1, 12)
    scores[9], scores[10] = math.inf, math.nan
    check(P, x, scores, 1, 3)
    check(P, x, scores, 4, 8)
    check(P, x, scores, 12, 16)
    best, _, tokens = check(P, x[4:6], scores[4:6], 1, 2)
    assert tokens[0].tolist() == [4321, -1] and best[0, 0] == scores[4] and tokens[1].tolist() == [0, 1]
    none = P.beam_select(x[:4].cuda(), scores[:4].cuda(), 4)
    assert (none[0] == -math.inf).all() and (none[1] == -1).all() and (none[2] == -1).all()
    finished = torch.ones(12, dtype=torch.bool)
    best, parents, tokens = check(P, x, scores, 4, 3, finished, end=2)       # logits of finished rows are not looked at
    assert parents[0].tolist() == [3, 2, 1]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_of_any_size(P, dtype):
    """Logits whose product with log2(e) has no fraction left, up to the type's largest: differences decide."""
    V = 9000
    x = torch.randn(10, V, generator=gen(1))
    for r, e in enumerate((20, 23, 24, 25, 30, 40, 80, 120, 125, 126)):
        x[r] = x[r] * 3 + 2.0 ** e if e < 25 else (x[r].abs().clamp(max=1.9)) * 2.0 ** e
        x[r, 5:9] = x[r].max()
    scores = torch.linspace(-3, -1, 10)
    for sign in (1, -1):
        check(P, (sign * x).to(dtype), scores, 1, 7)
        check(P, (sign * x).to(dtype), scores, 5, 9)


def test_signalling_nan_spoils_only_its_row(P):
    for dtype, ints, bits in ((BF16, torch.int16, 0x7f81), (F16, torch.int16, 0x7c01), (F32, torch.int32, 0x7f800001)):
        x = torch.randn(6, 5000, generator=gen(1)).to(dtype)
        clean = check(P, x, torch.zeros(6), 1, 4)
        x.view(ints)[2, 4000] = bits
        best, parents, tokens = check(P, x, torch.zeros(6), 1, 4)
        assert (tokens[2] == -1).all() and all(torch.equal(a[[0, 1, 3, 4, 5]], b[[0, 1, 3, 4, 5]]) for a, b in zip(clean, (best, parents, tokens)))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_rows_in_place_at_any_alignment(P, dtype):
    for V, ld, shift in ((1000, 1016, 3), (4001, 4005, 1), (9000, 9011, 7), (16390, 16391, 0)):
        base = torch.randn(6, ld + shift, generator=gen(V)).to(dtype)
        base[:, :shift] = 100                                # larger than anything in the rows
        base[:, shift + V:] = 100
        view = base.cuda()[:, shift:shift + V]
        check(P, base[:, shift:shift + V], -torch.rand(6, generator=gen(2)), 3, 6, device=view)


def test_rows_further_apart_than_32_bits(P):
    rows, V, ld = 600, 5000, 1 << 22                         # 2^22 values between rows is the most: 4.7 GiB
    base = torch.empty(rows * ld, dtype=F16, device="cuda").view(rows, ld)
    x = torch.randn(rows, V, generator=gen(3)).half()
    base[:, :V] = x.cuda()
    scores = -torch.rand(rows, generator=gen(4))
    got, want = (P.beam_select(t, scores.cuda(), 2, 5) for t in (base[:, :V], x.cuda()))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("keep", [16, 64])
def test_long_pieces_of_every_kind_of_row(P, dtype, keep):
    """A batch whose rows are cut into long pieces: rows in no order, of one value, rising, falling, of few values, masked by minus infinity or the type's lowest value."""
    B, W, V = 66, 8, 45003
    x = torch.randn(B * W, V, generator=gen(keep))
    at = torch.arange(V)
    x[0::9] = 1.5
    x[1::9] = (at * (40.0 / V)).repeat(len(x[1::9]), 1)
    x[2::9] = (-at * (40.0 / V)).repeat(len(x[2::9]), 1)
    x[3::9] = (at % 7).float().repeat(len(x[3::9]), 1)
    x[4::9, torch.randperm(V, generator=gen(1))[: V - 9]] = -math.inf
    x = x.to(dtype)
    x[5::9, 20:] = torch.finfo(dtype).min
    x[6, 39999], x[7, 3] = math.nan, math.inf
    scores = -20 * torch.rand(B * W, generator=gen(2))
    scores[100::37] = -math.inf
    check(P, x, scores, W, keep)


def test_beams_of_no_sequences_and_refusals(P):
    x = torch.zeros(4, 100, dtype=F16, device="cuda")
    s = torch.zeros(4, device="cuda")
    best, parents, tokens = P.beam_select(x[:0], s[:0], 4)
    assert best.shape == parents.shape == tokens.shape == (0, 4)
    for args, why in (((x, s, 3), "whole sequences"), ((x, s, 0), "beams"), ((x, s, 4, 65), "candidates"), ((x.t(), s, 4), "dense"), ((x.double(), s, 4), "float32"),
                      ((x, s[:3], 4), "elements"), ((x, s.half(), 4), "float32"), ((x, s, 4, 4, s), "uint8"), ((x, s, 4, 4, None, 1 << 40), "int32")):
        with pytest.raises(P.SampError, match=why):
            P.beam_select(*args)
    with pytest.raises(P.SampError, match="vocabulary"):
        P.beam_select(torch.zeros(1, (1 << 19) + 1, dtype=F16, device="cuda"), s[:1], 1)


def test_selection_in_graphs_and_on_two_streams(P):
    x = torch.randn(24, 33000, generator=gen(1)).half().cuda()
    s = -torch.rand(24, generator=gen(2)).cuda()
    side = [torch.cuda.Stream() for _ in range(2)]
    graphs = []
    P.beam_select(x, s, 4, 8)
    torch.cuda.synchronize()
    for st in side:
        with torch.cuda.stream(st):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                out = P.beam_select(x, s, 4, 8)
        graphs.append((g, out))
    for seed in range(3):
        x.copy_(torch.randn(24, 33000, generator=gen(seed)).half())
        torch.cuda.synchronize()
        for (g, _), st in zip(graphs, side):
            with torch.cuda.stream(st):
                g.replay()
        other = P.beam_select(x, s, 4, 8)
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, other))
    check(P, x.cpu(), s.cpu(), 4, 8)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_a_sequence_has_the_same_results_alone_in_a_batch_and_at_any_alignment(P, dtype):
    """The rows of a large batch are cut into long pieces, those of one sequence into short ones, and rows begin at any value: the totals have the same bits."""
    B, W, V, keep = 66, 8, 45003, 64
    g = gen(11)
    rows = (torch.randn(W, V, generator=g) * 3).to(dtype)
    rows[1, torch.rand(V, generator=g) < 0.3] = -math.inf
    rows[2] += 5000 if dtype is F32 else 30                  # (references of another size)
    rows[3, :100] = torch.finfo(dtype).min
    if dtype is not F16:
        rows[4] *= 2.0 ** 30
    scores = -torch.rand(W, generator=g)
    want = [t.cpu() for t in P.beam_select(rows.cuda(), scores.cuda(), W, keep)]
    for row in range(W):                                     # (each row's own best, also where others are far ahead)
        want_row = [t.cpu() for t in P.beam_select(rows[row:row + 1].cuda(), scores[row:row + 1].cuda(), 1, keep)]
        for shift in range(8):
            base = torch.zeros(V + shift, dtype=dtype)
            base[shift:] = rows[row]
            got = [t.cpu() for t in P.beam_select(base.cuda()[shift:][None], scores[row:row + 1].cuda(), 1, keep)]
            assert all(torch.equal(a, b) for a, b in zip(got, want_row)), (row, shift)
    batch, of = torch.randn(B * W, V, generator=g).to(dtype), -torch.rand(B * W, generator=g)
    for b in (0, 17, 65):
        batch[b * W:(b + 1) * W], of[b * W:(b + 1) * W] = rows, scores
    for ld in (V, V + 5):
        wide = torch.zeros(B * W, ld, dtype=dtype, device="cuda")
        wide[:, :V] = batch.cuda()
        best, parents, tokens = (t.cpu() for t in P.beam_select(wide[:, :V], of.cuda(), W, keep))
        for b in (0, 17, 65):
            assert torch.equal(best[b], want[0][0]) and torch.equal(parents[b] - b * W, want[1][0]) and torch.equal(tokens[b], want[2][0]), (ld, b)
    single = [t.cpu() for t in P.beam_select(batch.cuda(), of.cuda(), 1, keep)]              # long pieces, a row each
    for row in range(W):
        alone = [t.cpu() for t in P.beam_select(rows[row:row + 1].cuda(), scores[row:row + 1].cuda(), 1, keep)]
        assert torch.equal(single[0][17 * W + row], alone[0][0]) and torch.equal(single[2][17 * W + row], alone[2][0]), row


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_beams_that_are_alike_tie_wherever_their_rows_begin(P, dtype):
    """Rows of one content, each at an alignment of its own, have one log-sum-exp: their totals are equal, and the lower row comes first."""
    for V in (4001, 21127, 50257):
        x = (torch.randn(1, V, generator=gen(V)) * 2).to(dtype).repeat(8, 1)
        _, parents, tokens = P.beam_select(x.cuda(), torch.full((8,), -0.25, device="cuda"), 8, 64)
        order = torch.sort(x[0].double(), descending=True, stable=True).indices
        want, i = [], 0
        while len(want) < 64:
            same = [v for v in order[:200].tolist() if x[0, v] == x[0, order[i]]]
            want += [(r, v) for r in range(8) for v in same]
            i += len(same)
        assert list(zip(parents[0].tolist(), tokens[0].tolist())) == want[:64], V
