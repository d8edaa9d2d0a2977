"""The decoder's operators (per-token INT8 projection, paged int8 cache, attention over the cache and over whole prompts) against their
definitions in binary64, on the CPU.

Tolerances count roundings: half a step of the result's type (`half` below: 2^-11 fp16, 2^-8 bfloat16, relative, and 2^-25 below fp16's normal
numbers), half a step of the type that holds probabilities, and binary32 steps (2^-24) for what is summed and scaled in binary32.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

F16, BF16 = torch.float16, torch.bfloat16
HALF = {F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F16: 2.0 ** -25, BF16: 0.0}
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2209_09130_amd as P
    P.lib()
    return P


def gen(seed):
    return torch.Generator().manual_seed(seed)


def offsets(lengths):
    return torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32)


# ---- definitions ---------------------------------------------------------------------------------
def quantised(x):
    """(codes, steps) in binary64 over the last axis, by the definition in samp.h (steps rounded to binary32)."""
    x = x.double()
    top = x.abs().amax(-1)
    some = top >= 2.0 ** -60
    codes = torch.where(some[..., None], torch.round(127 * x / torch.where(some, top, 1.0)[..., None]), 0.0)
    return codes, torch.where(some, (top.float() / 127).double(), 1.0)


def attend(q, k, v, seen, scale):
    """q [n, H, D], k and v [m, G, D], seen [n, m] in binary64 -> (out [n, H, D], sum of p |v|, largest sum of |q k| scale [n, H])."""
    n, H, D = q.shape
    m, G, _ = k.shape
    out, size, big = torch.zeros(n, H, D).double(), torch.zeros(n, H, D).double(), torch.zeros(n, H).double()
    if m == 0:
        return out, size, big
    rows = seen.any(1)
    for h in range(H):
        kh, vh = k[:, h * G // H], v[:, h * G // H]
        sc = (q[:, h] @ kh.T * scale).masked_fill(~seen, -math.inf)
        p = torch.softmax(sc[rows], -1)
        vis = torch.nan_to_num(vh, nan=0.0)
        out[rows, h], size[rows, h] = p @ vis, p @ vis.abs()
        big[:, h] = ((q[:, h].abs() @ kh.abs().T) * scale).masked_fill(~seen, 0.0).amax(-1)
    return out, size, big


def check_attention(got, out, size, big, dtype, p_type, m, vmax):
    """p is rounded to p_type (relative half step; below 2^-14 an absolute 2^-25 in fp16, the largest being at least a half), scores are binary32
    sums of D products, sums run over m keys."""
    D = out.shape[-1]
    rel = HALF[p_type] + 2.0 ** -20 + (D + 4) * 2 * U32 * big[..., None] + (m + 8) * 2 * U32
    tol = HALF[dtype] * out.abs() * 1.01 + size * rel + m * 2 * TINY[p_type] * vmax + TINY[dtype]
    err = (got.double().cpu() - out).abs()
    worst = (err - tol).max().item()
    assert worst <= 0, (worst, err.max().item())


# ---- quantiser -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K", [(1, 8), (5, 64), (7, 520), (3, 1024), (2, 1032), (9, 2048), (3, 4096), (4, 4104), (2, 11008), (2, 20000)])
def test_quantize_tokens_takes_the_defined_codes_and_steps(P, dtype, M, K):
    x = torch.randn(M, K, generator=gen(M + K)).to(dtype)
    x[-1] *= 3e-5                                            # fp16: below the normal numbers
    codes, steps = P.quantize_tokens(x.cuda())
    want, s = quantised(x)
    assert torch.equal(codes.cpu().double(), want)
    assert torch.equal(steps.cpu().double(), s)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_quantize_tokens_ties_zeros_and_rows_that_are_not_finite(P, dtype):
    x = torch.randn(8, 256, generator=gen(3)).clamp(-3, 3).to(dtype)
    x[0, 5], x[0, 7:20] = 4.0, 2.0                           # 63.5 steps: to even
    x[1] = (torch.arange(256) - 127.5).to(dtype)             # absmax 128.5 or, rounded to eight bits, 128: ties at every other half
    x[2] = 0
    x[3, 100] = math.inf
    x[4, 200] = -math.nan
    x[5] = x[5] * 0 + (2.0 ** -24 if dtype == F16 else 2.0 ** -70)
    x[6, 0] = torch.finfo(dtype).max
    codes, steps = (t.cpu() for t in P.quantize_tokens(x.cuda()))
    keep = [0, 1, 2, 5, 6, 7]
    want, s = quantised(x[keep])
    assert torch.equal(codes[keep].double(), want) and torch.equal(steps[keep].double(), s)
    assert want[0, 7] == 64 and steps[2] == 1.0
    assert torch.isnan(steps[[3, 4]]).all() and not codes[[3, 4]].any()


def test_quantize_tokens_reads_rows_in_place(P):
    x = torch.randn(6, 400, generator=gen(9)).half().cuda()
    view = x[:, 40:296]
    codes, steps = P.quantize_tokens(view)
    again, s = P.quantize_tokens(view.contiguous())
    assert torch.equal(codes, again) and torch.equal(steps, s)


# ---- projection ----------------------------------------------------------------------------------
def weights(N, K, seed):
    W = torch.randint(-127, 128, (N, K), generator=gen(seed)).to(torch.int8)
    return W, torch.rand(N, generator=gen(seed + 1)) * 2e-3 + 1e-4


def check_linear(got, codes, steps, W, s_w, bias, gelu, dtype):
    main = (codes.double() @ W.double().T) * steps.double()[:, None] * s_w.double()
    y = main if bias is None else main + bias.double()
    # the integer becomes binary32, is scaled twice and added: four roundings; the GELU has 8e-7 of its argument and a slope below 1.13
    tol = 4 * U32 * (main.abs() + (0 if bias is None else bias.double().abs()))
    if gelu:
        tol, y = tol * 1.13 + 1.4e-6 * y.abs(), 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    tol = tol + HALF[dtype] * (y.abs() + tol) + TINY[dtype]
    assert ((got.double().cpu() - y).abs() <= tol).all()


@pytest.mark.parametrize("dtype,bias,gelu", [(F16, True, False), (BF16, False, False), (F16, False, True), (BF16, True, True)])
@pytest.mark.parametrize("M,N,K", [(1, 16, 64), (3, 80, 192), (16, 64, 256), (17, 144, 320), (5, 2512, 1600), (64, 256, 1024), (130, 528, 576), (300, 1024, 512),
                                   (33, 96, 4096), (2, 4096, 4096), (1, 6144, 2048), (700, 272, 64), (8, 1040, 11008)])
def test_linear_is_the_exact_sum_scaled_and_rounded(P, M, N, K, dtype, bias, gelu):
    x = torch.randn(M, K, generator=gen(M * 7 + K)).to(dtype)
    x[0] = 0
    W, s_w = weights(N, K, N)
    b = torch.randn(N, generator=gen(5)) if bias else None
    Wp = P.pack_weight_i8(W.cuda())
    dev = [t if t is None else t.cuda() for t in (s_w, b)]
    y = P.linear_i8_tokens(x.cuda(), Wp, *dev, gelu)
    codes, steps = P.quantize_tokens(x.cuda())
    z = P.gemm_i8_tokens_packed(codes, steps, Wp, *dev, gelu, dtype)
    assert torch.equal(y, z)
    check_linear(y, *quantised(x), W, s_w, b, gelu, dtype)


def test_linear_rows_that_are_not_finite_stay_alone(P):
    W, s_w = weights(320, 512, 8)
    x = torch.randn(40, 512, generator=gen(1)).half()
    Wp, s = P.pack_weight_i8(W.cuda()), s_w.cuda()
    want = P.linear_i8_tokens(x.cuda(), Wp, s)
    x[7, 3], x[20, 500] = math.nan, -math.inf
    got = P.linear_i8_tokens(x.cuda(), Wp, s)
    ok = torch.ones(40, dtype=torch.bool)
    ok[[7, 20]] = False
    assert torch.isnan(got[~ok.cuda()]).all() and torch.equal(got[ok.cuda()], want[ok.cuda()])
    for rows in ([7], [6, 7, 8], [20, 21], list(range(5, 15))):              # few rows, in one launch
        few = P.linear_i8_tokens(x[rows].cuda(), Wp, s)
        assert torch.equal(torch.isnan(few), torch.isnan(got[rows])) and torch.equal(torch.nan_to_num(few), torch.nan_to_num(got[rows]))


def test_linear_of_no_rows_and_of_rows_in_place(P):
    W, s_w = weights(64, 128, 8)
    Wp, s = P.pack_weight_i8(W.cuda()), s_w.cuda()
    assert P.linear_i8_tokens(torch.empty(0, 128, dtype=F16, device="cuda"), Wp, s).shape == (0, 64)
    x = torch.randn(50, 1024, generator=gen(2)).bfloat16().cuda()
    assert torch.equal(P.linear_i8_tokens(x[:, 256:384], Wp, s), P.linear_i8_tokens(x[:, 256:384].contiguous(), Wp, s))


# ---- cache ---------------------------------------------------------------------------------------
class Plan:
    """Sequences of `lens` positions of which the last `new` are new, in randomly ordered pages of a cache with spare ones."""

    def __init__(self, P, lens, new, G, D, page, seed=0, spare=3):
        self.lens, self.new, self.page, self.G, self.D = lens, new, page, G, D
        per = [-(-n // page) for n in lens]
        order = torch.randperm(sum(per) + spare, generator=gen(seed)).tolist()
        self.tables = [[order.pop() for _ in range(p)] for p in per]
        width = max(per + [1])
        self.table = torch.tensor([t + [-1] * (width - len(t)) for t in self.tables], dtype=torch.int32)
        self.cache = P.KVCache.empty(sum(per) + spare, G, page, D)
        for t in (self.cache.k, self.cache.v):
            t.fill_(55)
        for t in (self.cache.k_step, self.cache.v_step):
            t.fill_(math.nan)                                # what nobody has written must not be seen
        self.cu, self.total = offsets(new), sum(new)
        self.args = (self.table.cuda(), self.cu.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())

    def fill(self, P, dtype, seed):
        """Writes whole contexts; returns them as (k, v) per sequence, as the cache holds them, in binary64."""
        k, v = (torch.randn(sum(self.lens), self.G, self.D, generator=gen(seed + i)) * 1.5 for i in (0, 1))
        v[..., 0] *= 30
        k, v = k.to(dtype), v.to(dtype)
        if sum(self.lens):
            P.cache_write(self.cache, k.cuda(), v.cuda(), self.args[0], offsets(self.lens).cuda(), self.args[2], max(self.lens))
        held = []
        for x in (k, v):
            c, s = quantised(x)
            held.append((c * s[..., None]).split(self.lens))
        return list(zip(*held))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,G,page", [(64, 12, 16), (128, 8, 64), (128, 1, 256), (64, 3, 32), (128, 2, 1024)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([40, 7, 0, 129, 16], [3, 7, 0, 1, 16]), ([300, 257, 64], [300, 1, 20])])
def test_cache_write_and_read(P, D, G, page, lens, new, dtype):
    plan = Plan(P, lens, new, G, D, page, seed=D + G)
    before = plan.fill(P, dtype, 4)
    k, v = (torch.randn(plan.total + 2, G, D, generator=gen(i)).to(dtype) for i in (7, 8))   # two rows behind the last sequence
    snapshot = plan.cache.k.clone()
    P.cache_write(plan.cache, k.cuda(), v.cuda(), *plan.args, max(new))
    kr, vr = P.cache_read(plan.cache, plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens), sum(lens), dtype)
    want_k, want_v = [], []
    for b, (n, m) in enumerate(zip(lens, new)):
        for x, to, old in ((k, want_k, before[b][0]), (v, want_v, before[b][1])):
            c, s = quantised(x[plan.cu[b]:plan.cu[b] + m])
            to.append(torch.cat([old[: n - m], c * s[..., None]]))
    for got, want in ((kr, torch.cat(want_k)), (vr, torch.cat(want_v))):
        assert torch.equal(got.cpu(), want.float().to(dtype))         # code * step is one binary32 product, then one rounding
    used = {p for t in plan.tables for p in t}
    idle = [p for p in range(plan.cache.pages) if p not in used]
    assert torch.equal(plan.cache.k[idle], snapshot[idle])


def test_cache_rows_in_place_bad_pages_and_rows_that_are_left(P):
    plan = Plan(P, [40, 70], [40, 70], 4, 128, 16)
    qkv = torch.randn(110, (4 + 4 + 4) * 128, generator=gen(3)).bfloat16().cuda()
    k, v = (t.unflatten(1, (4, 128)) for t in (qkv[:, 512:1024], qkv[:, 1024:]))
    table = plan.args[0].clone()
    table[1, 1], table[1, 3] = 10 ** 6, -7
    P.cache_write(plan.cache, k, v, table, *plan.args[1:], 70)
    out = tuple(torch.full((115, 4, 128), 9.0, dtype=BF16, device="cuda") for _ in range(2))
    kr, vr = P.cache_read(plan.cache, table, *plan.args[1:], 70, 115, BF16, out=out)
    for got, src in ((kr.cpu(), k.cpu()), (vr.cpu(), v.cpu())):
        c, s = quantised(src)
        want = (c * s[..., None]).float().bfloat16()
        want[40 + 16:40 + 32], want[40 + 48:40 + 64] = 0, 0
        assert torch.equal(got[:110], want)
        assert (got[110:] == 9).all()
    # positions that the table has no room for, and more new rows than positions, are dropped and read as zeros
    lens = torch.tensor([20, 400], dtype=torch.int32, device="cuda")
    P.cache_write(plan.cache, k, v, plan.args[0], plan.args[1], lens, 70)
    kr, _ = P.cache_read(plan.cache, plan.args[0], plan.args[1], lens, 70, 110, BF16)
    c, s = quantised(k.cpu())
    want = (c * s[..., None]).float().bfloat16()
    assert not kr[:20].any() and torch.equal(kr[20:40].cpu(), want[20:40]) and not kr[40:].any()


def test_cache_rows_that_are_not_finite_poison_only_what_sees_them(P):
    plan = Plan(P, [20], [20], 2, 64, 16)
    k, v = (torch.randn(20, 2, 64, generator=gen(i)).half() for i in (1, 2))
    k[5, 0, 3], v[9, 1, 2] = math.inf, math.nan
    P.cache_write(plan.cache, k.cuda(), v.cuda(), *plan.args, 20)
    kr, vr = (t.cpu() for t in P.cache_read(plan.cache, *plan.args, 20, 20, F16))
    assert torch.isnan(kr[5, 0]).all() and torch.isnan(vr[9, 1]).all()
    assert torch.isfinite(kr).sum() == kr.numel() - 64 and torch.isfinite(vr).sum() == vr.numel() - 64
    q = torch.randn(20, 4, 64, generator=gen(4)).half()
    o = P.attention_cache(q.cuda(), plan.cache, *plan.args, 20).cpu()
    assert torch.isfinite(o[:5, :2]).all() and torch.isnan(o[5:, :2]).all()
    assert torch.isfinite(o[:9, 2:]).all() and torch.isnan(o[9:, 2:]).all()


# ---- attention over the cache ----------------------------------------------------------------------
def tree_words(new, seed):
    g, words = gen(seed), []
    for n in new:
        seen = []
        for i in range(n):
            seen.append((seen[int(torch.randint(0, i, (1,), generator=g))] if i else 0) | 1 << i)
        words += seen
    return words


def signed(words):
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64)


def run_cached(P, lens, new, H, G, D, page, dtype, words=None, seed=0, scale=None, max_len=None):
    plan = Plan(P, lens, new, G, D, page, seed)
    held = plan.fill(P, dtype, seed + 10)
    q = (torch.randn(plan.total, H, D, generator=gen(seed + 20)) * 2).to(dtype)
    got = P.attention_cache(q.cuda(), plan.cache, *plan.args, max(new), max_len=max_len or max(lens + [1]), scale=scale,
                            tree=None if words is None else signed(words).cuda())
    for b, (n, m) in enumerate(zip(lens, new)):
        if m == 0:
            continue
        at = int(plan.cu[b])
        pos, row = torch.arange(n)[None, :], torch.arange(m)[:, None]
        seen = pos <= n - m + row
        if words is not None:
            bits = torch.tensor([[bool(w >> j & 1) for j in range(m)] for w in words[at:at + m]])
            seen = torch.cat([torch.ones(m, max(n - m, 0), dtype=torch.bool), bits], 1)[:, :n] if n >= m else bits[:, m - n:]
        k, v = held[b]
        want = attend(q[at:at + m].double(), k, v, seen, scale or 1 / math.sqrt(D))
        check_attention(got[at:at + m], *want, dtype, F16, n, v.abs().max().item() if n else 0.0)
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,G,D,page", [(4, 4, 64, 16), (8, 2, 128, 64), (7, 1, 128, 32), (32, 8, 128, 16), (12, 12, 64, 256), (20, 1, 64, 128)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([2, 33, 5], [1, 1, 1]), ([40, 7, 129, 16, 300], [1, 1, 1, 1, 1]), ([31, 64, 200], [5, 0, 9]), ([1000], [1])])
def test_attention_cache(P, lens, new, H, G, D, page, dtype):
    run_cached(P, lens, new, H, G, D, page, dtype, seed=len(lens) + H)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_cache_long_contexts_are_cut_and_joined(P, dtype):
    run_cached(P, [5000, 3, 2049], [1, 2, 1], 8, 2, 128, 64, dtype, seed=1)
    run_cached(P, [4100], [40], 4, 4, 64, 16, dtype, seed=2)
    # the host's guess of the longest context decides the cut, not the result's meaning
    run_cached(P, [900, 40], [1, 1], 8, 1, 128, 32, dtype, seed=3, max_len=100000)
    run_cached(P, [9000, 40], [1, 1], 8, 1, 128, 32, dtype, seed=4, max_len=1)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,new", [([16], [16]), ([200, 64, 33], [64, 17, 1]), ([1500], [32])])
def test_attention_cache_of_drafts_in_a_tree(P, lens, new, dtype):
    run_cached(P, lens, new, 8, 4, 64, 32, dtype, tree_words(new, 3), seed=5)
    run_cached(P, lens, new, 4, 1, 128, 16, dtype, tree_words(new, 4), seed=6, scale=0.2)


def test_attention_cache_tokens_that_see_nothing_are_zeros(P):
    words = tree_words([8, 6], 1)
    words[2] = 0                                             # sees the context alone: there is none
    words[8 + 3] = 0                                         # sees the context of 30 positions
    got = run_cached(P, [8, 36], [8, 6], 4, 2, 64, 16, F16, words, seed=7)
    assert not got[2].any() and got[11].any()
    # no positions at all, and fewer positions than new tokens: the first have none
    plan = Plan(P, [0, 3], [2, 5], 2, 64, 16)
    plan.fill(P, F16, 3)
    q = torch.randn(7, 4, 64, generator=gen(1)).half().cuda()
    out = P.attention_cache(q, plan.cache, *plan.args, 5)
    assert not out[:4].any() and torch.isfinite(out).all() and out[4:].any()
    # pages that are none of the cache's are not seen
    plan = Plan(P, [40], [1], 2, 64, 16, seed=3)
    held = plan.fill(P, F16, 4)
    table = plan.args[0].clone()
    table[0, 1] = 12345
    got = P.attention_cache(q[:1], plan.cache, table, *plan.args[1:], 1)
    seen = torch.tensor([[not 16 <= j < 32 for j in range(40)]])
    check_attention(got, *attend(q[:1].double().cpu(), *held[0], seen, 0.125), F16, F16, 40, held[0][1].abs().max().item())


def test_attention_cache_leaves_rows_behind_the_last_sequence(P):
    plan = Plan(P, [50, 20], [2, 1], 2, 128, 16)
    plan.fill(P, BF16, 3)
    q = torch.randn(6, 4, 128, generator=gen(1)).bfloat16().cuda()
    for max_len in (50, 1 << 20):                            # in one piece, and in several
        out = torch.full((6, 4, 128), 7.0, dtype=BF16, device="cuda")
        P.attention_cache(q, plan.cache, *plan.args, 2, max_len=max_len, out=out)
        assert (out[3:] == 7).all() and (out[:3] != 7).any()
    want = P.attention_cache(q, plan.cache, *plan.args, 2, max_len=50)
    assert torch.equal(P.attention_cache(q, plan.cache, *plan.args, 4096, max_len=50)[:3], want[:3])      # a larger batch's maximum
    # no offsets: every sequence has max_new rows, and views of a wider projection are read in place
    wide = torch.randn(4, 10, 128, generator=gen(2)).bfloat16().cuda()
    a = P.attention_cache(wide[:, 2:6], plan.cache, plan.args[0], None, plan.args[2], 2)
    b = P.attention_cache(wide[:, 2:6].contiguous(), plan.cache, plan.args[0], offsets([2, 2]).cuda(), plan.args[2], 2)
    assert torch.equal(a, b)


def test_attention_cache_steps_of_very_different_size(P):
    """Keys and values of 2^-20 and 2^15 in one context: the running reference has to bound probability times step."""
    plan = Plan(P, [96], [1], 1, 64, 16)
    k, v = (torch.randn(96, 1, 64, generator=gen(i)) for i in (1, 2))
    v[::3] *= 2.0 ** -20
    v[1::7] *= 2.0 ** 13
    k[::5] *= 4
    k, v = k.bfloat16(), v.bfloat16()
    P.cache_write(plan.cache, k.cuda(), v.cuda(), plan.args[0], offsets([96]).cuda(), plan.args[2], 96)
    q = (torch.randn(1, 4, 64, generator=gen(3)) * 2.0 ** 9).bfloat16()            # beyond what binary16 sums would take
    held = [(c * s[..., None]) for c, s in (quantised(k), quantised(v))]
    got = P.attention_cache(q.cuda(), plan.cache, *plan.args, 1, scale=2.0 ** -11)
    check_attention(got, *attend(q.double(), *held, torch.ones(1, 96, dtype=torch.bool), 2.0 ** -11), BF16, F16, 96, held[1].abs().max().item())


def test_cache_offsets_pass_32_bits(P):
    """A cache of more than 2^31 codes each, used at its far end."""
    G, D, page = 8, 128, 256
    pages = (1 << 31) // (G * page * D) + 40
    cache = P.KVCache(*(torch.zeros((pages, G, page, D), dtype=torch.int8, device="cuda") for _ in range(2)),
                      *(torch.zeros((pages, G, page), device="cuda") for _ in range(2)))
    table = torch.arange(pages - 1, pages - 3, -1, dtype=torch.int32, device="cuda")[None]
    k, v = (torch.randn(300, G, D, generator=gen(i)).half() for i in (1, 2))
    lens = torch.tensor([300], dtype=torch.int32, device="cuda")
    P.cache_write(cache, k.cuda(), v.cuda(), table, None, lens, 300)
    kr, vr = P.cache_read(cache, table, None, lens, 300, 300, F16)
    held = []
    for x, got in ((k, kr), (v, vr)):
        c, s = quantised(x)
        held.append(c * s[..., None])
        assert torch.equal(got.cpu(), held[-1].float().half())
    assert not cache.k[: pages - 2].any()
    q = torch.randn(1, 8, D, generator=gen(5)).half()
    got = P.attention_cache(q.cuda(), cache, table, None, lens, 1)
    check_attention(got, *attend(q.double(), *held, torch.ones(1, 300, dtype=torch.bool), 1 / math.sqrt(D)), F16, F16, 300, held[1].abs().max().item())


# ---- attention of whole prompts ----------------------------------------------------------------------
def run_causal(P, lens, H, G, D, dtype, seed=0, scale=None):
    T = sum(lens)
    q, k, v = (torch.randn(T, n, D, generator=gen(seed + i)).to(dtype) for i, n in enumerate((H, G, G)))
    q = (q * 2).to(dtype)
    got = P.attention_causal(q.cuda(), k.cuda(), v.cuda(), offsets(lens).cuda(), max(lens), scale)
    at = 0
    for n in lens:
        s = slice(at, at + n)
        want = attend(q[s].double(), k[s].double(), v[s].double(), torch.ones(n, n, dtype=torch.bool).tril(), scale or 1 / math.sqrt(D))
        if n:
            check_attention(got[s], *want, dtype, dtype, n, v.abs().max().item())
        at += n
    return q, k, v, got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,G,D", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (12, 12, 64), (3, 3, 128)])
@pytest.mark.parametrize("lens", [[1], [2, 31, 0, 32, 33], [63, 64, 65, 1, 0], [127, 128, 129, 5], [300, 17, 257, 256, 255], [700]])
def test_attention_causal(P, lens, H, G, D, dtype):
    run_causal(P, lens, H, G, D, dtype, seed=sum(lens))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_causal_scale_and_rows_in_place(P, dtype):
    run_causal(P, [90, 200], 4, 2, 64, dtype, scale=0.5)
    H, G, D, lens = 8, 2, 128, [100, 3, 140]
    qkv = torch.randn(sum(lens), (H + 2 * G) * D, generator=gen(4)).to(dtype).cuda()
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split((H * D, G * D, G * D), 1))
    cu = offsets(lens).cuda()
    assert torch.equal(P.attention_causal(q, k, v, cu, 140), P.attention_causal(q.contiguous(), k.contiguous(), v.contiguous(), cu, 140))
    one = slice(0, 240)
    assert torch.equal(P.attention_causal(q[one], k[one], v[one], None, 80), P.attention_causal(q[one], k[one], v[one], offsets([80] * 3).cuda(), 80))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_causal_what_is_not_seen_has_no_part(P, dtype, D):
    lens, H, G = [150, 100], 4, 2
    T = sum(lens)
    q, k, v = (torch.randn(T, n, D, generator=gen(i)).to(dtype).cuda() for i, n in enumerate((H, G, G)))
    cu = offsets(lens).cuda()
    clean = P.attention_causal(q, k, v, cu, 150)
    k2, v2 = k.clone(), v.clone()
    k2[70, 0, 3], v2[75, 1, 5], v2[133, 0, 7], k2[249, 1, 0] = math.inf, math.nan, -math.inf, math.nan
    got = P.attention_causal(q, k2, v2, cu, 150)
    assert torch.equal(got[:70], clean[:70]) and torch.equal(got[150:249], clean[150:249])
    assert torch.equal(got[70:75, 2:], clean[70:75, 2:])                # the second key head's value comes later
    rest = torch.ones(D, dtype=torch.bool)
    rest[5] = False
    near = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2 * HALF[dtype], atol=2 * HALF[dtype])   # another order of the same sums at most
    assert torch.isnan(got[75:150, 2:, 5]).all() and near(got[75:150, 2:, rest], clean[75:150, 2:, rest])
    # key 70 of the first head has an infinite product with some queries: a score of +inf makes NaN, of -inf nothing
    dead = (q[70:150, :2, 3] > 0).cpu()
    assert torch.isnan(got[70:150, :2][dead.cuda()]).all()
    live = torch.isfinite(got[70:150, :2]).all(-1).cpu() | torch.isinf(got[70:150, :2]).any(-1).cpu()
    assert (live | dead).all()
    late = got[133:150, :2][~dead[63:].cuda()]
    assert (late[:, 7] == -math.inf).all()
    assert torch.equal(P.attention_causal(q, k, v, cu, 4096), clean)        # a larger batch's maximum
    # rows behind the last sequence, and of a sequence that is longer than the host said, are left
    out = torch.full((T, H, D), 5.0, dtype=dtype, device="cuda")
    P.attention_causal(q, k, v, cu[:2].contiguous(), 90, out=out)
    assert torch.equal(out[:90], clean[:90]) and (out[90:] == 5).all()


def test_attention_causal_scores_that_rise_all_along(P):
    """Each key's score is far above all earlier ones: the running reference moves in every tile."""
    n, D = 400, 64
    k = torch.zeros(n, 1, D)
    k[:, 0, 0] = torch.arange(n) * 0.5
    v = torch.randn(n, 1, D, generator=gen(1))
    q = torch.zeros(n, 1, D)
    q[:, 0, 0] = 8
    for dtype in (F16, BF16):
        a, b, c = q.to(dtype), k.to(dtype), v.to(dtype)
        got = P.attention_causal(a.cuda(), b.cuda(), c.cuda(), None, n)
        want = attend(a.double(), b.double(), c.double(), torch.ones(n, n, dtype=torch.bool).tril(), 0.125)
        check_attention(got, *want, dtype, dtype, n, c.abs().max().item())


def test_attention_causal_keys_of_the_lowest_value(P):
    """Keys of the type's lowest value: scores that binary32 cannot hold count as minus infinity, a row of nothing else is zeros or NaN alone."""
    n, D = 70, 64
    q = torch.ones(n, 1, D).bfloat16()
    k, v = torch.randn(n, 1, D, generator=gen(1)).bfloat16(), torch.randn(n, 1, D, generator=gen(2)).bfloat16()
    k[10:20] = torch.finfo(BF16).min
    got = P.attention_causal(q.cuda(), k.cuda(), v.cuda(), None, n).cpu()
    seen = torch.ones(n, n, dtype=torch.bool).tril()
    seen[:, 10:20] = False
    k[10:20] = 0
    want = attend(q.double(), k.double(), v.double(), seen, 0.125)
    check_attention(got, *want, BF16, BF16, n, v.abs().max().item())


# ---- streams, graphs, the block as a whole -------------------------------------------------------------
def test_calls_run_on_the_current_stream_and_in_graphs(P):
    lens, H, G, D = [300, 40, 128], 8, 2, 128
    plan = Plan(P, lens, [1, 1, 1], G, D, 64)
    plan.fill(P, F16, 1)
    W, s_w = weights((H + 2 * G) * D, 512, 2)
    Wp, s = P.pack_weight_i8(W.cuda()), s_w.cuda()
    x = torch.randn(3, 512, generator=gen(5)).half().cuda()

    def step():
        qkv = P.linear_i8_tokens(x, Wp, s)
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split((H * D, G * D, G * D), 1))
        P.cache_write(plan.cache, k, v, *plan.args, 1)
        return P.attention_cache(q, plan.cache, plan.args[0], None, plan.args[2], 1, max_len=8192)

    want = step().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want)
    graphs = []
    for _ in range(2):
        with torch.cuda.stream(side):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = step()
        graphs.append((g, out))
    for seed in range(3):
        x.copy_(torch.randn(3, 512, generator=gen(seed)).half())
        plan.args[2].copy_(torch.tensor([300 - seed, 40 - 5 * seed, 128 - 63 * seed], dtype=torch.int32))
        torch.cuda.synchronize()
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = step()
        for _, out in graphs:
            assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_block_of_a_decoder(P, dtype):
    """Prompts, then tokens one by one, then drafts: projection, cache, attention, projection, against binary64 from each call's own inputs on, and
    the whole against a block without any quantisation."""
    hidden, H, G, D, page, lens = 512, 8, 2, 64, 16, [37, 5, 90]
    W1 = torch.randn((H + 2 * G) * D, hidden, generator=gen(1)) / math.sqrt(hidden)
    W2 = torch.randn(hidden, H * D, generator=gen(2)) / math.sqrt(H * D)
    packed = []
    for W in (W1, W2):
        codes, s_w = P.quantize_weight(W.half().cuda())
        packed.append((P.pack_weight_i8(codes), s_w, codes.cpu(), s_w.cpu()))
    steps = [lens, [1, 1, 1], [1, 1, 1], [4, 4, 4]]
    final = [n + 6 for n in lens]
    plan = Plan(P, final, [0] * 3, G, D, page)
    history = [[], [], []]                                    # inputs of each sequence
    now = [0, 0, 0]
    for i, new in enumerate(steps):
        now = [a + b for a, b in zip(now, new)]
        x = torch.randn(sum(new), hidden, generator=gen(30 + i)).to(dtype)
        for b, part in enumerate(x.split(new)):
            history[b].append(part)
        cu, seqlens = offsets(new).cuda(), torch.tensor(now, dtype=torch.int32).cuda()
        words = signed([1, 3, 5, 13] * 3).cuda() if i == 3 else None
        qkv = P.linear_i8_tokens(x.cuda(), packed[0][0], packed[0][1])
        check_linear(qkv, *quantised(x), packed[0][2], packed[0][3], None, False, dtype)
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split((H * D, G * D, G * D), 1))
        P.cache_write(plan.cache, k, v, plan.args[0], cu, seqlens, max(new))
        if i == 0:
            o = P.attention_causal(q, k, v, cu, max(new))
        else:
            o = P.attention_cache(q, plan.cache, plan.args[0], cu, seqlens, max(new), tree=words)
        y = P.linear_i8_tokens(o.flatten(1), packed[1][0], packed[1][1])
        check_linear(y, *quantised(o.flatten(1).cpu()), packed[1][2], packed[1][3], None, False, dtype)
        # without quantisation
        at = 0
        for b in range(3):
            xs = torch.cat(history[b]).double()
            full = xs @ W1.double().T
            fq, fk, fv = (t.unflatten(1, (-1, D)) for t in full.split((H * D, G * D, G * D), 1))
            n, m = now[b], new[b]
            seen = torch.ones(n, n, dtype=torch.bool).tril()[-m:]
            if words is not None:
                seen[:, -4:] = torch.tensor([[bool(w >> j & 1) for j in range(4)] for w in (1, 3, 5, 13)])
            ref = attend(fq[-m:], fk, fv, seen, 1 / math.sqrt(D))[0].flatten(1) @ W2.double().T
            off = (y[at:at + m].double().cpu() - ref).norm() / ref.norm()
            # each 8-bit rounding is uniform within half a step of absmax / 127, about 3.3 sigma / 127: 0.0075 sigma; x, both weights, k, v and o
            # have one each (the scores' errors, of unit variance, count like another two): sqrt(8) * 0.0075 = 0.021, doubled; bfloat16's own roundings add 2^-8 a few times
            assert off < 0.045 + (0.02 if dtype == BF16 else 0.0), off
            at += m


def test_two_streams_at_once(P):
    """Calls on two streams overlap: each has a workspace of its own and shares nothing but what it reads."""
    plan = Plan(P, [5000, 900, 3000], [1, 1, 1], 2, 128, 64)
    plan.fill(P, F16, 1)
    q = torch.randn(3, 8, 128, generator=gen(5)).half().cuda()
    W, s_w = weights(1024, 1024, 2)
    Wp, s = P.pack_weight_i8(W.cuda()), s_w.cuda()
    x = torch.randn(600, 1024, generator=gen(6)).half().cuda()
    want = P.attention_cache(q, plan.cache, *plan.args, 1), P.linear_i8_tokens(x, Wp, s)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(10):
        for st in streams:
            with torch.cuda.stream(st):
                got.append((P.attention_cache(q, plan.cache, *plan.args, 1), P.linear_i8_tokens(x, Wp, s)))
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_sequences_share_the_pages_of_a_prefix(P):
    plan = Plan(P, [64, 64], [64, 64], 2, 64, 16)
    held = plan.fill(P, F16, 3)
    table = plan.args[0].clone()
    table[1, :2] = table[0, :2]                              # the first 32 positions are the first sequence's
    q = torch.randn(2, 4, 64, generator=gen(5)).half()
    got = P.attention_cache(q.cuda(), plan.cache, table, None, plan.args[2], 1)
    k, v = (torch.cat([held[0][i][:32], held[1][i][32:]]) for i in (0, 1))
    check_attention(got[1:], *attend(q[1:].double(), k, v, torch.ones(1, 64, dtype=torch.bool), 0.125), F16, F16, 64, v.abs().max().item())
