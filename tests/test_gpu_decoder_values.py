"""Attention over the cache and over whole prompts where values and scores are of very different size: rows of zeros, keys that most of the probability
falls on but whose value adds nothing, channels that one row alone is large in, contexts that are cut and joined.  Against the definition in binary64,
with tolerances relative to each result.

Over the cache a probability times a step is held in two bfloat16 numbers (half steps of 2^-8 each: 2^-16 of it, whatever its size); scores, sums and the
exponential are binary32, of which 2^-20 is allowed for the exponential.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

import test_gpu_decoder as basic  # noqa: E402
from test_gpu_decoder import BF16, F16, HALF, TINY, U32, P, Plan, attend, check_linear, gen, offsets, quantised, weights  # noqa: E402, F401


def check_close(got, out, size, big, dtype, m, p_half=2.0 ** -16):
    """size: sum of p |v|; big: the largest sum of |q k| scale; m keys.  Nothing in it grows with values other than the result's own terms.  A lane adds one in 16
    probabilities; a product adds 32 keys of one tile in four, twice; then two lanes' exchanges, four waves and at most 64 pieces are added."""
    D = out.shape[-1]
    rel = p_half + 2.0 ** -20 + (D + 4) * 2 * U32 * big[..., None] + (m / 16 + 128) * 2 * U32
    tol = HALF[dtype] * out.abs() * 1.01 + size * rel + TINY[dtype]
    err = (got.double().cpu() - out).abs()
    worst = (err - tol).max().item()
    assert worst <= 0, (worst, err.max().item(), (err / tol).max().item())


def written(P, k, v, page, n):
    """A plan of one sequence of n positions with these keys and values, and what the cache holds of them, in binary64."""
    plan = Plan(P, [n], [n], k.shape[1], k.shape[2], page, seed=n)
    P.cache_write(plan.cache, k.cuda(), v.cuda(), *plan.args, n)
    return plan, [c * s[..., None] for c, s in (quantised(k), quantised(v))]


def run(P, q, k, v, page, dtype, max_len=None):
    n, m = k.shape[0], q.shape[0]
    plan, held = written(P, k, v, page, n)
    got = P.attention_cache(q.cuda(), plan.cache, plan.args[0], None, plan.args[2], m, max_len=max_len or n)
    seen = torch.arange(n)[None, :] <= n - m + torch.arange(m)[:, None]
    out, size, big = attend(q.double(), *held, seen, 1 / math.sqrt(q.shape[2]))
    check_close(got, out, size, big, dtype, n)
    return got, out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,H,G,n,m", [(128, 4, 1, 32, 1), (64, 6, 2, 300, 1), (128, 8, 2, 70, 5), (64, 4, 4, 3000, 20)])
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-5, 1e-6])
def test_attention_cache_beside_value_rows_of_zeros(P, dtype, D, H, G, n, m, size):
    q = (torch.randn(m, H, D, generator=gen(1)) * 1.5).to(dtype)
    k, v = (torch.randn(n, G, D, generator=gen(i)) for i in (2, 3))
    v *= size
    v[7 % n], v[n // 2:n // 2 + 9, 0] = 0, 0
    run(P, q, k.to(dtype), v.to(dtype), 16, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("nats", [8, 11, 13, 15, 30])
@pytest.mark.parametrize("size", [1.0, 0.05])
def test_attention_cache_of_a_key_that_takes_the_probability_and_gives_nothing(P, dtype, nats, size):
    """The first key's score lies far above the rest, its value is zero."""
    D, G, n = 128, 2, 512
    q = torch.randn(1, G, D, generator=gen(1))
    k, v = (torch.randn(n, G, D, generator=gen(i)) for i in (2, 3))
    k[0] = q[0] * (nats * math.sqrt(D) / (q[0] ** 2).sum(-1, keepdim=True))
    v *= size
    v[0] = 0
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    # (at 30 nats the rest has 2^-34 of the sum: what is left of it is below fp16)
    got, out = run(P, q, k, v, 32, dtype)
    if dtype == BF16 or nats < 30:
        assert got.any()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("large,small", [(100.0, 1e-2), (3e4, 1e-2), (1e3, 1e-6)])
def test_attention_cache_channels_that_one_value_row_is_large_in(P, dtype, large, small):
    """In the other channels that row's codes are 0, and the result is that of the small rows alone."""
    D, G, n = 64, 2, 200
    q = torch.randn(3, 2 * G, D, generator=gen(1)).to(dtype)
    k, v = (torch.randn(n, G, D, generator=gen(i)) for i in (2, 3))
    v *= small
    v[90] = 0
    v[90, :, 5] = large
    run(P, q, k.to(dtype), v.to(dtype), 64, dtype)


def test_attention_cache_values_of_the_largest_bfloat16(P):
    """Probabilities that run above their reference times steps of 2^121 fit binary32."""
    D, n = 64, 100
    k, v = (torch.randn(n, 1, D, generator=gen(i)) for i in (2, 3))
    k *= torch.linspace(0.1, 2.5, n)[:, None, None]            # later keys have the higher scores
    v = torch.where(v > 0, 1.0, -1.0) * torch.finfo(BF16).max * 0.9
    v[::3] *= 2.0 ** -30
    q = torch.randn(1, 2, D, generator=gen(1)).to(BF16)
    run(P, q, k.to(BF16), v.to(BF16), 16, BF16)


@pytest.mark.parametrize("q_large,k_large", [(2.0 ** 30, 1.0), (2.0 ** 60, 2.0 ** 60), (2.0 ** 100, 2.0 ** 100), (2.0 ** -100, 2.0 ** 90)])
def test_attention_cache_channels_that_queries_or_keys_are_large_in_alone(P, q_large, k_large):
    """One channel of the queries is large and no key has anything there; one key is large in a channel that no query has.  The scores are those of the
    other channels."""
    D, G, n = 128, 2, 100
    q = torch.randn(2, 2 * G, D, generator=gen(1))
    k, v = (torch.randn(n, G, D, generator=gen(i)) for i in (2, 3))
    q[..., 0], k[..., 0] = q_large, 0
    q[..., 1], k[40, :, 1] = 0, k_large
    run(P, q.to(BF16), k.to(BF16), v.to(BF16), 16, BF16)


@pytest.mark.parametrize("M,K", [(1, 512), (9, 512), (70, 512), (40, 8192)])
def test_linear_of_the_largest_rows(P, M, K):
    """The sum times the row's step is past binary32, the channel's step brings it back."""
    x = torch.randn(M, K, generator=gen(M))
    x = (x / x.abs().amax(1, keepdim=True) * torch.finfo(BF16).max * 0.9).to(BF16)
    W, s_w = weights(96, K, 3)
    W = W.abs() * torch.where(x[:1].float() < 0, -1, 1).to(torch.int8)               # the first row's products add up
    s_w *= 2.0 ** -30
    got = P.linear_i8_tokens(x.cuda(), P.pack_weight_i8(W.cuda()), s_w.cuda())
    codes, steps = quantised(x)
    assert ((codes @ W.double().T) * steps[:, None]).abs().max() > torch.finfo(torch.float32).max
    check_linear(got, codes, steps, W, s_w, None, False, BF16)


def run_causal(P, q, k, v, dtype):
    """Probabilities have the type's half step, in binary16 at least 2^-32 of the largest (2^-25, the largest being 2^7 or more)."""
    n, D = q.shape[0], q.shape[2]
    got = P.attention_causal(q.cuda(), k.cuda(), v.cuda(), None, n)
    out, size, big = attend(q.double(), k.double(), v.double(), torch.ones(n, n, dtype=torch.bool).tril(), 1 / math.sqrt(D))
    if dtype == F16:
        every = v.double().abs().cumsum(0).repeat_interleave(q.shape[1] // v.shape[1], 1) * 2.0 ** -32
    else:
        every = torch.zeros(1)
    rel = HALF[dtype] + 2.0 ** -20 + (D + 4) * 2 * U32 * big[..., None] + (n + 8) * 2 * U32
    tol = HALF[dtype] * out.abs() * 1.01 + size * rel + TINY[dtype] + every
    err = (got.double().cpu() - out).abs()
    assert (err <= tol).all(), ((err - tol).max().item(), (err / tol).max().item())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("nats", [8, 11, 13, 15, 17])
def test_attention_causal_of_a_key_that_takes_the_probability_and_gives_nothing(P, dtype, nats):
    """The first key's score lies far above the rest for all queries, its value is zero."""
    D, G, n = 128, 2, 512
    q, k, v = (torch.randn(n, G, D, generator=gen(i)) for i in (1, 2, 3))
    q[..., 0] = 4.0
    k[..., 0] = 0
    k[0] = 0
    k[0, :, 0] = nats * math.sqrt(D) / 4.0
    v[0] = 0
    run_causal(P, q.to(dtype), k.to(dtype), v.to(dtype), dtype)


def test_attention_causal_values_of_the_largest_bfloat16(P):
    """Probabilities that run above their reference, and sums over keys, times values near the type's largest."""
    D, n = 64, 200
    q, k, v = (torch.randn(n, 1, D, generator=gen(i)) for i in (1, 2, 3))
    k *= torch.linspace(0.1, 2.5, n)[:, None, None]
    v = torch.where(v > -1, 1.0, -1.0) * torch.finfo(BF16).max * 0.9
    run_causal(P, q.to(BF16), k.to(BF16), v.to(BF16), BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,max_len", [(4100, 4100), (5000, 5000), (9000, 9000), (9000, 1), (700, 100000), (2049, 8192)])
@pytest.mark.parametrize("D,H,G,m", [(128, 8, 1, 1), (64, 4, 4, 40)])
def test_attention_cache_counts_each_key_once(P, dtype, n, max_len, D, H, G, m):
    """Queries of zeros: every key a token sees has the same probability, so the result is a count of keys, by tile (a lost or doubled tile is a third of a
    channel) or by place in the tile (one in some seventy of 32 channels)."""
    j = torch.arange(n)
    k = torch.randn(n, G, D, generator=gen(n)).to(dtype)
    q = torch.zeros(m, H, D, dtype=dtype)
    for channel in (j // 32 % D, j % D):
        v = torch.zeros(n, G, D)
        v[j, :, channel] = 1.0
        got, out = run(P, q, k, v.to(dtype), 64, dtype, max_len)
        seen = torch.stack([torch.bincount(channel[:n - m + 1 + i], minlength=D) / (n - m + 1 + i) for i in range(m)]).double()
        assert (out - seen[:, None]).abs().max() < 1e-6


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,new,H,G,D,page,drafts,max_len", [
    ([5000, 3, 2049], [1, 2, 1], 8, 2, 128, 64, False, None), ([4100], [40], 4, 4, 64, 16, False, None), ([900, 40], [1, 1], 8, 1, 128, 32, False, 100000),
    ([9000, 40], [1, 1], 8, 1, 128, 32, False, 1), ([1500], [32], 4, 1, 128, 16, True, None), ([200, 64, 33], [64, 17, 1], 8, 4, 64, 32, True, None),
    ([700, 300, 12], [600, 290, 12], 16, 8, 64, 32, False, None), ([2500, 1800], [300, 1], 32, 8, 128, 64, False, None)])
def test_attention_cache_within_its_own_roundings(P, monkeypatch, lens, new, H, G, D, page, drafts, max_len, dtype):
    """No part of the tolerance grows with values other than a result's own terms, so that a tile left out of a long context shows."""
    monkeypatch.setattr(basic, "check_attention", lambda got, out, size, big, t, p_type, m, vmax: check_close(got, out, size, big, t, m))
    basic.run_cached(P, lens, new, H, G, D, page, dtype, basic.tree_words(new, 3) if drafts else None, seed=9, max_len=max_len)


def test_the_tolerance_sees_a_tile_left_out():
    """The check itself, on the CPU: where the keys count alike, the definition without one tile of 32 of them is not within it."""
    n, D = 9000, 128
    q, k, v = (torch.randn(m, 1, D, generator=gen(m)).double() for m in (1, n, n + 1))
    q, v = q * 0.1, v[:n]
    v[..., 0] *= 30
    everything = torch.ones(1, n, dtype=torch.bool)
    out, size, big = attend(q, k, v, everything, 1 / math.sqrt(D))
    for dtype in (F16, BF16):
        check_close(out.to(dtype), out, size, big, dtype, n)
    everything[:, 4000:4032] = False
    less = attend(q, k, v, everything, 1 / math.sqrt(D))[0]
    for dtype in (F16, BF16):
        with pytest.raises(AssertionError):
            check_close(less.to(dtype), out, size, big, dtype, n)
