"""Sizes past int32 at the decoder's Python entry points: what the C entry cannot count is refused or counts as its largest, never as its low 32 bits."""
import ctypes as C
import os

import pytest
import torch

import paper_2209_09130_amd as P
from paper_2209_09130_amd import decoder as D

from test_gpu_decoder import BF16, F16, Plan, gen, offsets


def meta(*shape, dtype):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_shapes_past_int32_are_refused():
    for shape in ((2 ** 32 + 5, 8), (2 ** 31, 8), (1, 2 ** 32 + 64)):
        with pytest.raises(P.SampError, match="int32"):
            D._rows2("x", meta(*shape, dtype=torch.float16))
    for shape in ((1, 2 ** 32 + 1), (2 ** 31, 1)):
        with pytest.raises(P.SampError, match="int32"):
            D._places(-1, meta(*shape, dtype=torch.int32), None, meta(shape[0], dtype=torch.int32))


def test_maxima_past_int32_count_as_its_largest():
    assert [D._most(n) for n in (1, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 0, -3, -(2 ** 32) + 5)] == [1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 0, -1, -1]


def partial_bytes(batch, new, heads, kv_heads, dim, max_len):
    if not os.path.exists(P.lib_path()):
        from paper_2209_09130_amd import build as B
        B.build(force=True)
    return D._fn("samp_attention_cache_workspace_bytes")(batch * new, batch, heads, kv_heads, dim, new, max_len)


def test_calls_that_fill_the_chip_without_a_cut_have_few_partial_results():
    """Many new tokens have none; one token of many contexts has pieces in proportion; one context is cut as before."""
    for batch, new, heads, kv_heads, dim, max_len in ((64, 512, 32, 8, 128, 4500), (16, 128, 32, 8, 128, 8192), (1, 512, 32, 8, 128, 4500), (8, 2000, 64, 4, 128, 1 << 20)):
        assert partial_bytes(batch, new, heads, kv_heads, dim, max_len) == 0
    assert partial_bytes(4096, 1, 32, 8, 128, 131072) == 4096 * 32 * 2 * 130 * 4      # 4096 tiles in pieces of at most 48 * 64
    assert partial_bytes(128, 1, 32, 8, 128, 8192) <= 128 * 32 * 3 * 130 * 4 + 256
    assert partial_bytes(1, 1, 32, 8, 128, 4000) == 32 * 32 * 130 * 4            # 125 tiles, four of them a piece
    assert partial_bytes(64, 1, 32, 8, 128, 8192) == 64 * 32 * 6 * 130 * 4       # 256 tiles in pieces of at most 48


def test_a_scale_whose_log2_e_fold_overflows_is_refused():
    """Scores are multiplied by scale log2(e): an infinite factor times a product of 0 would be NaN."""
    import test_decoder_refusals as refusals
    fn = {n: D._fn(n) for n in D._SIGNATURES}
    at, kv = refusals.AT, refusals.cache()
    for scale in (2.5e38, 3.4e38):
        assert fn["samp_attention_causal"](at, 256, at, 128, at, 128, 1, 4, 2, 64, at, 2, 3, 5, scale, at, None) == refusals.SCALE
        assert fn["samp_attention_cache"](at, 256, 0, 4, C.addressof(kv), at, 2, at, at, 2, 3, 32, 5, scale, None, at, None, 0, None) == refusals.SCALE


@pytest.mark.gpu
def test_calls_with_maxima_past_int32():
    lens, H, G, dim = [70, 30], 4, 2, 64
    large = 2 ** 32 + 1
    plan = Plan(P, lens, lens, G, dim, 16)
    k, v = (torch.randn(100, G, dim, generator=gen(i)).half().cuda() for i in (1, 2))
    q = torch.randn(100, H, dim, generator=gen(3)).half().cuda()
    P.cache_write(plan.cache, k, v, *plan.args, large)
    want = P.cache_read(plan.cache, *plan.args, 70, 100, F16)
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    got = P.cache_read(plan.cache, *plan.args, large, 100, F16)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(P.attention_causal(q, k, v, plan.args[1], large), P.attention_causal(q, k, v, plan.args[1], 70))
    assert torch.equal(P.attention_cache(q, plan.cache, *plan.args, large, max_len=70), P.attention_cache(q, plan.cache, *plan.args, 70, max_len=70))
    assert torch.equal(P.attention_cache(q, plan.cache, *plan.args, 70, max_len=large), P.attention_cache(q, plan.cache, *plan.args, 70, max_len=70))
    for bad in (0, -3, -(2 ** 32) + 70):
        with pytest.raises(P.SampError):
            P.attention_causal(q, k, v, plan.args[1], bad)
        with pytest.raises(P.SampError):
            P.cache_write(plan.cache, k, v, *plan.args, bad)


@pytest.mark.gpu
def test_a_page_table_with_room_past_int32():
    """max_len None is what the table has room for, here 2^31 positions: the same cut, and so the same bytes, as of the largest int32."""
    plan = Plan(P, [1500], [1], 2, 128, 1024)
    plan.fill(P, BF16, 4)
    q = torch.randn(1, 4, 128, generator=gen(3)).bfloat16().cuda()
    table = torch.full((1, 2 ** 21), -1, dtype=torch.int32, device="cuda")
    table[:, :2] = plan.args[0]
    want = P.attention_cache(q, plan.cache, plan.args[0], None, plan.args[2], 1, max_len=2 ** 31 - 1)
    assert torch.equal(P.attention_cache(q, plan.cache, table, None, plan.args[2], 1), want)
