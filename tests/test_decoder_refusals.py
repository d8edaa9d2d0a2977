"""What the decoder's entry points refuse, on the host, before any launch (no GPU is needed, the pointers are host memory that nothing reads)."""
import ctypes as C
import os

import pytest
import torch

import paper_2209_09130_amd as P
from paper_2209_09130_amd import decoder as D


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(P.lib_path()):
        from paper_2209_09130_amd import build as B
        B.build(force=True)
    for name in D._SIGNATURES:
        D._fn(name)
    return P.lib()


_mem = (C.c_char * 8192)()
AT = (C.addressof(_mem) + 255) & ~255
ARG, SHAPE, SPACE, SCALE = -1, -2, -3, -5


def cache(**change):
    f = dict(k=AT, v=AT, k_step=AT, v_step=AT, pages=4, kv_heads=2, page_len=16, head_dim=64)
    f.update(change)
    return D._CacheStruct(*f.values())


def with_(args, **change):
    """A call's argument list with some of its named arguments replaced."""
    return [change.get(n, v) for n, v in args]


def refusals(f, base, cases):
    for change, code, word in cases:
        names = [n for n, _ in base]
        assert all(c in names for c in change), change
        assert f(*with_(base, **change)) == code, change
        assert word in P.lib().samp_last_error(), (change, P.lib().samp_last_error())


def test_quantize_tokens(L):
    base = [("x", AT), ("ldx", 64), ("type", 0), ("M", 2), ("K", 64), ("codes", AT), ("steps", AT), ("stream", None)]
    refusals(L.samp_quantize_tokens, base, [
        ({"x": None}, ARG, b"NULL"), ({"codes": None}, ARG, b"NULL"), ({"steps": None}, ARG, b"NULL"), ({"type": 2}, ARG, b"type"), ({"type": -1}, ARG, b"type"),
        ({"M": 0}, SHAPE, b"rows"), ({"M": (1 << 24) + 1}, SHAPE, b"rows"), ({"K": 0}, SHAPE, b"M=2"), ({"K": 12}, SHAPE, b"K=12"),
        ({"ldx": 56}, SHAPE, b"leading"), ({"ldx": 68}, ARG, b"aligned"), ({"ldx": (1 << 22) + 8}, SHAPE, b"leading"), ({"ldx": -64}, SHAPE, b"leading"),
        ({"x": AT + 8}, ARG, b"aligned"), ({"codes": AT + 4}, ARG, b"aligned"), ({"steps": AT + 2}, ARG, b"aligned")])


def test_products(L):
    base = [("codes", AT), ("steps", AT), ("Wp", AT), ("s_w", AT), ("bias", None), ("gelu", 0), ("out", AT), ("type", 0), ("M", 2), ("N", 64), ("K", 128),
            ("stream", None)]
    shared = [({"Wp": None}, ARG, b"NULL"), ({"s_w": None}, ARG, b"NULL"), ({"out": None}, ARG, b"NULL"), ({"type": 5}, ARG, b"type"), ({"M": 0}, SHAPE, b"rows"),
              ({"N": 24}, SHAPE, b"N=24"), ({"N": 0}, SHAPE, b"N=0"), ({"K": 96}, SHAPE, b"K=96"), ({"K": 131136}, SHAPE, b"K <="), ({"N": 1 << 20, "K": 4096}, SHAPE, b"2^31"),
              ({"Wp": AT + 8}, ARG, b"aligned"), ({"s_w": AT + 4}, ARG, b"aligned"), ({"bias": AT + 4}, ARG, b"aligned"), ({"out": AT + 2}, ARG, b"aligned")]
    refusals(L.samp_gemm_i8_tokens_packed, base, shared + [({"codes": None}, ARG, b"NULL"), ({"steps": None}, ARG, b"NULL"), ({"codes": AT + 8}, ARG, b"aligned")])
    need = L.samp_linear_i8_tokens_workspace_bytes(100, 128)
    assert need >= 100 * 128 + 400
    assert L.samp_linear_i8_tokens_workspace_bytes(0, 128) == 0 and L.samp_linear_i8_tokens_workspace_bytes(100, 100) == 0
    base = [("x", AT), ("ldx", 128), ("type", 0), ("Wp", AT), ("s_w", AT), ("bias", None), ("gelu", 0), ("out", AT), ("M", 2), ("N", 64), ("K", 128),
            ("workspace", AT), ("bytes", need), ("stream", None)]
    refusals(L.samp_linear_i8_tokens, base, shared + [
        ({"x": None}, ARG, b"NULL"), ({"ldx": 120}, SHAPE, b"leading"), ({"M": 100, "workspace": None}, SPACE, b"workspace"),
        ({"M": 100, "workspace": AT + 16}, SPACE, b"workspace"), ({"M": 100, "bytes": need - 1}, SPACE, b"workspace")])


BAD_CACHES = [(dict(k=None), ARG, b"NULL"), (dict(v_step=None), ARG, b"NULL"), (dict(v=AT + 8), ARG, b"aligned"), (dict(head_dim=96), SHAPE, b"head_dim"),
              (dict(page_len=8), SHAPE, b"page_len"), (dict(page_len=48), SHAPE, b"page_len"), (dict(page_len=2048), SHAPE, b"page_len"), (dict(pages=0), SHAPE, b"pages"),
              (dict(kv_heads=0), SHAPE, b"heads"), (dict(kv_heads=1025), SHAPE, b"heads")]


def cache_cases(most):
    places = [({"table": None}, ARG, b"table"), ({"lens": None}, ARG, b"NULL"), ({"width": 0}, SHAPE, b"width"), ({"batch": 0}, SHAPE, b"sequences"),
              ({"batch": 8193}, SHAPE, b"sequences"), ({most: 0}, SHAPE, most.encode()), ({most: 1 << 21, "rows": 1 << 21}, SHAPE, most.encode()), ({"rows": 0}, SHAPE, b"rows"),
              ({"rows": (1 << 24) + 1}, SHAPE, b"rows"), ({"cu": None}, SHAPE, b"without offsets"), ({"type": 3}, ARG, b"type"), ({"cache": None}, ARG, b"cache")]
    bad = [(cache(**c), code, word) for c, code, word in BAD_CACHES]
    return places + [({"cache": C.addressof(b)}, code, word) for b, code, word in bad], bad


def test_cache_write_and_read(L):
    ok = cache()
    places = [("type", 0), ("table", AT), ("width", 2), ("cu", AT), ("lens", AT), ("batch", 2), ("max_new", 3), ("rows", 5), ("stream", None)]
    base = [("cache", C.addressof(ok)), ("k", AT), ("ldk", 128), ("v", AT), ("ldv", 128)] + places
    cases, alive = cache_cases("max_new")
    refusals(L.samp_cache_write, base, cases + [
        ({"k": None}, ARG, b"k is NULL"), ({"v": None}, ARG, b"v is NULL"), ({"ldk": 120}, SHAPE, b"k: "), ({"ldv": 124}, ARG, b"v: "), ({"v": AT + 8}, ARG, b"v: ")])
    base = [("cache", C.addressof(ok)), ("k", AT), ("v", AT)] + [(n if n != "max_new" else "max_rows", v) for n, v in places]
    cases, alive = cache_cases("max_rows")
    refusals(L.samp_cache_read, base, cases + [({"k": None}, ARG, b"NULL"), ({"v": AT + 8}, ARG, b"aligned")])


def test_attention_cache(L):
    ok = cache()
    need = L.samp_attention_cache_workspace_bytes(5, 2, 4, 2, 64, 3, 4096)
    assert need > 0
    assert L.samp_attention_cache_workspace_bytes(5, 2, 3, 2, 64, 3, 32) == 0 and L.samp_attention_cache_workspace_bytes(5, 2, 4, 2, 80, 3, 32) == 0
    base = [("q", AT), ("ldq", 256), ("type", 0), ("heads", 4), ("cache", C.addressof(ok)), ("table", AT), ("width", 2), ("cu", AT), ("lens", AT), ("batch", 2),
            ("max_new", 3), ("max_len", 32), ("rows", 5), ("scale", 0.125), ("tree", None), ("out", AT), ("workspace", AT), ("bytes", need), ("stream", None)]
    cases, alive = cache_cases("max_new")
    refusals(L.samp_attention_cache, base, cases + [
        ({"q": None}, ARG, b"q is NULL"), ({"ldq": 248}, SHAPE, b"q: "), ({"heads": 3}, SHAPE, b"multiple"), ({"heads": 0}, SHAPE, b"multiple"), ({"heads": 1026}, SHAPE, b"1024"),
        ({"max_len": 0}, SHAPE, b"max_len"), ({"scale": 0.0}, SCALE, b"scale"), ({"scale": -1.0}, SCALE, b"scale"), ({"scale": float("nan")}, SCALE, b"scale"),
        ({"scale": float("inf")}, SCALE, b"scale"), ({"out": None}, ARG, b"out"), ({"out": AT + 8}, ARG, b"out"), ({"tree": AT + 4}, ARG, b"tree"),
        ({"tree": AT, "rows": 100, "max_new": 65}, SHAPE, b"64"), ({"max_len": 4096, "workspace": None}, SPACE, b"workspace"),
        ({"max_len": 4096, "bytes": need - 1}, SPACE, b"workspace"), ({"max_len": 4096, "workspace": AT + 8}, SPACE, b"workspace"), ({"rows": 1 << 20, "max_new": 1 << 20, "batch": 1000, "heads": 1024}, SHAPE, b"2^31"),
        ({"max_len": 1 << 30, "rows": 1 << 16, "max_new": 1 << 10, "batch": 8192, "heads": 64}, SHAPE, b"2^31")])


def test_attention_causal(L):
    base = [("q", AT), ("ldq", 256), ("k", AT), ("ldk", 128), ("v", AT), ("ldv", 128), ("type", 1), ("heads", 4), ("kv_heads", 2), ("head_dim", 64), ("cu", AT),
            ("batch", 2), ("max_len", 3), ("rows", 5), ("scale", 0.125), ("out", AT), ("stream", None)]
    refusals(L.samp_attention_causal, base, [
        ({"q": None}, ARG, b"q is"), ({"k": None}, ARG, b"k is"), ({"v": None}, ARG, b"v is"), ({"ldq": 252}, ARG, b"q: "), ({"ldk": 64}, SHAPE, b"k: "), ({"v": AT + 2}, ARG, b"v: "),
        ({"type": 2}, ARG, b"type"), ({"heads": 5}, SHAPE, b"multiple"), ({"kv_heads": 0}, SHAPE, b"multiple"), ({"head_dim": 32}, SHAPE, b"head_dim"),
        ({"cu": None}, SHAPE, b"without offsets"), ({"batch": 0}, SHAPE, b"sequences"), ({"batch": 8193}, SHAPE, b"sequences"), ({"max_len": 0}, SHAPE, b"max_len"),
        ({"cu": None, "max_len": 6}, SHAPE, b"without offsets"), ({"rows": 0}, SHAPE, b"rows"), ({"scale": float("nan")}, SCALE, b"scale"), ({"out": None}, ARG, b"out"),
        ({"batch": 8192, "max_len": 1 << 24, "rows": 1 << 24}, SHAPE, b"strips")])


def test_the_binding_refuses_tensors_that_do_not_fit():
    h = torch.zeros(2, 64, dtype=torch.float16)
    for call in (lambda: P.quantize_tokens(h), lambda: P.linear_i8_tokens(h, h, h), lambda: P.gemm_i8_tokens_packed(h, h, h, h),
                 lambda: P.attention_causal(h, h, h, None, 1), lambda: P.KVCache(h, h, h, h)):
        with pytest.raises(P.SampError, match="GPU"):
            call()
    f = torch.zeros(2, 4, 64, dtype=torch.float16)
    for t, why in ((f.float(), "bfloat16"), (f[0], "rows, heads"), (f.transpose(0, 1).contiguous().transpose(0, 1), "next to each other"), (f[..., ::2], "next to each other")):
        with pytest.raises(P.SampError, match=why):
            D._heads("q", t, -1)
    assert D._heads("q", f[:, 1:3], -1)[1] == 256 and D._heads("q", f[:1], -1)[1] == 256
    with pytest.raises(P.SampError, match="dense rows"):
        D._rows2("x", h.t())
    with pytest.raises(P.SampError, match="contiguous"):
        D._flat("t", h.t(), torch.float16, -1)
    with pytest.raises(P.SampError, match="different devices"):
        D._flat("t", h, torch.float16, 0)
    with pytest.raises(P.SampError, match="elements"):
        D._flat("t", h, torch.float16, -1, 3)
