"""What the entry points of beam selection, page bookkeeping and attention over chosen pages refuse, on the host, before any launch (no GPU is needed, the pointers are host memory
that nothing reads)."""
import ctypes as C

import pytest
import torch

import paper_2209_09130_amd as P
from paper_2209_09130_amd import decoder as D
from test_decoder_refusals import ARG, AT, L, SCALE, SHAPE, SPACE, cache, cache_cases, refusals  # noqa: F401

BIG = 1 << 40


def bounds(**change):
    f = dict(codes=AT, steps=AT)
    f.update(change)
    return D._BoundsStruct(*f.values())


def test_beam_select(L):
    need = L.samp_beam_select_workspace_bytes(0, 2, 3, 100, 5)
    assert need > 0
    assert not any(L.samp_beam_select_workspace_bytes(*a) for a in ((3, 2, 3, 100, 5), (0, 0, 3, 100, 5), (0, 2, 65, 100, 5), (0, 2, 3, 0, 5), (0, 2, 3, 100, 65)))
    base = [("logits", AT), ("ld", 100), ("type", 0), ("scores", AT), ("finished", None), ("end", -5), ("batch", 2), ("beams", 3), ("vocab", 100), ("keep", 5), ("best", AT),
            ("parents", AT), ("tokens", AT), ("workspace", AT), ("bytes", need), ("stream", None)]
    refusals(L.samp_beam_select, base, [
        ({"logits": None}, ARG, b"NULL"), ({"scores": None}, ARG, b"NULL"), ({"best": None}, ARG, b"NULL"), ({"parents": None}, ARG, b"NULL"), ({"tokens": None}, ARG, b"NULL"),
        ({"type": 3}, ARG, b"type"), ({"type": -1}, ARG, b"type"), ({"logits": AT + 1}, ARG, b"aligned"), ({"logits": AT + 2, "type": 2}, ARG, b"aligned"), ({"scores": AT + 2}, ARG, b"aligned"),
        ({"ld": 99}, SHAPE, b"leading"), ({"ld": BIG}, SHAPE, b"leading"), ({"batch": 0}, SHAPE, b"sequences"), ({"batch": 8193}, SHAPE, b"sequences"), ({"beams": 0}, SHAPE, b"beams"),
        ({"beams": 65}, SHAPE, b"beams"), ({"vocab": 0}, SHAPE, b"vocabulary"), ({"vocab": (1 << 19) + 1, "ld": 1 << 20}, SHAPE, b"vocabulary"), ({"keep": 0}, SHAPE, b"keep"),
        ({"keep": 65}, SHAPE, b"keep"), ({"workspace": None}, SPACE, b"workspace"), ({"workspace": AT + 16}, SPACE, b"workspace"), ({"bytes": need - 1}, SPACE, b"workspace")])


def test_pages_fork(L):
    need = L.samp_pages_fork_workspace_bytes(100000, 4, 8, 3)
    assert need >= 3 * 400000 and L.samp_pages_fork_workspace_bytes(100, 4, 8, 3) == 0
    assert not any(L.samp_pages_fork_workspace_bytes(*a) for a in ((0, 4, 8, 3), (1 << 30, 4, 8, 3), (100000, 0, 8, 3), (100000, 4, 0, 3), (100000, 4, 8, 8193)))
    base = [("refs", AT), ("pages", 100), ("table", AT), ("lens", AT), ("rows_from", 4), ("width", 8), ("page_len", 16), ("parents", None), ("cu", None), ("max_new", 1), ("rows", 3),
            ("refs_out", AT + 1024), ("table_out", AT + 2048), ("lens_out", AT + 3072), ("copies", AT), ("lacking", AT), ("workspace", AT), ("bytes", need), ("stream", None)]
    refusals(L.samp_pages_fork, base, [({n: None}, ARG, b"NULL") for n in ("refs", "table", "lens", "refs_out", "table_out", "lens_out", "copies", "lacking")] + [
        ({"pages": 0}, SHAPE, b"pages"), ({"pages": (1 << 26) + 1}, SHAPE, b"pages"), ({"page_len": 8}, SHAPE, b"power of two"), ({"page_len": 48}, SHAPE, b"power of two"),
        ({"rows": 0}, SHAPE, b"rows"), ({"rows": 8193}, SHAPE, b"rows"), ({"rows_from": 0}, SHAPE, b"rows"), ({"rows_from": 8193}, SHAPE, b"rows"), ({"width": 0}, SHAPE, b"width"),
        ({"max_new": -1}, SHAPE, b"max_new"), ({"rows": 8192, "width": (1 << 17) + 1}, SHAPE, b"2^30"), ({"rows_from": 8192, "width": (1 << 17) + 1}, SHAPE, b"2^30"),
        ({"refs_out": AT}, ARG, b"overlap"), ({"table_out": AT}, ARG, b"overlap"), ({"lens_out": AT}, ARG, b"overlap"),
        ({"pages": 100000, "workspace": None}, SPACE, b"workspace"), ({"pages": 100000, "bytes": need - 1}, SPACE, b"workspace")])


def test_pages_compact_and_cache_copy(L):
    need = L.samp_pages_compact_workspace_bytes(100000, 50)
    assert need > 0 and L.samp_pages_compact_workspace_bytes(100, 50) == 0 and L.samp_pages_compact_workspace_bytes(0, 50) == 0 and L.samp_pages_compact_workspace_bytes(10, -1) == 0
    base = [("refs", AT), ("pages", 100), ("table", AT), ("entries", 50), ("page_len", 16), ("refs_out", AT + 1024), ("table_out", AT + 2048), ("copies", AT), ("used", AT),
            ("workspace", AT), ("bytes", need), ("stream", None)]
    refusals(L.samp_pages_compact, base, [({n: None}, ARG, b"NULL") for n in ("refs", "table", "refs_out", "table_out", "copies", "used")] + [
        ({"pages": 0}, SHAPE, b"pages"), ({"entries": -1}, SHAPE, b"entries"), ({"page_len": 2048}, SHAPE, b"power of two"), ({"refs_out": AT}, ARG, b"overlap"),
        ({"table_out": AT}, ARG, b"overlap"), ({"pages": 100000, "workspace": AT + 8}, SPACE, b"workspace"), ({"pages": 100000, "bytes": 0}, SPACE, b"workspace")])
    ok, kb = cache(), bounds()
    base = [("cache", C.addressof(ok)), ("bounds", None), ("copies", AT), ("n", 3), ("stream", None)]
    bad = [cache(**c) for c in (dict(k=None), dict(head_dim=96), dict(page_len=8), dict(pages=0))]
    refusals(L.samp_cache_copy, base, [({"cache": C.addressof(b)}, code, word) for b, code, word in zip(bad, (ARG, SHAPE, SHAPE, SHAPE), (b"NULL", b"head_dim", b"page_len", b"pages"))] + [
        ({"cache": None}, ARG, b"cache"), ({"copies": None}, ARG, b"copies"), ({"n": 0}, SHAPE, b"copies"), ({"n": (1 << 26) + 1}, SHAPE, b"copies"),
        ({"bounds": C.addressof(bounds(codes=None))}, ARG, b"bounds"), ({"bounds": C.addressof(bounds(steps=AT + 4))}, ARG, b"aligned")])
    assert kb is not None


def test_cache_bounds(L):
    ok, kb = cache(), bounds()
    base = [("cache", C.addressof(ok)), ("bounds", C.addressof(kb)), ("table", AT), ("width", 2), ("cu", AT), ("lens", AT), ("batch", 2), ("max_new", 3), ("rows", 5), ("stream", None)]
    cases, alive = cache_cases("max_new")
    cases = [c for c in cases if "type" not in c[0]]
    nothing = [bounds(codes=None), bounds(steps=None), bounds(codes=AT + 8)]
    refusals(L.samp_cache_bounds, base, cases + [({"bounds": None}, ARG, b"bounds")] + [({"bounds": C.addressof(b)}, ARG, b"bounds") for b in nothing])


def test_cache_select_and_attention_sparse(L):
    ok, kb = cache(), bounds()
    assert L.samp_cache_select_workspace_bytes(2, 2, 256) == 0 and L.samp_cache_select_workspace_bytes(2, 2, 300) >= 2 * 2 * 300 * 4
    assert L.samp_cache_select_workspace_bytes(0, 2, 300) == 0 and L.samp_cache_select_workspace_bytes(2, 2, 32769) == 0
    need = L.samp_attention_sparse_workspace_bytes(5, 2, 4, 2, 64, 16, 40, 3, 32, 6)
    assert need >= 2 * 2 * 6 * 4 + 2 * 4
    assert not any(L.samp_attention_sparse_workspace_bytes(*a) for a in ((5, 2, 3, 2, 64, 16, 40, 3, 32, 6), (5, 2, 4, 2, 64, 20, 40, 3, 32, 6), (5, 2, 4, 2, 64, 16, 40, 3, 32, 0),
                                                                         (5, 2, 4, 2, 64, 16, 0, 3, 32, 6), (5, 2, 4, 2, 80, 16, 40, 3, 32, 6)))
    head = [("q", AT), ("ldq", 256), ("type", 0), ("heads", 4), ("cache", C.addressof(ok)), ("bounds", C.addressof(kb)), ("table", AT), ("width", 40), ("cu", AT), ("lens", AT), ("batch", 2),
            ("max_new", 3)]
    choice = [({"q": None}, ARG, b"q is NULL"), ({"ldq": 248}, SHAPE, b"q: "), ({"heads": 3}, SHAPE, b"multiple"), ({"bounds": None}, ARG, b"bounds"), ({"keep": 0}, SHAPE, b"keep"),
              ({"sinks": -1}, SHAPE, b"sinks"), ({"recent": 1}, SHAPE, b"recent"), ({"sinks": 5}, SHAPE, b"keep"), ({"width": 32769}, SHAPE, b"32768"), ({"keep": 40000}, SHAPE, b"keep"),
              ({"recent": 2 ** 31 - 1}, SHAPE, b"keep")]
    cases, alive = cache_cases("max_new")
    base = head + [("rows", 5), ("keep", 6), ("sinks", 1), ("recent", 2), ("tables", AT), ("lens_out", AT + 64), ("workspace", AT), ("bytes", 8192), ("stream", None)]
    refusals(L.samp_cache_select, base, cases + choice + [({"tables": None}, ARG, b"NULL"), ({"lens_out": None}, ARG, b"NULL"), ({"lens_out": AT}, ARG, b"overlap"),
                                                          ({"width": 300, "workspace": None}, SPACE, b"workspace"), ({"width": 300, "bytes": 1000}, SPACE, b"workspace")])
    base = head + [("max_len", 32), ("rows", 5), ("keep", 6), ("sinks", 1), ("recent", 2), ("scale", 0.125), ("tree", None), ("out", AT), ("workspace", AT), ("bytes", 1 << 30), ("stream", None)]
    refusals(L.samp_attention_sparse, base, cases + choice + [
        ({"max_len": 0}, SHAPE, b"max_len"), ({"scale": 0.0}, SCALE, b"scale"), ({"scale": float("nan")}, SCALE, b"scale"), ({"out": None}, ARG, b"out"), ({"out": AT + 8}, ARG, b"out"),
        ({"tree": AT + 4}, ARG, b"tree"), ({"tree": AT, "rows": 100, "max_new": 65, "recent": 6, "keep": 10}, SHAPE, b"64"), ({"workspace": None}, SPACE, b"workspace"),
        ({"bytes": need - 1}, SPACE, b"workspace"), ({"workspace": AT + 8}, SPACE, b"workspace")])


def test_launches_of_more_threads_than_there_are(L):
    """A launch has fewer than 2^32 threads: one sequence below, the next thing that is wrong is named, the workspace."""
    ok, kb, many = cache(kv_heads=8), bounds(), cache(kv_heads=1024)
    head = [("q", AT), ("ldq", 1 << 17), ("type", 0), ("heads", 8), ("cache", C.addressof(ok)), ("bounds", C.addressof(kb)), ("table", AT), ("width", 32768), ("cu", AT), ("lens", AT),
            ("batch", 8192), ("max_new", 1)]
    tail = [("keep", 6), ("sinks", 1), ("recent", 1)]
    choice = head + [("rows", 8192)] + tail + [("tables", AT), ("lens_out", AT + 64), ("workspace", None), ("bytes", 1 << 40), ("stream", None)]
    sparse = head + [("max_len", 32), ("rows", 8192)] + tail + [("scale", 0.125), ("tree", None), ("out", AT), ("workspace", None), ("bytes", 1 << 40), ("stream", None)]
    wide = {"cache": C.addressof(many), "heads": 1024}               # 256 threads for each 128 pages, or fewer: 2^24 blocks are one too many
    cases = [({}, SHAPE, b"launch"), ({"batch": 8191}, SPACE, b"workspace"), ({"width": 32641}, SHAPE, b"launch"), ({"width": 32640}, SPACE, b"workspace"),
             ({**wide, "width": 257, "batch": 5461}, SPACE, b"workspace"), ({**wide, "width": 257, "batch": 5462}, SHAPE, b"launch")]
    refusals(L.samp_cache_select, choice, cases)
    refusals(L.samp_attention_sparse, sparse, cases)
    assert L.samp_cache_select_workspace_bytes(8192, 8, 32768) == 0 and L.samp_cache_select_workspace_bytes(8191, 8, 32768) >= 8191 * 8 * 32768 * 4
    assert L.samp_attention_sparse_workspace_bytes(8192, 8192, 8, 8, 64, 16, 32768, 1, 32, 6) == 0 and L.samp_attention_sparse_workspace_bytes(8191, 8191, 8, 8, 64, 16, 32768, 1, 32, 6) > 0
    base = [("logits", AT), ("ld", 1 << 19), ("type", 0), ("scores", AT), ("finished", None), ("end", 0), ("batch", 8192), ("beams", 64), ("vocab", 1 << 19), ("keep", 5), ("best", AT),
            ("parents", AT), ("tokens", AT), ("workspace", None), ("bytes", 0), ("stream", None)]
    refusals(L.samp_beam_select, base, [({}, SHAPE, b"launch"), ({"vocab": (1 << 19) - 7}, SHAPE, b"launch"), ({"vocab": (1 << 19) - 7 - (1 << 15)}, SPACE, b"workspace"), ({"type": 2}, SHAPE, b"launch"), ({"batch": 4096}, SPACE, b"workspace")])


def test_the_binding_refuses_what_is_not_on_the_gpu():
    i = torch.zeros(2, 4, dtype=torch.int32)
    for call in (lambda: P.beam_select(torch.zeros(2, 8), torch.zeros(2), 1), lambda: P.pages_fork(i[0], i, i[:, 0], 16), lambda: P.pages_compact(i[0], i, 16),
                 lambda: P.KeyBounds(torch.zeros(1, 1, 2, 64, dtype=torch.int8), torch.zeros(1, 1))):
        with pytest.raises(P.SampError, match="GPU"):
            call()


@pytest.fixture
def passed(monkeypatch):
    """What the binding hands to each entry point, on the CPU: nothing is called."""
    seen = {}

    def entry(name):
        argtypes = D._SIGNATURES[name]

        def call(*args):
            assert len(args) == len(argtypes)
            seen[name] = [t(a).value for t, a in zip(argtypes, args)]          # as ctypes converts them
            return 0
        return call

    monkeypatch.setattr(D, "_fn", entry)
    monkeypatch.setattr(D, "_device", lambda t: -1)
    monkeypatch.setattr(D, "_current_device", lambda: -1)
    monkeypatch.setattr(D, "_raw_stream", lambda device: 0)
    D._workspace_bytes.cache_clear()
    yield seen
    D._workspace_bytes.cache_clear()


def test_numbers_past_int32_are_not_cut(passed):
    """ctypes passes the low 32 bits of a larger number: the entry has to see one that it refuses, or that counts as the largest."""
    i = torch.zeros(2, 4, dtype=torch.int32)
    most = 2 ** 31 - 1
    for n, want in ((16, 16), ((1 << 32) + 16, most), (-(1 << 32) + 16, -1)):
        P.pages_fork(i[0], i, i[0, :2], n)
        assert passed["samp_pages_fork"][6] == want
        P.pages_compact(i[0], i, n)
        assert passed["samp_pages_compact"][4] == want
        cache_ = P.KVCache.empty(4, 2, 16, 64, device="cpu")
        P.cache_bounds(cache_, P.KeyBounds.empty(cache_), i, torch.zeros(3, dtype=torch.int32), i[0, :2], 3, rows=n)
        assert passed["samp_cache_bounds"][8] == want
