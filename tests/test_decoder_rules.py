"""The rules that choose the kernels of the decoder's projection and cache (csrc/decoder_rules.h), compiled for the host, and that the shapes of
test_gpu_decoder_kernels.py reach every one of them."""
import ctypes as C
import os
import subprocess

import pytest

from test_gpu_decoder_kernels import CACHES, FEW, TILED

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2209_09130_amd", "csrc")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text('#include "decoder_rules.h"\n'
                                 'using namespace samp;\n'
                                 'extern "C" {\n'
                                 'int few(int M, int K) { return tokens_few(M, K); }\n'
                                 'int few_blocks(int K) { return tokens_few_blocks(K); }\n'
                                 'int fused(int M, int N, int K) { return tokens_fused(M, N, K); }\n'
                                 'int fused_any(int M, int K) { return tokens_fused_any(M, K); }\n'
                                 'int tile(int M, int N) { return tokens_tile(M, N); }\n'
                                 'int rows(int t) { return 16 * TOKENS_TILES[t].mt; }\n'
                                 'int channels(int t) { return 64 * TOKENS_TILES[t].ntw; }\n'
                                 'int depth(int t, int K) { return tokens_depth(t, K); }\n'
                                 'int band(int t) { return tokens_band(t); }\n'
                                 'int passes(long rows, int kv_heads) { return cache_passes(rows, kv_heads); }\n'
                                 '}\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "rules.so"), str(d / "rules.cpp")], check=True)
    lib = C.CDLL(str(d / "rules.so"))
    lib.passes.argtypes = [C.c_long, C.c_int]
    return lib


def test_the_shapes_of_many_rows_reach_every_tile_depth_band_and_remainder(rules):
    seen, parts = {}, {}
    for tile, depth, M, N, K in TILED:
        assert not rules.few(M, K) and rules.tile(M, N) == tile and rules.depth(tile, K) == depth, (M, N, K)
        rows = -(-M // rules.rows(tile))
        seen.setdefault((tile, depth), []).append(K // (128 * depth) and K % (128 * depth))
        parts.setdefault(tile, []).append((M % rules.rows(tile) > 0, N % rules.channels(tile) > 0, rows > rules.band(tile) and rows % rules.band(tile) > 0))
    assert sorted(seen) == [(0, 2), (0, 4), (1, 2), (1, 4), (2, 2), (2, 4), (3, 2), (4, 2)]
    for (tile, depth), left in seen.items():
        assert any(left), (tile, depth)                          # whole rounds of the ring, and some 64s of K behind them
    assert {k for left in seen.values() for k in left} >= {0, 64, 192, 448}
    for tile, p in parts.items():
        assert all(any(x[i] for x in p) for i in range(3)), (tile, p)        # a partial row tile, a partial channel tile, a partial last band


def test_the_shapes_of_few_rows_reach_every_kernel(rules):
    kinds = {(rules.few_blocks(K), bool(rules.fused(M, N, K))) for M, N, K in FEW if rules.few(M, K)}
    assert kinds == {(b, f) for b in (2, 4, 8, 16) for f in (True, False)}
    assert any(not rules.few(M, K) and M <= 16 for M, N, K in FEW)
    assert {M for M, N, K in FEW if rules.fused(M, N, K)} >= {1, 2, 3, 4, 5, 8, 9, 16}


def test_few_rows_are_quantised_in_the_same_launch_where_that_was_measured_to_be_no_loss(rules):
    for M, N, K, one in ((1, 4096, 4096, 1), (8, 8192, 4096, 1), (12, 4096, 4096, 0), (12, 8192, 4096, 0), (16, 6144, 3328, 0), (16, 4096, 2048, 1), (16, 8192, 2048, 0),
                         (1, 5120, 5120, 0), (8, 4096, 5120, 1), (9, 4096, 5120, 0), (1, 8192, 8192, 0), (1, 2048, 8192, 1), (17, 4096, 1024, 0)):
        assert rules.fused(M, N, K) == one, (M, N, K)
    for M in range(1, 17):                                       # no workspace is asked for only where no N needs one
        for K in (64, 2048, 2112, 4096, 4160, 8192):
            assert rules.fused_any(M, K) == all(rules.fused(M, N, K) for N in (16, 4096, 4112, 8192)), (M, K)


def test_the_caches_reach_both_kernels(rules):
    for lens, new, G, D, page in CACHES:
        assert rules.passes(sum(new), G) == 4 and rules.passes(sum(lens), G) == 4
    assert rules.passes(2048, 8) == 1 and rules.passes(4096, 8) == 4 and rules.passes(1 << 24, 1024) == 4
