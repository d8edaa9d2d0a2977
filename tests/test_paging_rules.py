"""The rules that choose the kernels of beam selection, page bookkeeping and the choice of pages (csrc/decoder_rules.h), compiled for the host, and that the GPU tests' sizes lie on
both sides of each."""
import ctypes as C
import os
import subprocess

import pytest

from test_gpu_pages import LARGE, SIZES

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2209_09130_amd", "csrc")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("paging")
    (d / "rules.cpp").write_text('#include "decoder_rules.h"\n'
                                 'using namespace samp;\n'
                                 'extern "C" {\n'
                                 'int chunks(int large, int wide, int vocab) { return piece_chunks(large ? LONG_PIECE : SHORT_PIECE, wide, vocab); }\n'
                                 'int values(int large, int wide) { return (large ? LONG_PIECE : SHORT_PIECE).threads * (large ? LONG_PIECE : SHORT_PIECE).vectors * (wide ? 4 : 8); }\n'
                                 'int large(int wide, int rows, int vocab) { return long_pieces(wide, rows, vocab); }\n'
                                 'long fork_lds(long pages, long from, long rows) { return fork_block_lds(pages, from, rows); }\n'
                                 'int fork(long pages, long from, long width, long rows) { return fork_in_block(pages, from, width, rows); }\n'
                                 'long compact_lds(long pages) { return compact_block_lds(pages); }\n'
                                 'int compact(long pages, long entries) { return compact_in_block(pages, entries); }\n'
                                 'int apart(int width) { return scores_apart(width); }\n'
                                 '}\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "rules.so"), str(d / "rules.cpp")], check=True)
    lib = C.CDLL(str(d / "rules.so"))
    for name, n in (("fork_lds", 3), ("fork", 4), ("compact_lds", 1), ("compact", 2)):
        getattr(lib, name).argtypes = [C.c_long] * n
    lib.fork_lds.restype = lib.compact_lds.restype = C.c_long
    return lib


def test_pieces_cover_a_row_that_begins_anywhere(rules):
    for wide in (0, 1):
        vector = 4 if wide else 8
        for large in (0, 1):
            for vocab in (1, 7, 8, 2047, 2048, 2049, 16384, 21128, 32768, 128256, 1 << 19):
                n, values = rules.chunks(large, wide, vocab), rules.values(large, wide)
                assert n * values >= vocab + vector - 1 > (n - 1) * values
                # a token fits 20 bits, and the places of a piece an int
                assert n * values < 1 << 20
    # first entries of all lists and the candidates that are ranked, 16 bytes each, fit the LDS of a CU
    for wide in (0, 1):
        for vocab in (1000, 30000, 128256, 300000, 1 << 19):
            for beams in (1, 4, 8, 16, 32, 64):
                for batch in (1, 2, 16, 64, 8192):
                    lists = beams * rules.chunks(rules.large(wide, batch * beams, vocab), wide, vocab)
                    assert 16 * (lists + 64 * 65 // 2) <= 150 << 10, (wide, vocab, beams, batch)


def test_both_pieces_are_tested(rules):
    assert not rules.large(0, 65 * 8, 33001) and rules.large(1, 65 * 8, 33001) and rules.large(0, 66 * 8, 45003) and rules.large(1, 66 * 8, 45003)
    assert rules.large(1, 2, 1 << 19) == 0 and rules.large(0, 160, 32000) == 0 and rules.large(1, 160, 32000)


def test_bookkeeping_in_one_block_fits_the_lds(rules):
    static = 4096
    for pages in (1, 1000, 8192, 8193, 12000, 15000, 20000):
        if rules.compact(pages, 100):
            assert rules.compact_lds(pages) + static <= 64 << 10 and pages <= 8 * 1024             # as much as a launch has by itself, eight pages a thread
        for rows in (1, 256, 2000, 8192):
            if rules.fork(pages, rows, 4, rows):
                assert rules.fork_lds(pages, rows, rows) + static <= 160 << 10 and pages < 65536                   # (the list of free pages is of 16 bits)
    assert rules.fork(4000, 256, 40, 256) and not rules.fork(9000, 1024, 64, 1024) and not rules.fork(40000, 4, 4, 4)
    assert rules.compact(8192, 65536) and not rules.compact(8193, 1) and not rules.compact(10, 65537)


def test_both_ways_of_bookkeeping_are_tested(rules):
    for rows, width, _, pages in SIZES:
        assert rules.fork(pages, rows, width, rows), (rows, width, pages)
    assert any(not rules.fork(pages, rows, width, rows) and rows * width > 49152 for rows, width, _, pages in LARGE)
    assert any(not rules.fork(pages, rows, width, rows) and pages > 15000 for rows, width, _, pages in LARGE)
    assert rules.fork_lds(8000, 60, 60) > 64 << 10 and rules.fork(8000, 60, 8, 60)


def test_scores_of_a_block_are_those_of_its_waves(rules):
    assert not rules.apart(256) and rules.apart(257)
