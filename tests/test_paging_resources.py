"""The kernels of beam selection, page bookkeeping and the choice of pages fit their registers: none of them uses scratch memory."""
import os

import pytest

from test_kernel_resources import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf is not installed")
@pytest.mark.parametrize("kernel,least", [("beam_pieces_kernel", 12), ("beam_join_kernel", 1), ("fork_block_kernel", 1), ("fork_clear_kernel", 1), ("fork_count_kernel", 1),
                                          ("fork_needs_kernel", 1), ("fork_free_kernel", 1), ("fork_entries_kernel", 1), ("compact_block_kernel", 2), ("compact_bits_kernel", 1), ("compact_before_kernel", 1),
                                          ("compact_list_kernel", 1), ("compact_finish_kernel", 1), ("cache_copy_kernel", 2), ("cache_bounds_kernel", 4), ("page_scores_kernel", 4),
                                          ("select_pages_kernel", 4), ("select_scored_kernel", 1)])
def test_kernels_use_no_scratch_memory(kernel, least, tmp_path):
    found = [(name, scratch) for name, scratch in kernels(tmp_path) if kernel in name]
    assert len(found) >= least, found
    assert not [k for k in found if k[1]]
