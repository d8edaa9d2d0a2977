"""The decoder's kernels fit their registers: none of them uses scratch memory (read from the built library's metadata)."""
import os

import pytest

from test_kernel_resources import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf is not installed")
@pytest.mark.parametrize("kernel,least", [("causal_attention_kernel", 4), ("cached_attention_kernel", 8), ("join_pieces_kernel", 4), ("gemm_tokens_kernel", 16),
                                          ("gemm_tokens_few_kernel", 16), ("quantize_tokens_kernel", 12), ("cache_write_kernel", 8), ("cache_read_kernel", 8)])
def test_kernels_use_no_scratch_memory(kernel, least, tmp_path):
    found = [(name, scratch) for name, scratch in kernels(tmp_path) if kernel in name]
    assert len(found) >= least, found
    assert not [k for k in found if k[1]]
