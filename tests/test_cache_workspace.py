"""The workspace of a cache attention never shrinks as one argument of the call grows, on the CPU."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def size():
    from paper_2606_23406_amd import build, hq
    if not os.path.exists(build.LIB):
        build.build()
    L = hq.lib()
    return lambda heads, block_tokens, *call: L.hq_cache_attention_workspace_bytes(
        C.byref(hq.CacheStruct(None, None, 1, block_tokens, heads, hq.HQ_INT8, 0, None)), *call)


@pytest.mark.parametrize("heads", [1, 2, 3, 8, 9, 16, 32, 100, 511, 512, 600])
@pytest.mark.parametrize("block_tokens", [16, 48, 512])
def test_never_less_for_a_larger_call(size, heads, block_tokens):
    """Over tables around 1024 tokens (none needed below) and batches around every switch of the rules:
    64 sequences, and where a sequence's most chunks exceed the even share of the workgroups."""
    edge = 1024 // block_tokens
    blocks = sorted({1, 2, edge - 1, edge, edge + 1, edge + 2, 2 * edge, 5 * edge, 40 * edge} - {0})
    batches = list(range(1, 70)) + [100, 199, 256, 257, 258, 259, 511, 512, 513, 514, 1025, 5000]
    for group in (1, 3, 15):
        for m in blocks:
            for b in batches:
                n = size(heads, block_tokens, b, heads * group, m)
                assert (n > 0) == (m * block_tokens > 1024)
                assert size(heads, block_tokens, b + 1, heads * group, m) >= n, (b, group, m)
                assert size(heads, block_tokens, b, heads * (group + 1), m) >= n, (b, group, m)
                assert size(heads, block_tokens, b, heads * group, m + 1) >= n, (b, group, m)
