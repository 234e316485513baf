"""Refusals of the cache and norm entry points that need no GPU, the split rule, and
the 64-bit oracle against itself."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from tests import cache64 as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import build, hq as H
    if not os.path.exists(build.LIB):
        build.build()
    return H


def test_null_plans_and_caches(hq):
    L = hq.lib()
    c = hq.CacheStruct()
    assert L.hq_cache_write(None, None, 0, None, None, None, 0, None, 0, 0, None, None) == -1
    assert L.hq_cache_write(None, None, 0, C.byref(c), None, None, 0, None, 0, 1, None, None) == -1
    assert L.hq_cache_read(None, C.byref(c), None, 1, None, 0, 0, None) == -1
    assert L.hq_cache_attention(None, C.byref(c), None, C.byref(c), None, 0, 1, 8, 0.1, None, 1, None, None, 0, None, 0,
                                None) == -1
    for fn in (L.hq_rmsnorm_act_prep, L.hq_rmsnorm_act_prep_fp8):
        assert fn(None, None, 0, None, 0, None, 0, 1e-5, 1, None, 0, None, None, None) == -1


def test_workspace_bytes(hq):
    L = hq.lib()
    c = hq.CacheStruct(None, None, 8, 64, 4, 3, 0, None)
    n = L.hq_cache_attention_workspace_bytes
    assert n(None, 1, 8, 4) == 0 and n(C.byref(c), 0, 8, 4) == 0 and n(C.byref(c), 1, 6, 4) == 0
    assert n(C.byref(c), 1, 8, 0) == 0 and n(C.byref(c), 1, 0, 4) == 0
    last = 0
    for batch in (1, 2, 7, 64, 500):
        for blocks in (1, 2, 30, 1000):
            assert n(C.byref(c), batch, 8, blocks) >= n(C.byref(c), max(1, batch // 2), 8, max(1, blocks // 2))
    assert n(C.byref(c), 1, 16, 100) >= n(C.byref(c), 1, 8, 100) > last


def test_split_rule(hq, tmp_path):
    """Each sequence gets at least one split, and the partial sums fit what the
    workspace bound allows, over many shapes."""
    src = tmp_path / "rule.cpp"
    src.write_text('#include "hq_internal.h"\n#include <cstdio>\n#include <initializer_list>\n'
                   'int main() {\n  for (long h : {1L, 2L, 7L, 8L, 100L, 511L, 512L, 513L, 4000L, 100000L})\n'
                   '    for (long t : {1L, 16L, 127L, 128L, 129L, 1000L, 8192L, 131072L, 1L << 30})\n'
                   '      printf("%ld %ld %ld\\n", h, t, (long)hq_cache_splits(h, t));\n}\n')
    exe = tmp_path / "rule"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2606_23406_amd", "csrc"), "-o", str(exe),
                    str(src)], check=True)
    L = hq.lib()
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        heads, tokens, splits = map(int, line.split())
        assert 1 <= splits <= (tokens + 127) // 128
        c = hq.CacheStruct(None, None, 1, 16, heads, 3, 0, None)
        blocks = (tokens + 15) // 16
        assert heads * splits * 130 * 4 <= L.hq_cache_attention_workspace_bytes(C.byref(c), 1, heads, blocks)


def test_the_oracle_transforms_back():
    x = np.random.default_rng(0).standard_normal((3, 2 * R.N))
    y, _ = R.transform(x, 5, 2)
    back = (y @ R.hadamard() / R.N).reshape(3, -1) * R.signs(5, 2 * R.N)
    assert np.abs(back - x).max() < 1e-12
    assert np.isnan(R.e4m3_values(np.array([0x7F, 0xFF]))).all() and R.e4m3_values(np.array([0x7E]))[0] == 448
