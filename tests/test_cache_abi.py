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


def test_chunks_fit_the_workspace(hq, tmp_path):
    """The chunks that the kernel cuts a batch into (its arithmetic, here in Python) are never more
    than the bound that the grid and the workspace go by, whatever the lengths."""
    src = tmp_path / "rule.cpp"
    src.write_text('#include "hq_internal.h"\n#include <cstdio>\n#include <cstdlib>\n'
                   'int main(int, char** a) {\n  printf("%d %d %ld %ld\\n", HQ_CACHE_WG_TARGET, HQ_CACHE_LEAST,\n'
                   '         (long)hq_cache_items(atol(a[1]), atol(a[2]), atol(a[3])),\n'
                   '         (long)hq_cache_joins(atol(a[1]), atol(a[2])));\n}\n')
    exe = tmp_path / "rule"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2606_23406_amd", "csrc"), "-o", str(exe),
                    str(src)], check=True)
    L = hq.lib()
    rng = np.random.default_rng(0)
    for batch, heads, blocks in [(1, 1, 1), (8, 8, 63), (8, 8, 64), (8, 8, 65), (1, 8, 8192), (3, 3, 400), (64, 8, 33), (65, 2, 700), (300, 1, 1000),
                                 (2000, 16, 64), (1, 512, 100), (7, 600, 90)]:
        target, least, items, joins = map(int, subprocess.run([str(exe), str(batch), str(heads), str(16 * blocks)],
                                                              capture_output=True, text=True, check=True).stdout.split())
        if 16 * blocks <= 1024:  # no sequence is split: workgroup j takes sequence j
            assert items == batch
            assert L.hq_cache_attention_workspace_bytes(C.byref(hq.CacheStruct(None, None, 1, 16, heads, 3, 0, None)),
                                                        batch, 2 * heads, blocks) == 0
            continue
        for lens in (np.full(batch, 16 * blocks), rng.integers(0, 16 * blocks + 1, batch),
                     np.where(np.arange(batch) == 0, 16 * blocks, 1), np.zeros(batch, np.int64)):
            even = -(-int(lens.sum()) * heads // target)
            for eighths in range(8, 17):  # the kernel takes one of these
                chunk = max(least, ((even * eighths >> 3) + 127) // 128 * 128)
                n = np.where(lens == 0, 1, -(-lens // chunk))
                assert batch <= n.sum() <= items, (batch, heads, blocks)
                assert (n > 1).sum() <= joins, (batch, heads, blocks)
                own = -(-lens // (n * 128)) * 128  # the even chunk of each
                assert (own * n >= lens).all() and (own * (n - 1) <= lens).all()
        c = hq.CacheStruct(None, None, 1, 16, heads, 3, 0, None)
        assert items * heads * 2 * 130 * 4 + batch * 8 + (joins + 1) * 4 == L.hq_cache_attention_workspace_bytes(C.byref(c), batch, 2 * heads, blocks)


def test_the_oracle_transforms_back():
    x = np.random.default_rng(0).standard_normal((3, 2 * R.N))
    y, _ = R.transform(x, 5, 2)
    back = (y @ R.hadamard() / R.N).reshape(3, -1) * R.signs(5, 2 * R.N)
    assert np.abs(back - x).max() < 1e-12
    assert np.isnan(R.e4m3_values(np.array([0x7F, 0xFF]))).all() and R.e4m3_values(np.array([0x7E]))[0] == 448
