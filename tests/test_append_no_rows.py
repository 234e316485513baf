"""A step without new tokens: an append of no rows, whose tensors have no address, is right with queries too."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23406_amd", "csrc")

PROGRAM = r"""
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include "hq_internal.h"

static int launched;
extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
int hq_launch_rope_table(const hq_rope_table_args&, void*) { return 0; }
int hq_launch_rope(const hq_rope_args&, void*) { return 0; }
int hq_launch_cache_attention(const hq_cache_attn_args&, int, void*) { return 0; }
int hq_launch_cache_append(const hq_cache_append_args&, int, void*) { return ++launched, 0; }

int main() {
  alignas(16) static char some[64];  // addresses
  hq_plan_s p = {};
  p.tile = HQ_TILE;
  p.cols = 512;
  hq_cache k = {some, some + 16, 8, 64, 4, HQ_INT8, 0, nullptr}, v = {some + 32, some + 48, 8, 64, 4, HQ_INT8, 0, nullptr};
  const hq_rotary r = {(const float*)some, 100, 128, 0, 1, 0, nullptr, nullptr};
  for (int64_t rows = 0; rows < 2; ++rows)
    for (int heads = 0; heads <= 8; heads += 8)
      for (int bad = 0; bad < 2; ++bad)
        printf("%d ", hq_cache_append(&p, nullptr, 512, &k, &p, nullptr, 512, &v, HQ_BF16, rows, nullptr, &r, nullptr, nullptr,
                                      1024, heads, nullptr, bad ? HQ_INT8 : HQ_BF16, 1024, nullptr));
  printf("%d\n", launched);
}
"""


def test_no_rows_and_no_addresses(tmp_path):
    """Nothing is launched and nothing refused but a type that queries cannot have; a row needs addresses."""
    src, exe = tmp_path / "append.cpp", tmp_path / "append"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, "-o", str(exe), str(src),
                    os.path.join(CSRC, "hq_rope_host.cpp")], check=True, timeout=300)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout
    assert list(map(int, out.split())) == [0, 0, 0, -1, -1, -1, -1, -1, 0]


@pytest.mark.gpu
def test_a_step_without_new_tokens():
    from paper_2606_23406_amd import hq
    kp, vp = (hq.hq_plan(cols=512, bps=4.0, rht_seed=s) for s in (1, 2))
    kc, vc = (hq.Cache(p, 2, 16, hq.HQ_E4M3, heads=4) for p in (kp, vp))
    rope = hq.Rope(torch.ones((8, 2, 64), device="cuda"))
    kv = torch.empty((0, 512), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((0, 2048), dtype=torch.bfloat16, device="cuda")
    slots, pos = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty((0, 1), dtype=torch.int32, device="cuda")
    out = hq.hq_cache_append(kp, kv, kc, vp, kv, vc, slots, rope, pos, q=q)
    assert out.shape == (0, 2048) and out.dtype == torch.bfloat16
    assert hq.hq_cache_append(kp, kv, kc, vp, kv, vc, slots, rope, pos) is None
    assert hq.hq_cache_append(kp, kv, kc, None, None, None, slots, rope, pos, q=q, q_out=q) is q
    assert not kc.codes.any() and not vc.codes.any() and kc.read_stats()["status"] == 0
