"""Split sequences anywhere in a batch, over many KV heads: every one is joined (against tests/cache64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R

pytestmark = pytest.mark.gpu
N, BT, BLOCKS = R.N, 64, 12


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def case(hq, fmt, batch, heads, group, seed):
    """Tables over a small cache (blocks repeat), 8192 tokens wide."""
    kp, vp = R.plans(hq, heads)
    kc, vc = (R.random_cache(hq, p, fmt, BLOCKS, heads, BT, seed + i) for i, p in enumerate((kp, vp)))
    g = torch.Generator().manual_seed(seed + 2)
    table = torch.randint(0, BLOCKS, (batch, 8192 // BT), generator=g).to(torch.int32)
    return kp, vp, kc, vc, table, torch.randn((batch, heads * group, N), generator=g)


@pytest.mark.parametrize("fmt,batch,heads,group", [("int8", 34, 16, 1), ("e4m3", 64, 16, 2), ("mxfp4", 58, 9, 1),
                                                   ("int8", 33, 32, 1), ("e4m3", 48, 12, 3), ("mxfp4", 33, 64, 1),
                                                   ("int8", 65, 16, 1), ("e4m3", 64, 8, 1)])
def test_long_sequences_at_the_end(hq, fmt, batch, heads, group):
    print(f"[cache] joins {fmt} {batch} x {heads} x {group}", flush=True)
    kp, vp, kc, vc, table, q = case(hq, fmt, batch, heads, group, batch + heads)
    lens = torch.full((batch,), 30, dtype=torch.int32)
    lens[1::3] = 0
    lens[batch - 3], lens[batch - 1] = 1537, 8192
    out = torch.full_like(q, float("nan"), device="cuda")
    hq.hq_cache_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda(), out=out)
    torch.cuda.synchronize()
    ref, tol = R.attend(q.numpy(), R.values(kc), R.values(vc), table.numpy(), lens.numpy(), BT, N ** -0.5, heads, group)
    got = out.cpu().numpy()
    assert not np.isnan(got).any(), np.unique(np.nonzero(np.isnan(got))[0])
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max())


def test_long_sequences_wander_through_a_replayed_batch(hq):
    batch, heads, group = 64, 16, 1
    kp, vp, kc, vc, table, q = case(hq, "int8", batch, heads, group, 5)
    table, q = table.cuda(), q.cuda()
    base = torch.full((batch,), 20, dtype=torch.int32)
    base[0], base[5] = 4000, 1100
    lens, out = base.cuda(), torch.empty_like(q)
    ws = torch.empty(hq.hq_cache_attention_workspace_bytes(kc, batch, heads * group, table.shape[1]), dtype=torch.uint8,
                     device="cuda")
    call = lambda o: hq.hq_cache_attention(kp, kc, vp, vc, q, table, lens, out=o, workspace=ws)
    call(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for shift in (0, 30, 33, 47, 58, 63):
        lens.copy_(base.roll(shift))
        out.fill_(float("nan"))
        graph.replay()
        got = out.clone()
        eager = call(torch.full_like(out, float("nan")))
        torch.cuda.synchronize()
        assert torch.isfinite(got).all() and torch.equal(got, eager)


@pytest.mark.parametrize("heads", [256, 512, 600])
def test_as_many_heads_as_workgroups(hq, heads):
    """From 512 KV heads on no sequence is split, however long the table."""
    lens = torch.tensor([1100, 0, 1500, 3], dtype=torch.int32)
    kp, vp, kc, vc, table, q = case(hq, "int8", len(lens), heads, 1, heads)
    out = torch.full_like(q, float("nan"), device="cuda")
    hq.hq_cache_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda(), out=out)
    torch.cuda.synchronize()
    ref, tol = R.attend(q.numpy(), R.values(kc), R.values(vc), table.numpy(), lens.numpy(), BT, N ** -0.5, heads, 1)
    assert (np.abs(out.cpu().numpy() - ref) <= tol).all()  # a NaN is not
