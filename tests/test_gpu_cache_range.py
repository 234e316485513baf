"""The fixed-rate cache at both ends of fp32's range, against tests/cache64.py: whatever is written without
a report reads back finite."""
import numpy as np
import pytest
import torch

from tests import cache64 as R

pytestmark = pytest.mark.gpu
N = R.N
TINY = 2.0 ** -149  # fp32's smallest


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def check_read(hq, plan, c, slots):
    """Every stage rounds by at most U of the sum of magnitudes (or of fp32's smallest number)."""
    at = slots.numpy()
    ref = R.rows_of(c, R.SEED_K, at)
    mag = np.repeat(np.abs(R.values(c)[at // c.block_tokens, :, at % c.block_tokens]).sum(-1), N, -1) / N
    out = hq.hq_cache_read(plan, c, slots.cuda(), out_dtype=torch.float32)
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    assert np.abs(ref).max() < 3.4e38 and np.isfinite(got).all(), int((~np.isfinite(got)).sum())
    assert (np.abs(got - ref) <= 9 * R.U * mag + TINY).all()
    assert torch.equal(hq.hq_cache_read(plan, c, slots.cuda()), out.to(torch.bfloat16))


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "mxfp4"])
def test_vectors_near_the_largest_that_can_be_written(hq, fmt):
    heads, bt, rows = 4, 16, 32
    plan, _ = R.plans(hq, heads)
    g = torch.Generator().manual_seed(3)
    x = torch.where(torch.rand((rows, heads * N), generator=g) < 0.5, -1.0, 1.0)
    x *= torch.logspace(32, 36.7, rows)[:, None]  # 5e36 at the end
    x[5, :N] = torch.from_numpy(R.signs(R.SEED_K, N)) * 2.5e36  # all of it in one value of y
    y, err = R.transform(x.numpy(), R.SEED_K, heads)
    assert 2.9e38 < np.abs(y).max() < 3.3e38
    c = hq.Cache(plan, rows // bt, bt, {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt], heads=heads)
    slots = torch.arange(rows).flip(0)
    hq.hq_cache_write(plan, x.cuda(), c, None, None, None, slots.cuda())
    torch.cuda.synchronize()
    assert c.read_stats()["status"] == 0 and c.read_stats()["overflow_tiles"] == 0
    at = slots.numpy()
    R.check_codes(fmt, y, err, R.values(c)[at // bt, :, at % bt])
    check_read(hq, plan, c, slots)


@pytest.mark.parametrize("low", [0, 5, 100, 240, 249])
def test_mxfp4_scales_of_the_whole_range(hq, low):
    """Bytes 0 .. 252 (a larger one stands for values past fp32); those of a vector differ by up to 3."""
    heads, bt = 4, 32
    plan, _ = R.plans(hq, heads)
    c = R.random_cache(hq, plan, "mxfp4", 2, heads, bt, 30 + low)
    g = torch.Generator().manual_seed(low)
    c.scales.copy_(torch.randint(low, low + 4, c.scales.shape, generator=g, dtype=torch.uint8))
    check_read(hq, plan, c, torch.randperm(2 * bt, generator=g))


def attend_over(hq, fmt, k, v, q, scale):
    """One sequence of all rows; the 64-bit form of what the caches hold."""
    heads, bt, T = 4, 16, k.shape[0]
    kp, vp = R.plans(hq, heads)
    form = {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]
    kc, vc = (hq.Cache(p, -(-T // bt), bt, form, heads=heads) for p in (kp, vp))
    hq.hq_cache_write(kp, k.cuda(), kc, vp, v.cuda(), vc, torch.arange(T, device="cuda"))
    table = torch.arange(kc.blocks, dtype=torch.int32).view(1, -1)
    lens = torch.tensor([T], dtype=torch.int32)
    out = hq.hq_cache_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda(), scale=scale)
    torch.cuda.synchronize()
    assert kc.read_stats()["status"] == 0 and vc.read_stats()["status"] == 0
    ref, tol = R.attend(q.numpy(), R.values(kc), R.values(vc), table.numpy(), lens.numpy(), bt, scale, heads,
                        q.shape[1] // heads)
    return out.cpu().numpy().astype(np.float64), ref, tol


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "mxfp4"])
@pytest.mark.parametrize("tokens", [1, 100, 1500])
@pytest.mark.parametrize("size", [2.1e36, 2.55e36])
def test_attention_over_values_at_the_stated_bound(hq, fmt, tokens, size):
    """tokens * |v| just below 2.6e36, every vector with all of it in one coordinate of y, the weights
    nearly alike: the largest sums that the bound allows.  The bound is of what the cache holds:
    2.55e36 / 1500 is 5.24 steps of MXFP4's block and stored as 6, so 1500 of them are 2.92e36, past it."""
    g = torch.Generator().manual_seed(tokens)
    k = 0.01 * torch.randn((tokens, 4 * N), generator=g)
    v = torch.from_numpy(R.signs(R.SEED_V, 4 * N)).float().repeat(tokens, 1) * (size / tokens)
    got, ref, tol = attend_over(hq, fmt, k, v, torch.randn((1, 8, N), generator=g), N ** -0.5)
    if tokens * np.abs(ref).max() < 2.6e36:  # the rows are alike, and so is their mean
        assert (np.abs(got - ref) <= tol).all() and np.abs(ref).min() > 1.5e36 / tokens
    else:
        assert (fmt, tokens, size) == ("mxfp4", 1500, 2.55e36) and tokens * np.abs(ref).max() > 2.9e36


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "mxfp4"])
def test_attention_of_queries_at_the_stated_bound(hq, fmt):
    g = torch.Generator().manual_seed(4)
    k, v = 1e-2 * torch.randn((70, 4 * N), generator=g), torch.randn((70, 4 * N), generator=g)
    q = torch.from_numpy(R.signs(R.SEED_K, 4 * N)).float().view(1, 4, N).repeat_interleave(2, 1) * 2.55e36
    q[:, 1::2] *= torch.where(torch.rand((1, 4, N), generator=g) < 0.5, -1.0, 1.0)
    got, ref, tol = attend_over(hq, fmt, k, v, q, 3e-35)
    assert (np.abs(got - ref) <= tol).all() and np.ptp(ref) > 0.1
