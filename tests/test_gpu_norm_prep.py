"""hq_rmsnorm_act_prep and its fp8 form against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import cache64 as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def make(rows, cols, seed, wdt=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    x[:, 7::101] *= 30
    return (x.to(torch.bfloat16), torch.randn((rows, cols), generator=g).to(torch.bfloat16),
            (1 + 0.2 * torch.randn(cols, generator=g)).to(wdt))


def prep(hq, fp8):
    return hq.hq_rmsnorm_act_prep_fp8 if fp8 else hq.hq_rmsnorm_act_prep


def check(h, w, seed, tile, eps, xq, sx, fp8):
    """Codes against y rms (they do not depend on the rms), scales against 64 bits."""
    h, w = h.double().numpy(), w.double().numpy()
    rows, cols = h.shape
    hw = (h * w * R.signs(seed, cols)).reshape(rows, -1, tile)
    y = (hw @ R.hadamard(tile)).reshape(rows, cols)
    # log2(tile) stages and the product's rounding
    err = ((np.log2(tile) + 1) * R.U * np.abs(hw).sum(-1)).max(-1, keepdims=True)
    top = 448.0 if fp8 else 127.0
    amax = np.abs(y).max(-1, keepdims=True)
    c = R.e4m3_values(xq.cpu().numpy()) if fp8 else xq.cpu().numpy().astype(np.float64)
    step = amax / top
    half = np.maximum(np.abs(y) * 2.0 ** -4, step * 2.0 ** -10) if fp8 else step / 2
    assert (np.abs(c * step - y) <= half * (1 + 8 * R.U) + 2 * err + 8 * R.U * amax).all()
    rms = np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    # the sum of squares: a lane's chain of up to 64, six steps in the wave, three across; the mean, the
    # root and two divisions round once each
    rel = (64 + 6 + 3 + 8) * R.U + (err / np.maximum(amax, 1e-300))
    want = amax / top / rms
    got = sx.cpu().double().numpy()[:, None]
    assert (np.abs(got - want) <= rel * want).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,cols,tile", [(1, 512, 128), (3, 1024, 128), (17, 2048, 256), (5, 2560, 512),
                                            (33, 4096, 128), (4, 4608, 128), (9, 8192, 512), (2, 8704, 128),
                                            (6, 14336, 128), (3, 16384, 256), (2, 1024, 1024), (4, 3584 * 2, 1024),
                                            (3, 2048, 2048), (2, 14336, 2048), (5, 9216, 1024), (2, 16384, 2048)])
def test_parity(hq, fp8, rows, cols, tile):
    print(f"[norm] fp8={fp8} {rows} x {cols} tile {tile}", flush=True)
    plan = hq.hq_plan(tile=tile, cols=cols, bps=4.0, rht_seed=9)
    for wdt, eps in ((torch.bfloat16, 1e-5), (torch.float32, 1e-2)):
        x, r, w = make(rows, cols, rows + cols, wdt)
        xq, sx, h = prep(hq, fp8)(plan, x.cuda(), w.cuda(), eps=eps, residual=r.cuda())
        want_h = (x.float() + r.float()).to(torch.bfloat16)
        assert torch.equal(h.cpu(), want_h)
        check(want_h, w, 9, tile, eps, xq, sx, fp8)
        xq, sx = prep(hq, fp8)(plan, x.cuda(), w.cuda(), eps=eps)
        check(x, w, 9, tile, eps, xq, sx, fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tile", [128, 512])
def test_codes_are_those_of_the_activation_prep(hq, fp8, tile):
    """With a weight of ones the codes are hq_act_prep's of the row itself, bit for bit."""
    plan = hq.hq_plan(tile=tile, cols=4096, bps=4.0, rht_seed=5)
    x, _, _ = make(20, 4096, 3)
    xq, sx = prep(hq, fp8)(plan, x.cuda(), torch.ones(4096, device="cuda"), eps=1e-6)
    ref, rs = (hq.hq_act_prep_fp8 if fp8 else hq.hq_act_prep)(plan, x.cuda())
    a, b = xq.cpu(), ref.cpu()
    if fp8:
        a, b = R.e4m3_values(a.numpy()), R.e4m3_values(b.numpy())
        assert np.array_equal(a, b)
    else:
        assert torch.equal(a, b)
    rms = (x.double().square().mean(-1) + 1e-6).sqrt()
    assert torch.allclose(sx.cpu().double() * rms, rs.cpu().double(), rtol=81 * R.U, atol=0)


def test_strides_and_the_residual_in_place(hq):
    plan = hq.hq_plan(cols=1024, bps=4.0, rht_seed=5)
    x, r, w = make(7, 1024, 4)
    ref = hq.hq_rmsnorm_act_prep(plan, x.cuda(), w.cuda(), residual=r.cuda())
    wide_x, wide_r = (torch.full((7, 1024 + 8), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wide_x[:, :1024], wide_r[:, :1024] = x.cuda(), r.cuda()
    for into in (wide_r, wide_x):
        keep = into.clone()
        xq, sx, h = hq.hq_rmsnorm_act_prep(plan, wide_x[:, :1024], w.cuda(), residual=wide_r[:, :1024],
                                           h=into[:, :1024])
        assert torch.equal(xq, ref[0]) and torch.equal(sx, ref[1]) and torch.equal(h, ref[2])
        assert into[:, 1024:].isnan().all()
        into.copy_(keep)


@pytest.mark.parametrize("fp8", [False, True])
def test_zero_rows_and_rows_that_are_not_finite(hq, fp8):
    plan = hq.hq_plan(cols=2048, bps=4.0, rht_seed=5)
    x, _, w = make(6, 2048, 8)
    x[0] = 0
    x[1, 77] = float("nan")
    x[2, 5] = float("inf")
    x[3] = x[3] * 1e-20
    xq, sx = prep(hq, fp8)(plan, x.cuda(), w.cuda())
    zero = R.e4m3_values(xq[0].cpu().numpy()) if fp8 else xq[0].cpu().numpy()  # E4M3 zeros have either sign
    assert not zero.any() and float(sx[0]) == 0.0
    assert sx[1].isnan() and sx[2].isnan() and torch.isfinite(sx[3:]).all()
    check(x[3:], w, 5, 128, 1e-5, xq[3:], sx[3:], fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tile", [128, 2048])
def test_weights_that_are_not_finite_reach_the_scale(hq, tile, fp8):
    plan = hq.hq_plan(tile=tile, cols=4096, bps=4.0, rht_seed=5)
    x, _, w = make(5, 4096, 12, torch.float32)
    ref = prep(hq, fp8)(plan, x.cuda(), w.cuda())
    assert torch.isfinite(ref[1]).all()
    for value in (float("nan"), float("inf"), float("-inf")):
        bad = w.clone()
        bad[4000] = value
        assert prep(hq, fp8)(plan, x.cuda(), bad.cuda())[1].isnan().all()
    big, bad = x.clone(), w.clone()
    big[:, 3], big[2, 3], bad[3] = 0, 1e18, 1e30  # one product past fp32, the squares' sum not
    xq, sx = prep(hq, fp8)(plan, big.cuda(), bad.cuda())
    assert sx[2].isnan() and torch.isfinite(sx[[0, 1, 3, 4]]).all()
    check(big[[0, 1, 3, 4]], bad, 5, tile, 1e-5, xq[[0, 1, 3, 4]], sx[[0, 1, 3, 4]], fp8)


def test_more_rows_than_a_grid_of_threads(hq):
    """2^32 threads at four waves a row: the rows behind are the same rows again."""
    plan = hq.hq_plan(cols=512, bps=4.0)
    rows, period = (1 << 24) + 3, 1 << 10
    x, _, w = make(period, 512, 21)
    x, w = x.cuda(), w.cuda()
    xq, sx = hq.hq_rmsnorm_act_prep(plan, x.repeat((rows + period - 1) // period, 1)[:rows], w)
    ref = hq.hq_rmsnorm_act_prep(plan, x, w)
    for at in (0, (1 << 21) - period, 1 << 21, (1 << 23) + period, (1 << 24) - period):
        assert torch.equal(xq[at:at + period], ref[0]) and torch.equal(sx[at:at + period], ref[1])
    assert torch.equal(xq[1 << 24:], ref[0][:3]) and torch.equal(sx[1 << 24:], ref[1][:3])


def test_graph_replays(hq):
    plan = hq.hq_plan(cols=1024, bps=4.0)
    x, r, w = (t.cuda() for t in make(5, 1024, 9))
    args = dict(residual=r, h=torch.empty_like(x), xq=torch.empty((5, 1024), dtype=torch.int8, device="cuda"),
                sx=torch.empty(5, device="cuda"))
    hq.hq_rmsnorm_act_prep(plan, x, w, **args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hq.hq_rmsnorm_act_prep(plan, x, w, **args)
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        got = [args[n].clone() for n in ("xq", "sx", "h")]
        want = hq.hq_rmsnorm_act_prep(plan, x, w, residual=r)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(hq):
    plan = hq.hq_plan(cols=1024, bps=4.0)
    L = hq.lib()
    x, r, w = (t.cuda() for t in make(4, 1024, 9))
    xq, sx = torch.empty((4, 1024), dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")

    def call(xp=x.data_ptr(), ldx=1024, rp=r.data_ptr(), ldr=1024, wp=w.data_ptr(), wt=0, eps=1e-5, M=4, h=None, ldh=0,
             q=xq.data_ptr(), s=sx.data_ptr(), pl=plan, fn=L.hq_rmsnorm_act_prep):
        return fn(pl.handle if pl else None, xp, ldx, rp, ldr, wp, wt, eps, M, h, ldh, q, s, None)

    for fn in (L.hq_rmsnorm_act_prep, L.hq_rmsnorm_act_prep_fp8):
        assert call(fn=fn) == 0 and call(fn=fn, rp=None, ldr=0) == 0 and call(fn=fn, M=0, xp=None, q=None) == 0
        assert call(fn=fn, pl=None) == -1 and call(fn=fn, M=-1) == -1 and call(fn=fn, wt=2) == -1
        assert call(fn=fn, eps=0.0) == -1 and call(fn=fn, eps=float("nan")) == -1 and call(fn=fn, eps=float("inf")) == -1
        assert call(fn=fn, xp=None) == -1 and call(fn=fn, xp=x.data_ptr() + 2) == -1 and call(fn=fn, ldx=1020) == -1
        assert call(fn=fn, ldx=1025) == -1 and call(fn=fn, ldr=512) == -1 and call(fn=fn, rp=r.data_ptr() + 8) == -1
        assert call(fn=fn, wp=None) == -1 and call(fn=fn, wp=w.data_ptr() + 2) == -1
        assert call(fn=fn, h=x.data_ptr(), ldh=1000) == -1 and call(fn=fn, q=xq.data_ptr() + 4) == -1
        assert call(fn=fn, s=None) == -1
    wide = hq.hq_plan(cols=16896, bps=4.0)
    assert call(pl=wide, ldx=16896) == -2
    with pytest.raises(ValueError):
        hq.hq_rmsnorm_act_prep(plan, x.float(), w)
    with pytest.raises(ValueError):
        hq.hq_rmsnorm_act_prep(plan, x, w[:512])
    with pytest.raises(ValueError):
        hq.hq_rmsnorm_act_prep(plan, x, w.cpu())
    with pytest.raises(ValueError):
        hq.hq_rmsnorm_act_prep(plan, x, w, xq=xq[:2])
    torch.cuda.synchronize()
