"""Rotary positions on the GPU (hq_rope_table, hq_rope) and the cache's append
(hq_cache_append) against their definitions in 64 bits (tests/rows64.py, tests/cache64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W

pytestmark = pytest.mark.gpu
FMTS = ["int8", "e4m3", "mxfp4"]
N = R.N
INVALID_ARG = -1 & 0xFFFFFFFF
BF16_HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def fmt_id(hq, fmt):
    return {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]


def freqs(pairs, base=10000.0):
    return torch.from_numpy(base ** (-np.arange(pairs) / pairs)).cuda()


def axis_of(pairs, axes, mixed):
    """Sections in order, or axes in turn from pair to pair."""
    return [i % axes if mixed else i * axes // pairs for i in range(pairs)]


def case(hq, rows, heads, dims, interleaved, axes, mixed, seed, count=1000):
    rng = np.random.default_rng(seed)
    table = hq.hq_rope_table(freqs(dims // 2), count)
    axis = axis_of(dims // 2, axes, mixed)
    rope = hq.Rope(table, interleaved=interleaved, axis=axis)
    pos = rng.integers(0, count, (rows, axes)).astype(np.int32)
    pos[0], pos[-1] = 0, count - 1
    return rope, table.cpu().numpy(), np.array(axis), pos, rng.standard_normal((rows, heads * N)).astype(np.float32)


@pytest.mark.parametrize("pairs,count,factor", [(64, 300, 1.0), (1, 7, 1.0), (5, 1000, 1.25), (48, 1, 1.0), (64, 70000, 1.0)])
def test_table(hq, pairs, count, factor):
    f = freqs(pairs)
    got = hq.hq_rope_table(f, count, factor).cpu().numpy().astype(np.float64)
    angle = np.arange(count)[:, None] * f.cpu().numpy()
    ref = factor * np.stack((np.cos(angle), np.sin(angle)), 1)
    # rounded once; the 64-bit functions differ by an ulp or two of theirs
    assert (np.abs(got - ref) <= R.U * np.abs(ref) + 1e-14).all()


def test_table_far_positions(hq):
    """Angles of far positions keep their low bits."""
    f = torch.tensor([1.0, 0.7], dtype=torch.float64, device="cuda")
    count = 1 << 24
    got = hq.hq_rope_table(f, count)[-3:].cpu().numpy().astype(np.float64)
    angle = np.arange(count - 3, count)[:, None] * f.cpu().numpy()
    assert np.abs(got - np.stack((np.cos(angle), np.sin(angle)), 1)).max() <= R.U + 1e-8 * 2 ** -3


@pytest.mark.parametrize("rows,heads", [(1, 1), (3, 2), (17, 3), (33, 8), (130, 5), (7, 32)])
@pytest.mark.parametrize("dims,interleaved,axes,mixed", [(128, False, 1, False), (128, True, 1, False), (64, False, 2, False),
                                                         (64, True, 3, False), (96, False, 3, True), (96, True, 4, True),
                                                         (16, False, 1, False), (16, True, 2, True), (112, False, 4, False),
                                                         (48, True, 1, False), (128, False, 3, True)])
@pytest.mark.parametrize("transposed", [False, True])
def test_rope(hq, rows, heads, dims, interleaved, axes, mixed, transposed):
    print(f"[rope] {rows} x {heads} dims={dims} il={interleaved} axes={axes} {mixed} {transposed}", flush=True)
    rope, table, axis, pos, x = case(hq, rows, heads, dims, interleaved, axes, mixed, rows + heads)
    p = torch.from_numpy(pos).cuda()
    ref, tol, _ = W.turn(x.reshape(rows, heads, N), table, pos, axis, interleaved, transposed)
    ref, tol = ref.reshape(rows, -1), tol.reshape(rows, -1)
    got = hq.hq_rope(rope, torch.from_numpy(x).cuda(), p, transposed=transposed)
    assert (np.abs(got.cpu().numpy() - ref) <= tol).all()
    out16 = hq.hq_rope(rope, torch.from_numpy(x).cuda(), p, transposed=transposed, out_dtype=torch.bfloat16)
    assert torch.equal(out16, got.to(torch.bfloat16))
    x16 = torch.from_numpy(x).to(torch.bfloat16)
    ref, tol, _ = W.turn(x16.float().numpy().reshape(rows, heads, N), table, pos, axis, interleaved, transposed)
    got = hq.hq_rope(rope, x16.cuda(), p, transposed=transposed).float().cpu().numpy().reshape(ref.shape)
    assert (np.abs(got - ref) <= tol + BF16_HALF * (np.abs(ref) + tol)).all()
    assert rope.read_stats()["status"] == 0


def test_rope_strides_and_in_place(hq):
    """A projection's queries among its keys and values, turned into another array and in place."""
    rows, heads = 50, 6
    rope, table, axis, pos, x = case(hq, rows, heads, 128, False, 1, False, 3)
    wide = torch.randn((rows, 2 * heads * N + 64), generator=torch.Generator().manual_seed(1)).cuda()
    wide[:, 64:64 + heads * N] = torch.from_numpy(x)
    before, p = wide.clone(), torch.from_numpy(pos).cuda()
    q = wide[:, 64:64 + heads * N]
    out = torch.full((rows, heads * N + 16), 7.0, device="cuda")
    hq.hq_rope(rope, q, p, out=out[:, 8:8 + heads * N])
    assert torch.equal(wide, before) and (out[:, :8] == 7).all() and (out[:, 8 + heads * N:] == 7).all()
    hq.hq_rope(rope, q, p[:, 0], out=q)
    assert torch.equal(q, out[:, 8:8 + heads * N])
    assert torch.equal(wide[:, :64], before[:, :64]) and torch.equal(wide[:, 64 + heads * N:], before[:, 64 + heads * N:])


def test_rope_padding_and_positions_out_of_range(hq):
    rows, heads = 40, 3
    rope, table, axis, pos, x = case(hq, rows, heads, 64, False, 3, True, 4)
    x[5], x[6] = np.nan, np.inf  # rows that are not looked at
    pos[5], pos[6, 0] = -1, -2 ** 31
    out = torch.full((rows, heads * N), 7.0, device="cuda")
    hq.hq_rope(rope, torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda(), out=out)
    assert rope.read_stats()["status"] == 0 and (out[5:7] == 7).all()
    pos[9, 0], pos[10, 2], pos[11, 1] = 1000, 2 ** 31 - 1, -1
    out.fill_(7.0)
    hq.hq_rope(rope, torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda(), out=out)
    assert rope.read_stats()["status"] == INVALID_ARG
    ref, tol, ok = W.turn(x.reshape(rows, heads, N), table, pos, axis, False)
    assert ok.sum() == rows - 5
    got = out.cpu().numpy().reshape(ref.shape)
    assert (got[~ok] == 7).all() and (np.abs(got - ref) <= tol)[ok].all()
    fresh = hq.hq_rope(rope, torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda())
    assert not fresh.cpu().numpy().reshape(ref.shape)[~ok].any()


def test_rope_values_that_do_not_turn_keep_infinities_and_nan(hq):
    rope, table, axis, pos, x = case(hq, 6, 2, 32, False, 1, False, 5)
    x[2, 40], x[3, 127], x[4, 3] = np.nan, np.inf, np.inf
    got = hq.hq_rope(rope, torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda()).cpu().numpy()
    same = np.ones(N, dtype=bool)
    same[:32] = False
    same = np.tile(same, 2)
    assert np.array_equal(got[:, same], x[:, same], equal_nan=True)
    turned = ~np.isfinite(got[:, ~same])
    assert turned[4, 3] and turned[4, 19] and turned.sum() <= 2


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient(hq, interleaved):
    """The transposed call is the gradient: against the formula's and against differences."""
    rows, heads = 9, 2
    rope, table, axis, pos, x = case(hq, rows, heads, 96, interleaved, 2, False, 6)
    p = torch.from_numpy(pos).cuda()
    rng = np.random.default_rng(7)
    g = rng.standard_normal(x.shape).astype(np.float32)
    dx = hq.hq_rope(rope, torch.from_numpy(g).cuda(), p, transposed=True).cpu().numpy().astype(np.float64)
    # d/dx sum(g * rope(x)) per value, by the rotation's own matrix
    eye_tol = 4 * R.U * np.abs(g).sum(1, keepdims=True)
    for col in (0, 1, 31, 47, 48, 95, 96, 127, 128 + 5):
        e = np.zeros_like(x)
        e[:, col] = 1.0
        up = hq.hq_rope(rope, torch.from_numpy(x + 0.5 * e).cuda(), p).cpu().numpy().astype(np.float64)
        down = hq.hq_rope(rope, torch.from_numpy(x - 0.5 * e).cuda(), p).cpu().numpy().astype(np.float64)
        exact, tol, _ = W.turn(e.reshape(rows, heads, N), table, pos, axis, interleaved)
        assert (np.abs((g * exact.reshape(rows, -1)).sum(1) - dx[:, col]) <= eye_tol[:, 0]).all()
        # x + e / 2 and the turned values round: 8 U of the values' size
        room = 8 * R.U * (np.abs(g) * (np.abs(up) + np.abs(down) + 2)).sum(1) + 4 * R.U * np.abs(x).max() * np.abs(g).sum(1)
        assert (np.abs((g * (up - down)).sum(1) - dx[:, col]) <= room).all()
    back = hq.hq_rope(rope, hq.hq_rope(rope, torch.from_numpy(x).cuda(), p), p, transposed=True).cpu().numpy()
    assert np.abs(back - x).max() <= 16 * R.U * np.abs(x).max()


def test_rope_rows_past_32_bit_offsets(hq):
    rope, table, axis, pos, x = case(hq, 5, 2, 128, False, 1, False, 8)
    ld = (1 << 29) + 8
    big = torch.empty(4 * ld + 2 * N, dtype=torch.bfloat16, device="cuda")
    rows = big.as_strided((5, 2 * N), (ld, 1))
    rows.copy_(torch.from_numpy(x))
    want = hq.hq_rope(rope, rows.contiguous(), torch.from_numpy(pos).cuda())
    hq.hq_rope(rope, rows, torch.from_numpy(pos).cuda(), out=rows)
    assert torch.equal(rows, want)


# ------------------------------------------------------------------ append

def append_case(hq, fmt, rows, heads, group, dims, interleaved, axes, dtype, bt, seed):
    rope, table, axis, pos, _ = case(hq, rows, heads, dims, interleaved, axes, False, seed)
    kp, vp = R.plans(hq, heads)
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn((rows, (group + 2) * heads * N), generator=g)
    wide[:, group * heads * N + 3:(group + 1) * heads * N:N] *= 10
    wide = wide.to(dtype)
    blocks = -(-rows // bt) + 2
    slots = torch.randperm(blocks * bt, generator=g)[:rows]
    if rows > 2:
        slots[1] = -1
    return rope, table, axis, pos, kp, vp, wide, blocks, slots


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,heads,group,dims,interleaved,axes,dtype,bt", [
    (1, 1, 1, 128, False, 1, torch.bfloat16, 16), (17, 2, 4, 128, True, 1, torch.float32, 16),
    (33, 3, 0, 96, False, 3, torch.bfloat16, 48), (129, 4, 2, 64, True, 2, torch.bfloat16, 128),
    (300, 8, 4, 128, False, 1, torch.float32, 64), (5, 16, 1, 32, False, 4, torch.bfloat16, 32),
    (66, 5, 3, 128, False, 3, torch.bfloat16, 80)])
def test_append(hq, fmt, rows, heads, group, dims, interleaved, axes, dtype, bt):
    print(f"[rope] append {fmt} {rows} x {heads} x {group} dims={dims}", flush=True)
    rope, table, axis, pos, kp, vp, wide, blocks, slots = append_case(hq, fmt, rows, heads, group, dims, interleaved, axes,
                                                                      dtype, bt, rows)
    if rows > 8:
        pos[4] = -1                      # a row of padding with a slot
        pos[7, axes - 1] = 5000          # one with a position that the table lacks
    p = torch.from_numpy(pos).cuda()
    kc, vc = R.random_cache(hq, kp, fmt, blocks, heads, bt, 1), R.random_cache(hq, vp, fmt, blocks, heads, bt, 2)
    before = [(c.codes.clone(), c.scales.clone()) for c in (kc, vc)]
    w = wide.cuda()
    q, k, v = w.split([group * heads * N, heads * N, heads * N], 1)
    out = torch.full((rows, group * heads * N), 7.0, dtype=dtype, device="cuda") if group else None
    got = hq.hq_cache_append(kp, k, kc, vp, v, vc, slots.cuda(), rope, p, q=q if group else None, q_out=out)
    assert got is out
    _, _, ok = W.turn(np.zeros((rows, heads, N)), table, pos, axis, interleaved)
    assert rope.read_stats()["status"] == (INVALID_ARG if rows > 8 else 0)
    # the same bits as the rotation in fp32 followed by the write
    turned = hq.hq_rope(rope, k, p, out_dtype=torch.float32)
    k2, v2 = (R.random_cache(hq, pl, fmt, blocks, heads, bt, i) for i, pl in ((1, kp), (2, vp)))
    left = torch.where(torch.from_numpy(ok), slots, torch.full_like(slots, -1)).cuda()
    hq.hq_cache_write(kp, turned, k2, vp, v.float(), v2, left)
    for a, b in ((kc, k2), (vc, v2)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    if group:
        want = torch.full_like(out, 7.0)
        hq.hq_rope(rope, q, p, out=want)
        assert torch.equal(out, want)
    # and the definition
    live = (slots.numpy() >= 0) & ok
    at = slots.numpy()[live]
    for x, c, seed, rotate in ((k, kc, R.SEED_K, True), (v, vc, R.SEED_V, False)):
        x = x.float().cpu().numpy().reshape(rows, heads, N)
        y, tol, _ = W.turn(x, table, pos, axis, interleaved) if rotate else (x.astype(np.float64), np.zeros(x.shape), ok)
        z, err = R.transform(y[live].reshape(len(at), -1), seed, heads)
        R.check_codes(fmt, z, err + tol[live].sum(-1, keepdims=True), R.values(c)[at // bt, :, at % bt])
    # every other slot is as it was
    keep = torch.ones(blocks * bt, dtype=torch.bool)
    keep[torch.from_numpy(at)] = False
    keep = keep.view(blocks, bt).cuda()
    for c, old in zip((kc, vc), before):
        assert torch.equal(c.codes.transpose(1, 2)[keep], old[0].transpose(1, 2)[keep])
        assert torch.equal(c.scales.transpose(1, 2)[keep], old[1].transpose(1, 2)[keep])


@pytest.mark.parametrize("fmt", FMTS)
def test_append_keys_alone_and_queries_in_place(hq, fmt):
    rope, table, axis, pos, kp, _, wide, blocks, slots = append_case(hq, fmt, 20, 4, 2, 128, False, 1, torch.bfloat16, 16, 9)
    p, w = torch.from_numpy(pos).cuda(), wide.cuda()
    q, k, v = w.split([8 * N, 4 * N, 4 * N], 1)
    a, b = (hq.Cache(kp, blocks, 16, fmt_id(hq, fmt), heads=4) for _ in range(2))
    want = hq.hq_rope(rope, q, p)
    kept = w[:, 8 * N:].clone()
    hq.hq_cache_append(kp, k, a, None, None, None, slots.cuda(), rope, p, q=q, q_out=q)
    other = hq.Cache(kp, blocks, 16, fmt_id(hq, fmt), heads=4)
    hq.hq_cache_append(kp, k, b, kp, v, other, slots.cuda(), rope, p)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    assert torch.equal(q, want) and torch.equal(w[:, 8 * N:], kept)
    out32 = torch.empty((20, 8 * N), device="cuda")
    q.copy_(wide[:, :8 * N])
    hq.hq_cache_append(kp, k, a, None, None, None, slots.cuda(), rope, p, q=q, q_out=out32)
    assert torch.equal(out32, hq.hq_rope(rope, q, p, out_dtype=torch.float32))


@pytest.mark.parametrize("fmt", FMTS)
def test_append_values_that_are_not_finite_and_slots_past_the_cache(hq, fmt):
    rope, table, axis, pos, kp, vp, wide, blocks, slots = append_case(hq, fmt, 6, 4, 0, 64, False, 1, torch.float32, 16, 10)
    wide[2, 5], wide[3, 5 * N + 7] = float("inf"), float("nan")  # key head 0, value head 1
    slots = torch.tensor([0, 1, 2, 3, 16 * blocks, 2 ** 40])
    kc, vc = (hq.Cache(pl, blocks, 16, fmt_id(hq, fmt), heads=4) for pl in (kp, vp))
    k, v = wide.cuda().split([4 * N, 4 * N], 1)
    hq.hq_cache_append(kp, k, kc, vp, v, vc, slots.cuda(), rope, torch.from_numpy(pos).cuda())
    rk, rv = (hq.hq_cache_read(pl, c, torch.arange(4, device="cuda"), out_dtype=torch.float32).view(4, 4, N).isnan().cpu()
              for pl, c in ((kp, kc), (vp, vc)))
    assert rk[2, 0].all() and rk.sum() == N and rv[3, 1].all() and rv.sum() == N
    for c in (kc, vc):
        st = c.read_stats()
        assert st["overflow_tiles"] == 1 and st["status"] in (INVALID_ARG, -4 & 0xFFFFFFFF)
        assert int((R.values(c) != 0).any(-1).sum()) <= 16  # nothing outside the four slots


def test_append_captured_and_on_another_stream(hq):
    rope, table, axis, pos, kp, vp, wide, blocks, slots = append_case(hq, "int8", 64, 8, 4, 128, False, 1, torch.bfloat16, 64, 11)
    p, w, s = torch.from_numpy(pos).cuda(), wide.cuda(), slots.cuda()
    q, k, v = w.split([32 * N, 8 * N, 8 * N], 1)
    kc, vc, k2, v2 = (hq.Cache(pl, blocks, 64, hq.HQ_INT8, heads=8) for pl in (kp, vp, kp, vp))
    out, out2 = torch.zeros((64, 32 * N), dtype=torch.bfloat16, device="cuda"), torch.zeros((64, 32 * N), dtype=torch.bfloat16, device="cuda")
    hq.hq_cache_append(kp, k, kc, vp, v, vc, s, rope, p, q=q, q_out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hq.hq_cache_append(kp, k, kc, vp, v, vc, s, rope, p, q=q, q_out=out)
    side = torch.cuda.Stream()
    for i in range(3):
        w.copy_(wide.roll(i, 0))
        p.copy_(torch.from_numpy(pos).roll(i, 0))
        for t in (kc.codes, kc.scales, vc.codes, out, k2.codes, out2):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        hq.hq_cache_append(kp, k, k2, vp, v, v2, s, rope, p, q=q, q_out=out2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(kc.codes, k2.codes) and torch.equal(kc.scales, k2.scales) and torch.equal(vc.codes, v2.codes)
        assert torch.equal(out, out2) and out.any()
