"""The fixed-rate KV cache on the GPU (hq_cache_write, hq_cache_read,
hq_cache_attention) against its definition in 64 bits (tests/cache64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R

pytestmark = pytest.mark.gpu
FMTS = ["int8", "e4m3", "mxfp4"]
N = R.N
INVALID_ARG = -1 & 0xFFFFFFFF
OVERFLOW = -4 & 0xFFFFFFFF


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def fmt_id(hq, fmt):
    return {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]


def inputs(rows, heads, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    k = torch.randn((rows, heads * N), generator=g)
    k[:, 3::N] *= 10
    return k.to(dtype), torch.randn((rows, heads * N), generator=g).to(dtype)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,heads,bt,dtype", [(1, 1, 16, torch.bfloat16), (17, 2, 16, torch.float32),
                                                 (33, 3, 48, torch.bfloat16), (129, 4, 128, torch.bfloat16),
                                                 (300, 8, 64, torch.float32), (5, 16, 32, torch.bfloat16)])
def test_write_and_read(hq, fmt, rows, heads, bt, dtype):
    print(f"[cache] write {fmt} rows={rows} heads={heads} bt={bt} {dtype}", flush=True)
    kp, vp = R.plans(hq, heads)
    k, v = inputs(rows, heads, dtype, 7)
    k[rows // 2] = 0  # a zero vector
    blocks = -(-rows // bt) + 2
    kc, vc = R.random_cache(hq, kp, fmt, blocks, heads, bt, 1), R.random_cache(hq, vp, fmt, blocks, heads, bt, 2)
    before = [(c.codes.clone(), c.scales.clone()) for c in (kc, vc)]
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(blocks * bt, generator=g)[:rows]
    slots[0] = -1 if rows > 1 else slots[0]  # a padded row
    wide = torch.empty((rows, heads * N + 64), dtype=dtype, device="cuda")  # rows with a stride
    wide[:, :heads * N] = k.cuda()
    hq.hq_cache_write(kp, wide[:, :heads * N], kc, vp, v.cuda(), vc, slots.cuda())
    torch.cuda.synchronize()
    live = slots >= 0
    at = slots[live].numpy()
    for x, c, seed, old in ((k, kc, R.SEED_K, before[0]), (v, vc, R.SEED_V, before[1])):
        y, err = R.transform(x[live].float().numpy(), seed, heads)
        got = R.values(c)[at // bt, :, at % bt]
        R.check_codes(fmt, y, err, got)
        # every other slot is as it was
        keep = torch.ones(blocks * bt, dtype=torch.bool)
        keep[slots[live]] = False
        keep = keep.view(blocks, bt)
        for now, was in ((c.codes, old[0]), (c.scales, old[1])):
            assert torch.equal(now.transpose(1, 2)[keep.cuda()], was.transpose(1, 2)[keep.cuda()])
        # read back, in another order, with a padded and a repeated slot
        order = torch.cat((slots[live].flip(0), torch.tensor([-5]), slots[live][:1]))
        ref = np.zeros((len(order), heads * N))
        ok = order.numpy() >= 0
        ref[ok] = R.rows_of(c, seed, order[ok].numpy())
        mag = np.zeros_like(ref)
        mag[ok] = np.repeat(np.abs(R.values(c)[order[ok].numpy() // bt, :, order[ok].numpy() % bt]).sum(-1), N, -1) / N
        plan = kp if c is kc else vp
        out = hq.hq_cache_read(plan, c, order.cuda(), out_dtype=torch.float32).cpu().numpy()
        assert (np.abs(out - ref) <= 9 * R.U * mag).all()
        assert not out[~ok].any()
        out16 = hq.hq_cache_read(plan, c, order.cuda())
        assert out16.dtype == torch.bfloat16 and torch.equal(out16.cpu(), torch.from_numpy(out).to(torch.bfloat16))
        assert c.read_stats()["status"] == 0 and c.read_stats()["overflow_tiles"] == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_write_keys_alone(hq, fmt):
    kp, _ = R.plans(hq, 4)
    k, _ = inputs(9, 4, torch.bfloat16, 5)
    a, b = (hq.Cache(kp, 2, 16, fmt_id(hq, fmt)) for _ in range(2))
    other = hq.Cache(kp, 2, 16, fmt_id(hq, fmt))
    slots = torch.arange(9, device="cuda")
    hq.hq_cache_write(kp, k.cuda(), a, None, None, None, slots)
    hq.hq_cache_write(kp, k.cuda(), b, kp, k.cuda(), other, slots)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    assert torch.equal(a.codes, other.codes)


@pytest.mark.parametrize("fmt", FMTS)
def test_vectors_that_are_not_finite_or_tiny(hq, fmt):
    """An infinity or a NaN poisons its own head vector, and attention over it."""
    heads, bt = 4, 16
    kp, vp = R.plans(hq, heads)
    k, v = inputs(6, heads, torch.float32, 6)
    k[1, 5] = float("inf")
    k[2, N + 7] = float("nan")
    v[3, 2 * N + 1] = -float("inf")
    k[4, 3 * N:] = 1e-38  # too small for a scale
    kc, vc = hq.Cache(kp, 1, bt, fmt_id(hq, fmt)), hq.Cache(vp, 1, bt, fmt_id(hq, fmt))
    slots = torch.arange(6, device="cuda")
    hq.hq_cache_write(kp, k.cuda(), kc, vp, v.cuda(), vc, slots)
    rk = hq.hq_cache_read(kp, kc, slots, out_dtype=torch.float32).cpu().view(6, heads, N)
    rv = hq.hq_cache_read(vp, vc, slots, out_dtype=torch.float32).cpu().view(6, heads, N)
    bad = torch.zeros((6, heads), dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = True
    assert torch.equal(rk.isnan().all(-1), bad) and torch.equal(rk.isnan().any(-1), bad)
    assert rv[3, 2].isnan().all() and rv.isnan().sum() == N
    assert rk[4, 3].abs().max() <= 2e-37
    st = kc.read_stats()
    assert st["overflow_tiles"] == 2 and st["status"] == OVERFLOW
    assert vc.read_stats()["overflow_tiles"] == 1
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    q = torch.randn((1, heads * 2, N), generator=torch.Generator().manual_seed(1)).cuda()
    out = hq.hq_cache_attention(kp, kc, vp, vc, q, table, torch.tensor([6], dtype=torch.int32, device="cuda"))
    nan = out.cpu().view(heads, 2, N).isnan()
    assert nan[:3].all() and not nan[3].any()
    out = hq.hq_cache_attention(kp, kc, vp, vc, q, table, torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert not out.isnan().any()  # the poisoned tokens lie behind the sequence


def attention_case(hq, fmt, lens, heads, group, bt, seed=0, qdt=torch.float32, scale=N ** -0.5, extra=0, spare=1):
    kp, vp = R.plans(hq, heads)
    B = len(lens)
    nb = max(1, -(-max(lens) // bt)) + extra
    blocks = B * nb + spare
    kc, vc = R.random_cache(hq, kp, fmt, blocks, heads, bt, 10 + seed), R.random_cache(hq, vp, fmt, blocks, heads, bt, 20 + seed)
    g = torch.Generator().manual_seed(30 + seed)
    table = torch.randperm(blocks, generator=g)[:B * nb].view(B, nb).to(torch.int32)
    q = torch.randn((B, heads * group, N), generator=g).to(qdt)
    return kp, vp, kc, vc, table, q, torch.tensor(lens, dtype=torch.int32), scale


def run_attention(hq, case, **kw):
    kp, vp, kc, vc, table, q, lens, scale = case
    return hq.hq_cache_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda(), scale=scale, **kw)


def check_attention(hq, case, heads, group, bt, lens=None):
    kp, vp, kc, vc, table, q, ln, scale = case
    out = run_attention(hq, case)
    out16 = run_attention(hq, case, out_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    ref, tol = R.attend(q.float().numpy(), R.values(kc), R.values(vc), table.numpy(),
                        ln.numpy() if lens is None else lens, bt, scale, heads, group)
    got = out.cpu().numpy()
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max())
    # all outputs together: the worst case above allows what a lost term of a query or a
    # weight (2^-16) would show; errors that are independent roundings stay below 16 U a score
    # unit and 16 U of the sums
    size = np.linalg.norm(ref)
    assert np.linalg.norm(got - ref) <= 64 * R.U * max(1.0, float(np.abs(scale) * N ** 0.5)) * size + 1e-30
    assert torch.equal(out16.cpu(), out.cpu().to(torch.bfloat16))
    assert torch.equal(out, run_attention(hq, case))  # the same bits again
    return out


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bt", [16, 48, 128])
def test_attention_lengths(hq, fmt, bt):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511]
    print(f"[cache] attention lengths {fmt} bt={bt}", flush=True)
    case = attention_case(hq, fmt, lens, 4, 4, bt, extra=1)
    out = check_attention(hq, case, 4, 4, bt)
    assert not out[0].any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (2, 3), (3, 5), (4, 7), (4, 8), (8, 2), (16, 1), (1, 12)])
def test_attention_heads(hq, fmt, heads, group):
    print(f"[cache] attention heads {fmt} {heads} x {group}", flush=True)
    case = attention_case(hq, fmt, [301, 64, 130], heads, group, 32, seed=heads, qdt=torch.bfloat16)
    check_attention(hq, case, heads, group, 32)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("lens", [[1000], [2500, 3, 0, 700], [9000], [64] * 70, [5] * 600, [0] * 66 + [600, 1, 1300], [1000] * 9, [1024, 0, 513],
                                  [129 * (i % 7) for i in range(150)], [0, 0, 513]])
def test_attention_splits_and_joins(hq, fmt, lens):
    print(f"[cache] attention splits {fmt} {len(lens)} x {max(lens)}", flush=True)
    case = attention_case(hq, fmt, lens, 2, 4, 64, seed=3)
    check_attention(hq, case, 2, 4, 64)


def many_case(hq, fmt, B, heads, group, bt, seed):
    """B sequences over a small cache (blocks repeat), most of them short or empty, a few long."""
    kp, vp = R.plans(hq, heads)
    kc, vc = (R.random_cache(hq, p, fmt, 40, heads, bt, seed + i) for i, p in enumerate((kp, vp)))
    g = torch.Generator().manual_seed(seed + 2)
    lens = torch.randint(-40, 90, (B,), generator=g).clamp(min=0).to(torch.int32)
    lens[torch.randint(0, B, (5,), generator=g)] = torch.tensor([1023, 1024, 1025, 1536, 2000], dtype=torch.int32)
    table = torch.randint(0, 40, (B, -(-2000 // bt)), generator=g).to(torch.int32)
    q = torch.randn((B, heads * group, N), generator=g)
    return kp, vp, kc, vc, table, q, lens, N ** -0.5


@pytest.mark.parametrize("B,heads,group", [(64, 1, 2), (65, 1, 2), (129, 3, 5), (528, 1, 1), (529, 1, 1), (1024, 2, 1),
                                           (1025, 1, 4), (4097, 1, 1)])
def test_attention_many_sequences(hq, B, heads, group):
    print(f"[cache] attention many {B} x {heads} x {group}", flush=True)
    check_attention(hq, many_case(hq, "int8", B, heads, group, 48, B), heads, group, 48)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads,group", [(4, 2), (2, 6), (4, 8), (3, 9), (2, 16)])
def test_attention_enough_for_the_chip(hq, fmt, heads, group):
    """Every head layout with more workgroups than one CU in two has."""
    print(f"[cache] attention enough {fmt} {heads} x {group}", flush=True)
    check_attention(hq, many_case(hq, fmt, 71, heads, group, 32, group), heads, group, 32)
    short = list(many_case(hq, fmt, 71, heads, group, 32, group))
    short[4], short[6] = short[4][:, :32].contiguous(), short[6].clamp(max=1024)  # no sequence is split
    check_attention(hq, tuple(short), heads, group, 32)


def test_attention_many_sequences_replayed_and_out_of_range(hq):
    case = many_case(hq, "e4m3", 200, 2, 2, 64, 7)
    kp, vp, kc, vc, table, q, lens, scale = case
    cap = table.shape[1] * 64
    q, table, ln, out = q.cuda(), table.cuda(), lens.cuda(), torch.empty_like(q, device="cuda")
    ws = torch.empty(hq.hq_cache_attention_workspace_bytes(kc, 200, 4, table.shape[1]), dtype=torch.uint8, device="cuda")
    call = lambda o: hq.hq_cache_attention(kp, kc, vp, vc, q, table, ln, out=o, workspace=ws)
    call(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        ln.copy_(lens.roll(61 * i))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(torch.empty_like(out)))
    assert kc.read_stats()["status"] == 0
    ln[3], ln[150], ln[199] = -5, cap + 1, 2 ** 31 - 1
    graph.replay()
    assert kc.read_stats()["status"] == INVALID_ARG
    ln[3], ln[150], ln[199] = 0, cap, cap
    assert torch.equal(out, call(torch.empty_like(out)))


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0])
def test_attention_scales(hq, scale):
    case = attention_case(hq, "int8", [200, 33], 4, 2, 16, seed=5, scale=scale)
    check_attention(hq, case, 4, 2, 16)


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_ignores_what_lies_behind_a_sequence(hq, fmt):
    """Stale codes and scales of any bit pattern behind the last token, in blocks that no
    sequence has, and table entries behind the last block."""
    lens = [37, 5, 128, 0]
    case = attention_case(hq, fmt, lens, 4, 4, 64, seed=6, extra=2)
    kp, vp, kc, vc, table, q, ln, scale = case
    clean = run_attention(hq, case)
    live = torch.zeros((kc.blocks, 64), dtype=torch.bool)
    for b, n in enumerate(lens):
        t = torch.arange(n)
        live[table[b, t // 64].long(), t % 64] = True
        table[b, -(-n // 64):] = -7
    dead = (~live).cuda()
    for c in (kc, vc):
        c.codes.view(torch.uint8).transpose(1, 2)[dead] = 0x7F if fmt == "e4m3" else 0x80
        c.scales.transpose(1, 2)[dead] = float("nan") if fmt != "mxfp4" else 255
    assert torch.equal(clean, run_attention(hq, case))
    assert kc.read_stats()["status"] == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_bad_blocks_and_lengths(hq, fmt):
    case = attention_case(hq, fmt, [100, 70, 300, 40], 4, 2, 32, seed=8)
    kp, vp, kc, vc, table, q, ln, scale = case
    table[0, 1] = kc.blocks  # out of the cache: left out
    table[1, 0] = -1
    table[3, :] = 1 << 30    # nothing left
    out = check_attention(hq, case, 4, 2, 32)
    assert not out[3].any()
    assert kc.read_stats()["status"] == INVALID_ARG
    kc.reset_stats()
    cap = table.shape[1] * 32
    table[:] = torch.arange(4 * table.shape[1], dtype=torch.int32).view(4, -1)
    bad = (kp, vp, kc, vc, table, q, torch.tensor([-3, cap + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32), scale)
    out = check_attention(hq, bad, 4, 2, 32, lens=np.array([0, cap, cap, 0]))
    assert not out[0].any() and not out[3].any() and kc.read_stats()["status"] == INVALID_ARG


def test_slots_past_the_cache_are_skipped_and_reported(hq):
    kp, _ = R.plans(hq, 4)
    k, _ = inputs(4, 4, torch.bfloat16, 9)
    c = hq.Cache(kp, 2, 16, hq.HQ_INT8)
    slots = torch.tensor([0, 32, 2 ** 40, 31], device="cuda")
    hq.hq_cache_write(kp, k.cuda(), c, None, None, None, slots)
    assert c.read_stats()["status"] == INVALID_ARG
    assert int((c.scales != 0).sum()) == 2 * 4
    c.reset_stats()
    out = hq.hq_cache_read(kp, c, slots, out_dtype=torch.float32)
    assert c.read_stats()["status"] == INVALID_ARG
    assert not out[1:3].any() and out[0].any() and out[3].any()


@pytest.mark.parametrize("fmt", FMTS)
def test_caches_past_32_bit_offsets(hq, fmt):
    """Slots whose bytes lie past 4 GiB are written, read and attended to."""
    heads, bt = 8, 256
    kp, vp = R.plans(hq, heads)
    blocks = (5 << 30) // (heads * bt * (64 if fmt == "mxfp4" else 128))
    kc, vc = (hq.Cache(p, blocks, bt, fmt_id(hq, fmt), heads=heads) for p in (kp, vp))
    rows = 300
    k, v = inputs(rows, heads, torch.bfloat16, 11)
    table = torch.tensor([[blocks - 1, blocks // 2]], dtype=torch.int32)
    t = torch.arange(rows)
    slots = (table[0].long()[t // bt] * bt + t % bt).cuda()
    hq.hq_cache_write(kp, k.cuda(), kc, vp, v.cuda(), vc, slots)
    small_k, small_v = (hq.Cache(p, 2, bt, fmt_id(hq, fmt), heads=heads) for p in (kp, vp))
    hq.hq_cache_write(kp, k.cuda(), small_k, vp, v.cuda(), small_v, t.cuda())
    q = torch.randn((1, heads * 4, N), generator=torch.Generator().manual_seed(2)).cuda()
    ln = torch.tensor([rows], dtype=torch.int32, device="cuda")
    assert torch.equal(hq.hq_cache_read(kp, kc, slots), hq.hq_cache_read(kp, small_k, t.cuda()))
    far = hq.hq_cache_attention(kp, kc, vp, vc, q, table.cuda(), ln)
    near = hq.hq_cache_attention(kp, small_k, vp, small_v, q, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), ln)
    assert torch.equal(far, near) and far.any()


def test_workspace_of_the_largest_call_serves_smaller_ones(hq):
    big = attention_case(hq, "e4m3", [3000, 100], 4, 4, 64)
    kc = big[2]
    nb = hq.hq_cache_attention_workspace_bytes(kc, 2, 16, big[4].shape[1])
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    a = run_attention(hq, big, workspace=ws)
    assert torch.equal(a, run_attention(hq, big))
    for B in range(1, 40):
        for nblk in (1, 3, 50, 400):
            assert hq.hq_cache_attention_workspace_bytes(kc, B, 16, nblk) <= \
                hq.hq_cache_attention_workspace_bytes(kc, B + 1, 16, nblk + 1)
    with pytest.raises(hq.HQError):
        run_attention(hq, big, workspace=ws[:nb - 16])


def test_streams_and_graphs(hq):
    """A step (write, attend) on a side stream and captured, each replay equal to the eager run on
    the same inputs."""
    heads, group, bt = 4, 4, 32
    case = attention_case(hq, "int8", [1700, 33], heads, group, bt, seed=12)
    kp, vp, kc, vc, table, q, ln, scale = case
    table, q, ln = table.cuda(), q.cuda(), ln.cuda()
    k, v = (x.cuda() for x in inputs(2, heads, torch.bfloat16, 13))
    last = ln.long() - 1
    slots = table.long().gather(1, (last // bt)[:, None])[:, 0] * bt + last % bt
    ws = torch.empty(hq.hq_cache_attention_workspace_bytes(kc, 2, heads * group, table.shape[1]), dtype=torch.uint8,
                     device="cuda")
    out = torch.empty((2, heads * group, N), device="cuda")

    def step():
        hq.hq_cache_write(kp, k, kc, vp, v, vc, slots)
        hq.hq_cache_attention(kp, kc, vp, vc, q, table, ln, scale=scale, out=out, workspace=ws)

    step()
    eager = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out, eager)
    # the stream given to the calls, which take their workspace and outputs from it
    side.wait_stream(torch.cuda.current_stream())
    hq.hq_cache_write(kp, k, kc, vp, v, vc, slots, stream=side)
    got = hq.hq_cache_attention(kp, kc, vp, vc, q, table, ln, scale=scale, stream=side)
    back = hq.hq_cache_read(kp, kc, slots, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, eager) and torch.equal(back, hq.hq_cache_read(kp, kc, slots))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        k.copy_(torch.randn(k.shape, generator=torch.Generator().manual_seed(i)))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(50 + i)))
        out.zero_()
        graph.replay()
        got = out.clone()
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and got.any()


def test_refusals(hq):
    import ctypes as C
    L = hq.lib()
    heads, bt = 4, 32
    case = attention_case(hq, "int8", [40], heads, 2, bt)
    kp, vp, kc, vc, table, q, ln, scale = case
    table, q, ln = table.cuda(), q.cuda(), ln.cuda()
    out = torch.empty_like(q)
    x = torch.zeros((2, heads * N), device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")

    def cache(**kw):
        c = hq.CacheStruct.from_buffer_copy(kc.c)
        for n, v in kw.items():
            setattr(c, n, v)
        return c

    def attend(k=kc.c, v=vc.c, kpl=kp, heads_q=heads * 2, qt=1, ot=1, s=0.1, mb=table.shape[1], qp=None, batch=1):
        return L.hq_cache_attention(kpl.handle, C.byref(k), vp.handle, C.byref(v), q.data_ptr() if qp is None else qp,
                                    qt, batch, heads_q, s, table.data_ptr(), mb, ln.data_ptr(), out.data_ptr(), ot,
                                    None, 0, None)

    def write(c=kc.c, plan=kp, ptr=None, ld=heads * N, rows=2, xt=1, sl=None, v=None):
        return L.hq_cache_write(plan.handle, x.data_ptr() if ptr is None else ptr, ld, C.byref(c), v and plan.handle,
                                v and x.data_ptr(), ld if v else 0, v and C.byref(v), xt, rows,
                                slots.data_ptr() if sl is None else sl, None)

    def read(c=kc.c, plan=kp, ld=heads * N, rows=2, yt=1):
        return L.hq_cache_read(plan.handle, C.byref(c), slots.data_ptr(), rows, x.data_ptr(), yt, ld, None)

    kv = hq.hq_plan(cols=512, bps=2.0, rotation=hq.HQ_ROT_SIGNS, dither=True, norm_fp16=True)
    long = hq.hq_plan(tile=256, cols=512, bps=4.0)
    assert attend() == 0 and write() == 0 and read() == 0
    assert write(rows=0, ptr=0, sl=0) == 0 and read(rows=0) == 0 and attend(batch=0) == 0
    for call in (lambda **k: attend(**{("kpl" if n == "plan" else "k" if n == "c" else n): v for n, v in k.items()}),
                 write, read):
        assert call(plan=kv) == -2 and call(plan=long) == -2
        assert call(c=cache(format=2)) == -1 and call(c=cache(heads=0)) == -1 and call(c=cache(heads=5)) == -1
        assert call(c=cache(block_tokens=24)) == -2 and call(c=cache(block_tokens=0)) == -1
        assert call(c=cache(blocks=1 << 30)) == -2 and call(c=cache(blocks=0)) == -1
        assert call(c=cache(codes=None)) == -1 and call(c=cache(scales=kc.scales.data_ptr() + 4)) == -1
    assert attend(k=cache(blocks=0), v=cache(blocks=0)) == -1
    assert attend(v=cache(format=4)) == -1 and attend(v=cache(blocks=kc.blocks - 1)) == -1
    assert attend(heads_q=6) == -1 and attend(heads_q=0) == -1 and attend(heads_q=heads * 17) == -2
    assert attend(qt=2) == -1 and attend(ot=3) == -1 and attend(s=float("nan")) == -1 and attend(mb=0) == -1
    assert attend(qp=q.data_ptr() + 4) == -1 and attend(batch=-1) == -1
    assert attend(mb=(1 << 30) // bt + 1) == -2
    assert write(ld=heads * N - 4) == -1 and write(ptr=x.data_ptr() + 8) == -1 and write(rows=-1) == -1
    assert write(xt=2) == -1 and write(rows=1 << 30) == -2 and write(sl=slots.data_ptr() + 4) == -1
    assert write(v=cache()) == -1  # one cache for both
    assert read(ld=heads * N + 2) == -1 and read(yt=3) == -1
    with pytest.raises(ValueError):
        hq.hq_cache_write(kp, x, kc, None, None, None, slots.int())
    with pytest.raises(ValueError):
        hq.hq_cache_write(kp, x, kc, None, None, None, slots.cpu())
    with pytest.raises(ValueError):
        hq.hq_cache_read(kp, kc, slots, out=x[:, :128])
    with pytest.raises(ValueError):
        hq.hq_cache_attention(kp, kc, vp, vc, q[:, :, :64], table, ln)
    with pytest.raises(ValueError):
        hq.Cache(kp, 2, 32, hq.HQ_INT8, codes=torch.zeros((2, 4, 32, 64), dtype=torch.int8, device="cuda"))
    torch.cuda.synchronize()


def test_more_work_than_a_grid_holds_is_refused(hq):
    """2^32 threads: 2^28 vectors of a write or a read, 2^24 workgroups of an attention."""
    import ctypes as C
    L = hq.lib()
    heads, bt = 4, 32
    kp, vp, kc, vc, table, q, ln, scale = attention_case(hq, "int8", [40], heads, 2, bt)
    p = q.cuda().data_ptr()  # never reached
    k, v = C.byref(kc.c), C.byref(vc.c)
    rows = (1 << 28) // heads + 1
    assert L.hq_cache_write(kp.handle, p, heads * N, k, None, None, 0, None, 1, rows, p, None) == -2
    assert L.hq_cache_read(kp.handle, k, p, rows, p, 1, heads * N, None) == -2
    for blocks in (2, 400):
        assert L.hq_cache_attention(kp.handle, k, vp.handle, v, p, 1, (1 << 24) // heads, heads, 0.1, p, blocks, p, p,
                                    1, p, 1 << 60, None) == -2


def test_attention_block_step_on_casts(hq):
    """A layer's attention block as it is served: residual and norm into int8, the fused QKV
    product on a coded weight, the new keys and values into the cache, attention over it; each
    stage against 64 bits on what the stage before it gave."""
    hidden, heads, group, bt, B = 1024, 4, 2, 16, 5
    g = torch.Generator().manual_seed(21)
    width = (heads * group + 2 * heads) * N
    W = 0.03 * torch.randn((width, hidden), generator=g)
    plan = hq.hq_plan(cols=hidden, bps=4.0, rht_seed=3)
    s = hq.EncodedStream(plan, width)
    hq.hq_encode(plan, W.cuda(), s)
    codes, gs = hq.hq_decode_int8(plan, s)
    w_hat = hq.hq_decode(plan, s, out_dtype=torch.float32).cpu().double().numpy()
    kp, vp = R.plans(hq, heads)
    nb = 4
    kc, vc = R.random_cache(hq, kp, "int8", B * nb, heads, bt, 4), R.random_cache(hq, vp, "int8", B * nb, heads, bt, 5)
    table = torch.randperm(B * nb, generator=g).view(B, nb).to(torch.int32)
    lens = torch.tensor([1, 17, 64, 33, 50], dtype=torch.int32)
    weight = (1 + 0.1 * torch.randn(hidden, generator=g)).to(torch.bfloat16)
    x, r = (torch.randn((B, hidden), generator=g).to(torch.bfloat16) for _ in range(2))
    xq, sx, h = hq.hq_rmsnorm_act_prep(plan, x.cuda(), weight.cuda(), residual=r.cuda())
    qkv = hq.hq_gemm_int8_blockscaled(plan, xq, sx, codes, gs, out_dtype=torch.float32)
    nq = heads * group * N
    last = lens.long() - 1
    slots = (table.long().gather(1, (last // bt)[:, None])[:, 0] * bt + last % bt).cuda()
    hq.hq_cache_write(kp, qkv[:, nq:nq + heads * N], kc, vp, qkv[:, nq + heads * N:], vc, slots)
    q = qkv[:, :nq].contiguous().view(B, heads * group, N)
    out = hq.hq_cache_attention(kp, kc, vp, vc, q, table.cuda(), lens.cuda())
    torch.cuda.synchronize()
    hd = h.cpu().double().numpy()
    assert torch.equal(h.cpu(), (x.float() + r.float()).to(torch.bfloat16))
    n64 = hd * weight.double().numpy() / np.sqrt((hd * hd).mean(-1, keepdims=True) + 1e-5)
    # int8 activations: each rotated value is at most half of s_x off, so a product with a weight
    # row by at most half of s_x times the row's rotated coordinates' magnitudes
    rot = np.abs((w_hat * R.signs(3, hidden)).reshape(width, -1, N) @ R.hadamard() / N).reshape(width, -1)
    room = sx.cpu().double().numpy()[:, None] * 0.501 * rot.sum(-1) + 1e-4
    got = qkv.cpu().double().numpy()
    assert (np.abs(got - n64 @ w_hat.T) <= room).all()
    at = slots.cpu().numpy()
    for part, c, seed in ((got[:, nq:nq + heads * N], kc, R.SEED_K), (got[:, nq + heads * N:], vc, R.SEED_V)):
        y, err = R.transform(part, seed, heads)
        R.check_codes("int8", y, err, R.values(c)[at // bt, :, at % bt])
    ref, tol = R.attend(q.cpu().numpy(), R.values(kc), R.values(vc), table.numpy(), lens.numpy(), bt, N ** -0.5, heads,
                        group)
    assert (np.abs(out.cpu().numpy() - ref) <= tol).all()
