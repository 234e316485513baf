"""One-token attention over a window of the cache with sinks (hq_cache_window_attention) against
its definition in 64 bits (tests/rows64.py)."""
import numpy as np
import pytest
import torch

from tests import cache64 as R
from tests import rows64 as W

pytestmark = pytest.mark.gpu
FMTS = ["int8", "e4m3", "mxfp4"]
N = R.N
INVALID_ARG = -1 & 0xFFFFFFFF


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    assert torch.cuda.is_available()
    return H


def case(hq, fmt, lens, heads, group, bt, seed=0, qdt=torch.float32, pool=None):
    """`pool`: blocks of the cache, shared by the sequences; else each has its own."""
    kp, vp = R.plans(hq, heads)
    B, nb = len(lens), max(1, -(-max(lens) // bt))
    blocks = pool or B * nb + 1
    kc, vc = (R.random_cache(hq, p, fmt, blocks, heads, bt, 10 * i + seed) for i, p in ((1, kp), (2, vp)))
    g = torch.Generator().manual_seed(30 + seed)
    table = (torch.randint(0, blocks, (B, nb), generator=g) if pool else torch.randperm(blocks, generator=g)[:B * nb].view(B, nb))
    q = torch.randn((B, heads * group, N), generator=g).to(qdt)
    return kp, vp, kc, vc, table.to(torch.int32), q, torch.tensor(lens, dtype=torch.int32)


def run(hq, c, window, sinks, **kw):
    kp, vp, kc, vc, table, q, lens = c
    return hq.hq_cache_window_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda(), window, sinks, **kw)


def reference(c, window, sinks, heads, group, bt, lens=None):
    kp, vp, kc, vc, table, q, ln = c
    kv, vv = R.values(kc), R.values(vc)
    parts = [W.attend(q[b:b + 1].float().numpy(), kv, vv, table[b].numpy(), W.visible(int(n), window, sinks)[None], bt,
                      N ** -0.5, heads, group) for b, n in enumerate(ln if lens is None else lens)]
    return np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])


def check(hq, c, window, sinks, heads, group, bt, lens=None):
    out = run(hq, c, window, sinks, out=torch.full((len(c[6]), heads * group, N), float("nan"), device="cuda"))
    W.check(out.cpu().numpy(), *reference(c, window, sinks, heads, group, bt, lens))
    assert torch.equal(run(hq, c, window, sinks, out_dtype=torch.bfloat16), out.to(torch.bfloat16))
    assert torch.equal(run(hq, c, window, sinks), out)  # the same bits again
    return out


LENS = [0, 1, 2, 15, 16, 17, 33, 64, 100, 127, 128, 129, 300, 511]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bt", [16, 48, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (31, 16), (32, 17), (100, 40), (128, 128), (255, 0),
                                          (1, 300), (2000, 3)])
def test_lengths(hq, fmt, bt, window, sinks):
    print(f"[window] lengths {fmt} bt={bt} {window} {sinks}", flush=True)
    check(hq, case(hq, fmt, LENS, 2, 2, bt), window, sinks, 2, 2, bt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (3, 5), (4, 8), (8, 4), (16, 1), (2, 12)])
def test_heads(hq, fmt, heads, group):
    print(f"[window] heads {fmt} {heads} x {group}", flush=True)
    check(hq, case(hq, fmt, [301, 64, 130, 0], heads, group, 32, seed=heads, qdt=torch.bfloat16), 99, 5, heads, group, 32)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("lens,window,sinks", [([9000], 3000, 4), ([9000], 1008, 1), ([9000], 1009, 1), ([20000, 3, 0, 700], 5000, 0),
                                               ([6000] * 9, 1999, 67), ([5000] * 40, 100, 1500), ([129 * i for i in range(64)], 2500, 33),
                                               ([64] * 70, 30, 2), ([97 * (i % 50) for i in range(150)], 1500, 20)])
def test_splits_and_joins(hq, fmt, lens, window, sinks):
    print(f"[window] splits {fmt} {len(lens)} x {max(lens)} {window} {sinks}", flush=True)
    check(hq, case(hq, fmt, lens, 2, 4, 64, seed=3, pool=40), window, sinks, 2, 4, 64)


@pytest.mark.parametrize("B", [64, 65, 600])
def test_many_sequences(hq, B):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 3000, (B,), generator=g)
    lens[::7] = 0
    check(hq, case(hq, "int8", lens.tolist(), 1, 2, 48, seed=B, pool=30), 1100, 7, 1, 2, 48)


@pytest.mark.parametrize("fmt", FMTS)
def test_a_window_of_everything_is_the_attention(hq, fmt):
    c = case(hq, fmt, [3000, 5, 0, 1024], 4, 4, 64, seed=5)
    kp, vp, kc, vc, table, q, lens = c
    whole = hq.hq_cache_attention(kp, kc, vp, vc, q.cuda(), table.cuda(), lens.cuda())
    for window, sinks in ((table.shape[1] * 64, 0), (2 ** 31 - 1, 0), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        got = run(hq, c, window, sinks)
        if sinks == 0 or window > 1:
            assert torch.equal(got, whole)
        else:
            W.check(got.cpu().numpy(), *reference(c, window, sinks, 4, 4, 64))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(40, 0), (37, 5), (1, 1), (70, 33)])
def test_ignores_what_nobody_sees(hq, fmt, window, sinks):
    """Any bit pattern in tokens between the sinks and the window and behind the sequence, in the
    same blocks as visible ones; table entries of blocks without a visible token may name none."""
    lens, bt = [333, 5, 128, 90, 0], 32
    c = case(hq, fmt, lens, 4, 4, bt, seed=6)
    kp, vp, kc, vc, table, q, ln = c
    clean = run(hq, c, window, sinks)
    live = torch.zeros((kc.blocks, bt), dtype=torch.bool)
    for b, n in enumerate(lens):
        t = torch.from_numpy(np.nonzero(W.visible(n, window, sinks))[0])
        live[table[b, t // bt].long(), t % bt] = True
        used = torch.zeros(table.shape[1], dtype=torch.bool)
        used[t // bt] = True
        table[b, ~used] = -7
    dead = (~live).cuda()
    for x in (kc, vc):
        x.codes.view(torch.uint8).transpose(1, 2)[dead] = 0x7F if fmt == "e4m3" else 0x80
        x.scales.transpose(1, 2)[dead] = float("nan") if fmt != "mxfp4" else 255
    assert torch.equal(clean, run(hq, c, window, sinks))
    assert kc.read_stats()["status"] == 0


def test_bad_blocks_and_lengths(hq):
    c = case(hq, "int8", [100, 70, 300, 40], 4, 2, 32, seed=8)
    kp, vp, kc, vc, table, q, ln = c
    table[0, 2], table[1, 0], table[3, :] = kc.blocks, -1, 1 << 30
    out = check(hq, c, 50, 10, 4, 2, 32)
    assert not out[3].any() and kc.read_stats()["status"] == INVALID_ARG
    kc.reset_stats()
    cap = table.shape[1] * 32
    table[:] = torch.arange(table.numel(), dtype=torch.int32).view(table.shape)
    bad = (kp, vp, kc, vc, table, q, torch.tensor([-3, cap + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
    out = check(hq, bad, 50, 10, 4, 2, 32, lens=[0, cap, cap, 0])
    assert not out[0].any() and kc.read_stats()["status"] == INVALID_ARG


def test_replayed_while_the_sequences_grow(hq):
    """A captured call follows the lengths, across a window's block borders and its splits."""
    c = case(hq, "e4m3", [4000, 3000, 4000, 100], 2, 4, 64, seed=9)
    kp, vp, kc, vc, table, q, lens = c
    q, table, ln, out = q.cuda(), table.cuda(), lens.cuda(), torch.empty_like(q, device="cuda")
    ws = torch.empty(hq.hq_cache_window_workspace_bytes(kc, 4, 8, table.shape[1], 1500, 20), dtype=torch.uint8, device="cuda")
    call = lambda o, w: hq.hq_cache_window_attention(kp, kc, vp, vc, q, table, ln, 1500, 20, out=o, workspace=w)
    call(out, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    other = torch.empty_like(ws)
    for n in (0, 1, 19, 21, 1024, 1519, 1520, 1521, 1536, 1537, 3999):
        ln.copy_(torch.tensor([n, min(n, 3000), 4000 - n, 100], dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        eager = call(torch.full_like(out, float("nan")), other)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.isfinite(out).all()


def test_workspaces(hq):
    c = case(hq, "int8", [3000, 2000], 4, 4, 64)
    kc, nb = c[2], c[4].shape[1]
    n = lambda w, s: hq.hq_cache_window_workspace_bytes(kc, 2, 16, nb, w, s)
    assert n(1000, 0) == 0 and 0 < n(1100, 0) <= n(1100, 64) <= n(3000, 64) == n(2 ** 31 - 1, 2 ** 31 - 1)
    assert n(2 ** 31 - 1, 0) == hq.hq_cache_attention_workspace_bytes(kc, 2, 16, nb)
    with pytest.raises(hq.HQError):
        run(hq, c, 2000, 0, workspace=torch.empty(n(2000, 0) - 1, dtype=torch.uint8, device="cuda"))
    big = torch.empty(n(3000, 64), dtype=torch.uint8, device="cuda")
    assert torch.equal(run(hq, c, 1200, 0, workspace=big), run(hq, c, 1200, 0))
    for bad in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(hq.HQError):
            run(hq, c, *bad)


@pytest.mark.parametrize("fmt", FMTS)
def test_on_another_stream_and_past_32_bit_offsets(hq, fmt):
    heads, bt, rows = 8, 256, 900
    kp, vp = R.plans(hq, heads)
    blocks = (5 << 30) // (heads * bt * (64 if fmt == "mxfp4" else 128))
    form = {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]
    far = [hq.Cache(p, blocks, bt, form, heads=heads) for p in (kp, vp)]
    near = [R.random_cache(hq, p, fmt, 4, heads, bt, i) for i, p in enumerate((kp, vp))]
    table = torch.tensor([[blocks - 1, 3, blocks // 2, blocks - 2]], dtype=torch.int32)
    for a, b in zip(far, near):
        a.codes[table[0].long().cuda()], a.scales[table[0].long().cuda()] = b.codes, b.scales
    q = torch.randn((1, heads * 4, N), generator=torch.Generator().manual_seed(2)).cuda()
    ln = torch.tensor([rows], dtype=torch.int32, device="cuda")
    want = hq.hq_cache_window_attention(kp, near[0], vp, near[1], q, torch.arange(4, dtype=torch.int32, device="cuda")[None], ln, 300, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hq.hq_cache_window_attention(kp, far[0], vp, far[1], q, table.cuda(), ln, 300, 9, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and got.any()
