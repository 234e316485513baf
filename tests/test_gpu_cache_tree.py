"""The attention of drafted tokens over the cache (hq_cache_tree_attention) against its definition
in 64 bits (tests/rows64.py), and a step of drafting with the cache's append."""
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


class Case:
    def __init__(self, hq, fmt, lens, trees, heads, group, bt, seed=0, qdt=torch.float32, pool=None, window=0, sinks=0,
                 masks=None, max_tree=None, scale=N ** -0.5):
        self.hq, self.heads, self.group, self.bt, self.window, self.sinks, self.scale = hq, heads, group, bt, window, sinks, scale
        self.kp, self.vp = R.plans(hq, heads)
        B, nb = len(lens), max(1, -(-max(lens) // bt))
        blocks = pool or B * nb + 1
        self.kc, self.vc = (R.random_cache(hq, p, fmt, blocks, heads, bt, 10 * i + seed) for i, p in ((1, self.kp), (2, self.vp)))
        g, rng = torch.Generator().manual_seed(30 + seed), np.random.default_rng(seed)
        self.table = (torch.randint(0, blocks, (B, nb), generator=g) if pool
                      else torch.randperm(blocks, generator=g)[:B * nb].view(B, nb)).to(torch.int32)
        self.lens, self.trees = list(lens), list(trees)
        self.masks = masks or [m for n in trees for m in W.random_tree(rng, n)]
        self.starts = np.concatenate(([0], np.cumsum(trees))).astype(np.int32)
        self.max_tree = max_tree or max(max(trees), 1)
        self.q = torch.randn((int(self.starts[-1]), heads * group, N), generator=g).to(qdt)

    def run(self, **kw):
        args = dict(window=self.window, sinks=self.sinks, scale=self.scale, **kw)
        return self.hq.hq_cache_tree_attention(self.kp, self.kc, self.vp, self.vc, self.q.cuda(), W.mask_tensor(self.masks).cuda(),
                                               torch.from_numpy(self.starts).cuda(), self.max_tree, self.table.cuda(),
                                               torch.tensor(self.lens, dtype=torch.int32, device="cuda"), **args)

    def reference(self):
        kv, vv = R.values(self.kc), R.values(self.vc)
        out, tol = np.zeros(self.q.shape), np.full(self.q.shape, 1e-30)
        for b, n in enumerate(self.lens):
            r = slice(self.starts[b], self.starts[b + 1])
            live = W.tree_visible(n, self.masks[r], self.window, self.sinks)
            out[r], tol[r] = W.attend(self.q[r].float().numpy(), kv, vv, self.table[b].numpy(), live, self.bt, self.scale, self.heads,
                                      self.group)
        return out, tol

    def check(self):
        out = self.run(out=torch.full(self.q.shape, float("nan"), device="cuda"))
        W.check(out.cpu().numpy(), *self.reference(), scale=self.scale)
        assert torch.equal(self.run(out_dtype=torch.bfloat16), out.to(torch.bfloat16))
        assert torch.equal(self.run(), out)  # the same bits again
        assert self.kc.read_stats()["status"] == 0
        return out


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 47, 64, 65, 100, 127, 129, 256, 511]
TREES = [0, 1, 2, 3, 16, 1, 7, 8, 12, 13, 0, 5, 16, 9, 4, 16]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bt", [16, 48, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4)])
def test_lengths(hq, fmt, bt, heads, group):
    print(f"[tree] lengths {fmt} bt={bt} {heads} x {group}", flush=True)
    Case(hq, fmt, LENS, TREES, heads, group, bt).check()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads,group,tree", [(1, 1, 64), (1, 16, 64), (2, 3, 5), (3, 5, 25), (4, 7, 9), (4, 8, 33), (8, 4, 64), (16, 1, 17),
                                              (2, 12, 11), (2, 16, 1), (8, 2, 8)])
def test_heads(hq, fmt, heads, group, tree):
    print(f"[tree] heads {fmt} {heads} x {group} x {tree}", flush=True)
    Case(hq, fmt, [301, 64, 130], [tree, min(tree, 30), max(1, tree // 2)], heads, group, 32, seed=heads, qdt=torch.bfloat16).check()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("lens,trees", [([1000], [7]), ([2500, 3, 0, 700], [8, 3, 0, 1]), ([9000], [64]), ([1024, 0, 513], [4, 0, 40]),
                                        ([129 * (i % 30) for i in range(64)], [min(129 * (i % 30), 1 + i % 9) for i in range(64)]),
                                        ([0, 0, 1300], [0, 0, 30])])
def test_splits_and_joins(hq, fmt, lens, trees):
    print(f"[tree] splits {fmt} {len(lens)} x {max(lens)}", flush=True)
    Case(hq, fmt, lens, trees, 2, 4, 64, seed=3, pool=40).check()


@pytest.mark.parametrize("B,heads,group,tree", [(64, 1, 2, 4), (65, 1, 2, 9), (129, 2, 3, 3), (600, 1, 1, 20), (300, 3, 5, 2)])
def test_many_sequences(hq, B, heads, group, tree):
    print(f"[tree] many {B} x {heads} x {group} x {tree}", flush=True)
    rng = np.random.default_rng(B)
    lens = np.maximum(rng.integers(-40, 90, B), 0)
    lens[rng.integers(0, B, 5)] = [1023, 1024, 1025, 1536, 2000]
    Case(hq, "int8", lens.tolist(), np.minimum(lens, rng.integers(0, tree + 1, B)).tolist(), heads, group, 48, seed=B, pool=30,
         max_tree=tree).check()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(64, 0), (65, 1), (70, 17), (100, 300), (128, 16), (900, 5), (5000, 0)])
@pytest.mark.parametrize("lens,trees", [([300, 64, 65, 80, 513, 1, 0], [20, 30, 1, 30, 30, 1, 0]), ([4000, 1200, 64], [30, 12, 30])])
def test_windows(hq, fmt, window, sinks, lens, trees):
    print(f"[tree] windows {fmt} {window} {sinks} {lens[0]}", flush=True)
    Case(hq, fmt, lens, trees, 2, 4, 32, seed=4, window=window, sinks=sinks).check()


@pytest.mark.parametrize("fmt", FMTS)
def test_a_chain_is_a_causal_step(hq, fmt):
    """Row i of a chain is the one-token attention of the sequence cut behind its token."""
    n, heads, group, bt = 9, 4, 4, 32
    c = Case(hq, fmt, [300], [n], heads, group, bt, seed=5, masks=[(2 << i) - 1 for i in range(n)])
    out = c.check()
    one = hq.hq_cache_attention(c.kp, c.kc, c.vp, c.vc, c.q.cuda(), c.table.expand(n, -1).contiguous().cuda(),
                                torch.arange(300 - n + 1, 301, dtype=torch.int32, device="cuda"))
    _, tol = c.reference()
    assert (np.abs((out - one).cpu().numpy()) <= 2 * tol).all()


@pytest.mark.parametrize("window", [0, 64])
def test_rows_that_see_nothing(hq, window):
    """A mask of zeros without a context, and masks whose bits lie behind the tree."""
    masks = [0, 1, 0, 1 << 3 | 1, -1 & (2 ** 64 - 1), 0, (2 ** 64 - 1) << 3 & (2 ** 64 - 1)]
    c = Case(hq, "e4m3", [3, 4], [3, 4], 2, 4, 16, seed=6, masks=masks, window=window, max_tree=4)
    out = c.check()
    assert not out[0].any() and not out[2].any() and not out[5].any() and out[1].any() and out[6].any()


def test_rows_of_no_sequence_are_left(hq):
    c = Case(hq, "int8", [100, 50, 60], [5, 4, 6], 2, 2, 16, seed=7)
    whole = c.check()
    c.starts = np.array([2, 5, 9, 13], dtype=np.int32)  # rows 0, 1, 13 and 14 are nobody's
    out = c.run(out=torch.full(c.q.shape, 7.0, device="cuda"))
    assert (out[:2] == 7).all() and (out[13:] == 7).all() and torch.isfinite(out).all()
    assert not c.run()[13:].any()
    assert c.kc.read_stats()["status"] == 0 and whole.any()


@pytest.mark.parametrize("starts,lens,left", [([0, 5, 3, 15], [100, 50, 60], [1, 2]), ([-1, 5, 9, 15], [100, 50, 60], [0]),
                                              ([0, 5, 9, 16], [100, 50, 60], [2]), ([0, 7, 9, 15], [100, 50, 60], [0]),
                                              ([0, 5, 9, 15], [100, 3, 60], [1]), ([0, 5, 9, 15], [4, 50, 0], [0, 2]),
                                              ([0, 2 ** 31 - 1, 9, 15], [100, 50, 60], [0, 1])])
def test_sequences_out_of_range_are_left_out_and_reported(hq, starts, lens, left):
    """Rows that fall, lie outside the call, or are more than max_tree (6) or than the tokens: the other
    sequences' rows are right, nothing else is written."""
    c = Case(hq, "int8", [100, 50, 60], [5, 4, 6], 2, 2, 16, seed=8)
    c.starts, c.lens = np.array(starts, dtype=np.int32), lens
    out = c.run(out=torch.full(c.q.shape, 7.0, device="cuda")).cpu().numpy()
    assert c.kc.read_stats()["status"] == INVALID_ARG
    kv, vv = R.values(c.kc), R.values(c.vc)
    rest = np.ones(15, dtype=bool)
    for b in range(3):
        if b in left:
            continue
        r = slice(starts[b], starts[b + 1])
        rest[r] = False
        live = W.tree_visible(lens[b], c.masks[r])
        W.check(out[r], *W.attend(c.q[r].numpy(), kv, vv, c.table[b].numpy(), live, 16, N ** -0.5, 2, 2))
    assert (out[rest] == 7).all()


def test_bad_blocks_and_lengths(hq):
    c = Case(hq, "int8", [100, 70, 300, 40], [5, 9, 3, 8], 4, 2, 32, seed=9)
    c.table[0, 1], c.table[1, 0], c.table[3, :] = c.kc.blocks, -1, 1 << 30
    out = c.run()
    W.check(out.cpu().numpy(), *c.reference())
    assert not out[17:].any() and c.kc.read_stats()["status"] == INVALID_ARG
    c.kc.reset_stats()
    c.table[:] = torch.arange(c.table.numel(), dtype=torch.int32).view(c.table.shape)
    cap = c.table.shape[1] * 32
    c.lens = [cap, cap, cap, cap]
    want = c.run()
    assert c.kc.read_stats()["status"] == 0
    c.lens = [cap + 1, cap, 2 ** 31 - 1, cap]
    assert torch.equal(c.run(), want) and c.kc.read_stats()["status"] == INVALID_ARG


@pytest.mark.parametrize("fmt", FMTS)
def test_ignores_what_lies_behind_a_sequence(hq, fmt):
    lens, trees = [37, 5, 128, 0], [9, 5, 16, 0]
    c = Case(hq, fmt, lens, trees, 4, 4, 64, seed=10)
    clean = c.run()
    live = torch.zeros((c.kc.blocks, 64), dtype=torch.bool)
    for b, n in enumerate(lens):
        t = torch.arange(n)
        live[c.table[b, t // 64].long(), t % 64] = True
        c.table[b, -(-n // 64):] = -7
    dead = (~live).cuda()
    for x in (c.kc, c.vc):
        x.codes.view(torch.uint8).transpose(1, 2)[dead] = 0x7F if fmt == "e4m3" else 0x80
        x.scales.transpose(1, 2)[dead] = float("nan") if fmt != "mxfp4" else 255
    assert torch.equal(clean, c.run()) and c.kc.read_stats()["status"] == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("side", ["k", "v"])
def test_a_token_that_is_not_finite_reaches_the_rows_that_see_it(hq, fmt, side):
    """A drafted token stored as NaN makes its descendants NaN and leaves the other branches; one
    between the sinks and a window leaves every row."""
    rng = np.random.default_rng(11)
    n = 24
    masks = W.random_tree(rng, n)
    c = Case(hq, fmt, [200], [n], 2, 4, 32, seed=11, masks=masks, window=64, sinks=3)
    clean = c.check().cpu().numpy()
    cache = c.kc if side == "k" else c.vc
    poison = next(j for j in range(n) if 1 < sum(m >> j & 1 for m in masks) < n // 2)
    for t in (200 - n + poison, 50):
        blk = int(c.table[0, t // 32])
        cache.codes[blk, :, t % 32] = 0
        cache.scales[blk, :, t % 32] = float("nan") if fmt != "mxfp4" else 255
    out = c.run().cpu().numpy()
    sees = np.array([bool(m >> poison & 1) for m in masks])
    assert np.isnan(out[sees]).all() and not np.isnan(out[~sees]).any()
    assert np.array_equal(out[~sees], clean[~sees])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("spread", [3, 10])
def test_scales_far_apart(hq, fmt, spread):
    """Values of very different size, zero vectors among them: a term is right relative to the
    largest that the row sums."""
    c = Case(hq, fmt, [400, 90], [9, 20], 2, 4, 32, seed=12)
    g = torch.Generator().manual_seed(1)
    c.vc.scales.copy_(10.0 ** (spread * (2 * torch.rand(c.vc.scales.shape, generator=g) - 1)))
    c.vc.scales[:, :, 5::11] = 0.0
    c.kc.scales[:, :, 7::13] = 0.0
    out = c.run()
    ref, tol = c.reference()
    # of the largest weight times value instead of the largest value times any weight: the bound
    # per row goes by what the row sums
    off = np.abs(out.cpu().numpy() - ref)
    assert (off <= tol).all()
    size = np.linalg.norm(ref, axis=-1)
    assert (np.linalg.norm(off, axis=-1) <= 64 * R.U * 4 * size).all()


@pytest.mark.parametrize("factor", [1e-30, 1e-6, 1e6, 1e20])
def test_queries_and_values_of_any_size(hq, factor):
    c = Case(hq, "e4m3", [300, 40], [9, 20], 2, 4, 32, seed=13)
    c.q = c.q * factor
    c.kc.scales.copy_(c.kc.scales / factor)
    out = c.run()
    ref, tol = c.reference()
    W.check(out.cpu().numpy(), ref, tol)
    c.vc.scales.copy_(c.vc.scales * factor)
    ref, tol = c.reference()
    W.check(c.run().cpu().numpy(), ref, tol)


def test_rows_of_very_different_size(hq):
    c = Case(hq, "int8", [300], [16], 1, 4, 32, seed=14)
    c.q = c.q * (10.0 ** torch.arange(-8, 8).float())[:, None, None].clamp(max=3.0)
    c.q[3], c.q[4, 1] = 0.0, 0.0
    c.check()


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0])
def test_scales(hq, scale):
    Case(hq, "int8", [200, 33], [12, 5], 4, 2, 16, seed=15, scale=scale).check()


def test_replayed_beside_another_graph_and_on_another_stream(hq):
    a = Case(hq, "e4m3", [3000, 1500, 40, 2000], [20, 1, 30, 32], 2, 4, 64, seed=16, max_tree=32)
    dev = lambda x: x.cuda()
    q, masks, starts = dev(a.q), dev(W.mask_tensor(a.masks)), dev(torch.from_numpy(a.starts))
    table, lens = dev(a.table), torch.tensor(a.lens, dtype=torch.int32, device="cuda")
    nbytes = hq.hq_cache_tree_workspace_bytes(a.kc, 4, 8, table.shape[1], 32)
    ws = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs = [torch.empty_like(q) for _ in range(3)]

    def call(i, stream=None):
        return hq.hq_cache_tree_attention(a.kp, a.kc, a.vp, a.vc, q, masks, starts, 32, table, lens, out=outs[i], workspace=ws[i],
                                          stream=stream)
    call(0)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    side = torch.cuda.Stream()
    for shift in range(4):
        lens.copy_(torch.tensor(np.maximum(np.array(a.lens) - 7 * shift, a.trees), dtype=torch.int32))
        starts.copy_(torch.from_numpy(a.starts) if shift != 2 else torch.tensor([0, 10, 21, 51, 83], dtype=torch.int32))
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        call(2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.isfinite(outs[0]).all()


def test_workspaces(hq):
    c = Case(hq, "int8", [3000, 2000], [8, 30], 4, 4, 64, seed=17)
    nb = c.table.shape[1]
    n = lambda **k: hq.hq_cache_tree_workspace_bytes(c.kc, k.get("batch", 2), k.get("heads_q", 16), k.get("nb", nb), k.get("tree", 30),
                                                     k.get("window", 0), k.get("sinks", 0))
    assert n(window=100) == 0 and n() > 0 and n(tree=65) == 0 and n(tree=0) == 0
    with pytest.raises(hq.HQError):
        c.run(workspace=torch.empty(n() - 1, dtype=torch.uint8, device="cuda"))
    big = torch.empty(n(batch=5, heads_q=64, nb=nb + 9, tree=64), dtype=torch.uint8, device="cuda")
    assert torch.equal(c.run(workspace=big), c.run(workspace=torch.empty(n(), dtype=torch.uint8, device="cuda")))
    c.window = 29
    with pytest.raises(hq.HQError):
        c.run()


@pytest.mark.parametrize("fmt", FMTS)
def test_caches_past_32_bit_offsets(hq, fmt):
    heads, bt = 8, 256
    kp, vp = R.plans(hq, heads)
    blocks = (5 << 30) // (heads * bt * (64 if fmt == "mxfp4" else 128))
    form = {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]
    near = Case(hq, fmt, [500], [7], heads, 4, bt, seed=18)
    want = near.run()
    place = torch.tensor([blocks - 1, blocks // 2])
    old = near.table[0].long().cuda()
    for name in ("kc", "vc"):
        small, plan = getattr(near, name), near.kp if name == "kc" else near.vp
        far = hq.Cache(plan, blocks, bt, form, heads=heads)
        far.codes[place.cuda()], far.scales[place.cuda()] = small.codes[old], small.scales[old]
        setattr(near, name, far)
    near.table = place.to(torch.int32)[None]
    assert torch.equal(near.run(), want) and want.any()


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (96, 4)])
def test_a_drafted_step(hq, fmt, window, sinks):
    """As a server drafts: a prompt is appended with its positions, a tree of drafted tokens behind
    it (positions by depth), the trees are checked in one call, the accepted path stays and the
    next token attends over what is left, with a window too; each against 64 bits."""
    heads, group, bt, rope_dims = 4, 4, 32, 128
    rng, g = np.random.default_rng(19), torch.Generator().manual_seed(19)
    kp, vp = R.plans(hq, heads)
    form = {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[fmt]
    prompts, trees = [150, 33, 270], [13, 1, 24]
    nb = 10
    table = torch.randperm(3 * nb, generator=g).view(3, nb).to(torch.int32)
    kc, vc = (hq.Cache(p, 3 * nb, bt, form, heads=heads) for p in (kp, vp))
    freq = torch.from_numpy(10000.0 ** (-np.arange(64) / 64)).cuda()
    rope = hq.Rope(hq.hq_rope_table(freq, 512))
    slot = lambda b, t: int(table[b, t // bt]) * bt + t % bt

    def append(places, positions):
        rows = len(places)
        qkv = torch.randn((rows, (group + 2) * heads * N), generator=g).to(torch.bfloat16).cuda()
        q, k, v = qkv.split([group * heads * N, heads * N, heads * N], 1)
        slots = torch.tensor([slot(b, t) for b, t in places], device="cuda")
        return hq.hq_cache_append(kp, k, kc, vp, v, vc, slots, rope, torch.tensor(positions, dtype=torch.int32, device="cuda"), q=q)

    append([(b, t) for b, n in enumerate(prompts) for t in range(n)], [t for n in prompts for t in range(n)])
    masks = [W.random_tree(rng, n) for n in trees]
    q = append([(b, prompts[b] + i) for b, n in enumerate(trees) for i in range(n)],
               [prompts[b] + bin(m).count("1") - 1 for b in range(3) for m in masks[b]])
    lens = np.array(prompts) + trees
    starts = np.concatenate(([0], np.cumsum(trees))).astype(np.int32)
    out = hq.hq_cache_tree_attention(kp, kc, vp, vc, q.view(-1, heads * group, N), W.mask_tensor(sum(masks, [])).cuda(),
                                     torch.from_numpy(starts).cuda(), 24, table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(),
                                     window=window, sinks=sinks)
    kv, vv = R.values(kc), R.values(vc)
    got, qn = out.cpu().numpy(), q.float().cpu().numpy().reshape(-1, heads * group, N)
    for b in range(3):
        r = slice(starts[b], starts[b + 1])
        live = W.tree_visible(int(lens[b]), masks[b], window, sinks)
        W.check(got[r], *W.attend(qn[r], kv, vv, table[b].numpy(), live, bt, N ** -0.5, heads, group))
    # the longest path of each tree is accepted: its rows move behind the prompt
    paths = [[j for j in range(n) if max(m, key=lambda x: bin(x).count("1")) >> j & 1] for n, m in zip(trees, masks)]
    source = torch.tensor([slot(b, prompts[b] + j) for b in range(3) for j in paths[b]], device="cuda")
    target = torch.tensor([slot(b, prompts[b] + i) for b in range(3) for i in range(len(paths[b]))], device="cuda")
    for c in (kc, vc):
        codes, scales = c.codes.transpose(1, 2), c.scales.transpose(1, 2)
        codes[target // bt, target % bt], scales[target // bt, target % bt] = codes[source // bt, source % bt], scales[source // bt, source % bt]
    lens = [n + len(p) for n, p in zip(prompts, paths)]
    q = append([(b, n) for b, n in enumerate(lens)], lens).view(3, heads * group, N)
    lens = [n + 1 for n in lens]
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kv, vv = R.values(kc), R.values(vc)
    if window:
        out = hq.hq_cache_window_attention(kp, kc, vp, vc, q, table.cuda(), ln, window, sinks)
    else:
        out = hq.hq_cache_attention(kp, kc, vp, vc, q, table.cuda(), ln)
    for b, n in enumerate(lens):
        live = W.visible(n, window or n, sinks)[None]
        W.check(out[b:b + 1].cpu().numpy(), *W.attend(q[b:b + 1].float().cpu().numpy(), kv, vv, table[b].numpy(), live, bt, N ** -0.5,
                                                       heads, group))


@pytest.mark.parametrize("fmt", FMTS)
def test_windows_of_many_long_sequences(hq, fmt):
    """More sequences than a wave has lanes, split and joined, each looked at from its window on."""
    rng = np.random.default_rng(20)
    lens = np.maximum(rng.integers(-500, 3500, 90), 0)
    lens[::5] = 3500
    Case(hq, fmt, lens.tolist(), np.minimum(lens, rng.integers(0, 12, 90)).tolist(), 1, 4, 48, seed=20, pool=30, window=1500,
         sinks=21, max_tree=12).check()


@pytest.mark.parametrize("heads", [512, 600])
def test_as_many_heads_as_workgroups(hq, heads):
    """From 512 KV heads on no sequence is split, however long the table."""
    Case(hq, "int8", [1100, 0, 1500, 3], [2, 0, 1, 3], heads, 1, 64, seed=heads, pool=12).check()


def test_no_rows_and_no_sequences(hq):
    c = Case(hq, "int8", [100, 30], [0, 0], 2, 2, 32, seed=21)
    assert c.run().shape == (0, 4, N)
    c = Case(hq, "int8", [100], [3], 2, 2, 32, seed=21)
    empty = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    out = torch.full((3, 4, N), 7.0, device="cuda")
    hq.hq_cache_tree_attention(c.kp, c.kc, c.vp, c.vc, c.q.cuda(), W.mask_tensor(c.masks).cuda(), empty(1), 3, empty(0, 4), empty(0),
                               out=out)
    assert (out == 7).all()


def test_two_calls_at_once(hq):
    """Two calls on two streams over one cache, a workspace each."""
    c = Case(hq, "int8", [3000, 1200], [30, 17], 4, 4, 64, seed=22)
    want, streams, got = c.run(), [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(3):
        torch.cuda.synchronize()
        outs = [torch.empty_like(want) for _ in streams]
        torch.cuda.synchronize()
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                c.run(out=o)
        torch.cuda.synchronize()
        got += outs
    assert all(torch.equal(o, want) for o in got)
