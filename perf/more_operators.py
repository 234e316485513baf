"""The operators around a fixed-rate key-value cache that rotary positions,
sliding windows and drafted tokens need, as cases that can be timed and checked.

A case is a dict of plain values.  `op` says which operator a pass runs:

  rope    rows of head vectors turned by their positions (one to three axes), or
          the gradient of that with respect to its input
  append  new keys turned by their positions and new values, H D k and H D v per
          head, cast to the cache's format and stored at the slots given, the
          queries turned beside them (MXFP4: keys and values read back)
  window  one query token per sequence over the last `window` tokens of a paged
          cache and its first `sinks`
  tree    up to 64 drafted tokens per sequence, the last ones of a paged cache,
          each attending over the tokens before them and its own ancestors

Formats: int8 and E4M3 with one fp32 scale per head vector, MXFP4 with one
power of two per 32 values.  H is the 128-point Sylvester Hadamard matrix, D the
+-1 diagonal of the plan's seed.  Positions go through a table of cosines and
sines, made in 64 bits.

`run` computes the plain form with elementary torch operations, or, where
`own` is set, makes the library's calls.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
N = 128             # values of a head vector
SEED_K, SEED_V = 41, 51
TOP = {"int8": 127.0, "e4m3": 448.0}


def listed():
    return [
        # the queries of one new token of 16 sequences
        {"name": "rope_step_bf16", "op": "rope", "rows": 16, "heads": 32, "dims": 128, "interleaved": False,
         "axes": 1, "x": "bf16", "out": "bf16", "transposed": False},
        # the patches of a short video: time, height and width, 20 heads
        {"name": "rope_video_bf16", "op": "rope", "rows": 7800, "heads": 20, "dims": 128, "interleaved": True,
         "axes": 3, "x": "bf16", "out": "bf16", "transposed": False},
        # the gradient of a rotation of half of each head, in training
        {"name": "rope_grad_fp32", "op": "rope", "rows": 1999, "heads": 8, "dims": 64, "interleaved": False,
         "axes": 1, "x": "fp32", "out": "fp32", "transposed": True},
        # one new token of 16 sequences: keys and values into the cache, queries for its attention
        {"name": "append_step_int8", "op": "append", "rows": 16, "heads": 8, "group": 4, "dims": 128,
         "interleaved": False, "axes": 1, "fmt": "int8", "block": 128, "x": "bf16"},
        # the tokens of a prefill
        {"name": "append_prompt_e4m3", "op": "append", "rows": 8192, "heads": 8, "group": 4, "dims": 128,
         "interleaved": False, "axes": 1, "fmt": "e4m3", "block": 64, "x": "bf16"},
        # a prompt of text and pictures with positions on three axes, its uneven end padded; keys and values alone
        {"name": "append_axes_mxfp4", "op": "append", "rows": 1999, "heads": 4, "group": 0, "dims": 96,
         "interleaved": False, "axes": 3, "fmt": "mxfp4", "block": 16, "x": "fp32"},
        # the smallest decoding step: a short window of one sequence
        {"name": "window_1x300_e4m3", "op": "window", "batch": 1, "tokens": 5000, "ragged": False, "heads": 8,
         "group": 4, "fmt": "e4m3", "block": 16, "window": 296, "sinks": 4, "q": "bf16", "out": "bf16"},
        # a decoding step of 64 long sequences in a layer that sees 4096 tokens
        {"name": "window_64x4096_int8", "op": "window", "batch": 64, "tokens": 16384, "ragged": False, "heads": 4,
         "group": 4, "fmt": "int8", "block": 128, "window": 4096, "sinks": 0, "q": "bf16", "out": "bf16"},
        # sequences of very uneven length, most of them longer than the window, 7 query heads per KV head
        {"name": "window_ragged_mxfp4", "op": "window", "batch": 24, "tokens": 6001, "ragged": True, "heads": 4,
         "group": 7, "fmt": "mxfp4", "block": 48, "window": 1999, "sinks": 67, "q": "fp32", "out": "fp32"},
        # the smallest check of drafted tokens: seven of one sequence
        {"name": "tree_1x777_e4m3", "op": "tree", "batch": 1, "tokens": 777, "ragged": False, "heads": 8, "group": 4,
         "fmt": "e4m3", "block": 16, "tree": 7, "window": 0, "sinks": 0, "q": "bf16", "out": "bf16"},
        # trees of 64 drafted tokens behind 8192 tokens each
        {"name": "tree_8x8192_int8", "op": "tree", "batch": 8, "tokens": 8192, "ragged": False, "heads": 8,
         "group": 4, "fmt": "int8", "block": 128, "tree": 64, "window": 0, "sinks": 0, "q": "bf16", "out": "bf16"},
        # uneven trees and lengths, an idle sequence among them, 7 query heads per KV head
        {"name": "tree_ragged_mxfp4", "op": "tree", "batch": 24, "tokens": 6001, "ragged": True, "heads": 4,
         "group": 7, "fmt": "mxfp4", "block": 48, "tree": 25, "window": 0, "sinks": 0, "q": "fp32", "out": "fp32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "window", "tree"])
    fmt = rng.choice(["int8", "e4m3", "mxfp4"])
    block = 16 * _log_int(rng, 1, 16)
    types = ["bf16", "fp32"]
    if op in ("rope", "append"):
        turn = {"dims": rng.choice([128, 128, 128, 32, 64, 96]), "interleaved": rng.random() < 0.4,
                "axes": rng.choice([1, 1, 2, 3])}
        if op == "rope":
            heads = rng.choice([1, 3, 8, 16, 20, 32, 40])
            return {"op": op, "rows": _log_int(rng, 1, 180000 // heads), "heads": heads, **turn, "x": rng.choice(types),
                    "out": rng.choice(types), "transposed": rng.random() < 0.3}
        heads, group = rng.choice([1, 2, 4, 5, 8, 8, 16]), rng.choice([0, 1, 4, 4, 7, 8])
        return {"op": op, "rows": _log_int(rng, 1, 65536 // (heads * max(group, 2))), "heads": heads, "group": group,
                **turn, "fmt": fmt, "block": block, "x": rng.choice(types)}
    heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 4, 4, 5, 7, 8, 10, 16])
    io = {"fmt": fmt, "block": block, "q": rng.choice(types), "out": rng.choice(types)}
    sinks = rng.choice([0, 0, 1, 4, 16, rng.randint(5, 300)])
    batch = _log_int(rng, 1, 128)
    if op == "window":
        tokens = _log_int(rng, 1, min(131072, 2097152 // (batch * heads)))
        seen = (1048576 if group <= 4 else 524288) // (batch * heads)  # of a sequence, at most
        return {"op": op, "batch": batch, "tokens": tokens, "ragged": rng.random() < 0.5, "heads": heads, "group": group,
                **io, "window": _log_int(rng, 1, max(1, min(8192, seen - sinks))), "sinks": sinks}
    tree = _log_int(rng, 1, 64)
    most = min(1 << 19, (1 << 27) // (tree * group)) // heads  # tokens of all sequences
    batch = min(batch, max(1, most // (2 * tree)))
    tokens = _log_int(rng, tree, max(tree, min(131072, most // batch)))
    window = rng.choice([0, 0, 0, _log_int(rng, 64, 8192)])
    return {"op": op, "batch": batch, "tokens": tokens, "ragged": rng.random() < 0.5, "heads": heads, "group": group, **io,
            "tree": tree, "window": window, "sinks": sinks if window else 0}


def _lens(case):
    """Tokens of each sequence: all alike, or falling from the longest to an idle one."""
    b, t = case["batch"], case["tokens"]
    if not case["ragged"]:
        return [t] * b
    return [max(0, t * (b - i) // b - 3 * i) if i + 1 < b or b == 1 else 0 for i in range(b)]


def _trees(case):
    """Drafted tokens of each sequence, the last ones of its length."""
    n = case["tree"]
    return [min(t, n if not case["ragged"] else max(0, n - (5 * i) % (n + 1))) for i, t in enumerate(_lens(case))]


def _seen(case, length):
    return length if not case["window"] else min(length, case["window"] + min(case["sinks"], max(0, length - case["window"])))


def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    if case["op"] in ("rope", "append"):
        rows, table = case["rows"], case["rows"] * (4 * case["dims"] + 4 * case["axes"])
        if case["op"] == "rope":
            n = rows * case["heads"]
            return {"bytes": n * N * (_size(case["x"]) + _size(case["out"])) + table, "flops": 3 * n * case["dims"]}
        n, size = rows * case["heads"], _size(case["x"])
        vec = N + 4 if case["fmt"] != "mxfp4" else N // 2 + 4
        back = (2 * N + vec) if case["fmt"] == "mxfp4" else 0  # read back as bf16
        return {"bytes": 2 * n * (N * size + vec + back) + 2 * n * case["group"] * N * size + rows * 8 + table,
                "flops": 2 * n * N * 10 + 3 * n * (1 + case["group"]) * case["dims"]}
    vec = N + 4 if case["fmt"] != "mxfp4" else N // 2 + 4  # bytes of a stored head vector
    hq, lens = case["heads"] * case["group"], _lens(case)
    if case["op"] == "window":
        tokens, rows = sum(_seen(case, n) for n in lens), case["batch"]
        pairs = tokens
    else:
        trees = _trees(case)
        rows = sum(trees)
        tokens = sum(_seen(case, n - d) + d for n, d in zip(lens, trees) if d)
        pairs = sum((_seen(case, n - d) + d) * d for n, d in zip(lens, trees))
    io = rows * hq * N * (_size(case["q"]) + _size(case["out"]))
    return {"bytes": 2 * tokens * case["heads"] * vec + io, "flops": 4 * pairs * hq * N}


# ---------------------------------------------------------------- inputs

def _type(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _signs(seed, cols):
    """The +-1 diagonal D: -1 where bit 63 of the j-th SplitMix64 output is set."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + (np.arange(cols, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return torch.from_numpy(np.where(z >> np.uint64(63), -1.0, 1.0).astype(np.float32)).to(DEV)


def _codes(fmt, blocks, heads, block, gen):
    """A cache's blocks as earlier tokens left them: Gaussian head vectors in the format."""
    shape = (blocks, heads, block)
    if fmt == "mxfp4":
        codes = torch.randint(0, 256, shape + (N // 2,), generator=gen, device=DEV, dtype=torch.uint8)
        return codes, torch.randint(127, 131, shape + (N // 32,), generator=gen, device=DEV, dtype=torch.uint8)
    v = torch.randn(shape + (N,), generator=gen, device=DEV)
    s = 0.2 + 0.1 * torch.rand(shape, generator=gen, device=DEV)
    if fmt == "int8":
        return (v * 45.0).round_().clamp_(-127, 127).to(torch.int8), s
    return (v * 160.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s * (45.0 / 160.0)


def _empty(fmt, blocks, heads, block):
    shape = (blocks, heads, block)
    if fmt == "mxfp4":
        return (torch.zeros(shape + (N // 2,), dtype=torch.uint8, device=DEV),
                torch.zeros(shape + (N // 32,), dtype=torch.uint8, device=DEV))
    return (torch.zeros(shape + (N,), dtype=torch.int8 if fmt == "int8" else torch.uint8, device=DEV),
            torch.zeros(shape, device=DEV))


def _slots(rows, block, blocks, gen):
    """The slots of consecutive tokens whose blocks lie anywhere in the pool; every 50th row is padding."""
    perm = torch.randperm(blocks, generator=gen, device=DEV)
    t = torch.arange(rows, device=DEV)
    slots = perm[t // block] * block + t % block
    return torch.where(t % 50 == 49, torch.full_like(slots, -1), slots)


def _axis(case):
    """The axis of each pair: sections in the order time, height, width, the first a little shorter."""
    pairs, axes = case["dims"] // 2, case["axes"]
    return [min(axes - 1, (i + axes - 1) * axes // (pairs + axes - 1)) for i in range(pairs)]


def _angles(case):
    """(cosines and sines fp32 [positions, 2, pairs], the angles' frequencies fp64)"""
    pairs = case["dims"] // 2
    count = 32768 if case["axes"] == 1 else 2048
    freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / pairs)
    angle = torch.arange(count, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.stack((angle.cos(), angle.sin()), 1).to(torch.float32), freq


def _positions(case, gen):
    """A prompt's consecutive positions from anywhere; of several axes a raster of patches."""
    rows, axes = case["rows"], case["axes"]
    t = torch.arange(rows, device=DEV)
    first = torch.randint(0, 2048 if axes == 1 else 512, (1,), generator=gen, device=DEV)
    if axes == 1:
        return ((t + first) % 32768).to(torch.int32)[:, None].contiguous()
    return torch.stack([first + t // (30 * 52) % 1024, t // 52 % 30, t % 52][:axes], 1).to(torch.int32)


def _masks(trees, gen):
    """Ancestors of each drafted token, itself among them, as bits, [rows]: parents drawn among the tokens before."""
    most = max(trees + [1])
    up = torch.rand((len(trees), most), generator=gen, device=DEV).cpu().numpy()
    rows = []
    for b, n in enumerate(trees):
        bits = []
        for i in range(n):
            parent = int(up[b, i] * (i + 1)) - 1  # -1: the context's last token
            bits.append((1 << i) | (bits[parent] if parent >= 0 else 0))
        rows += bits
    return torch.from_numpy(np.array(rows, dtype=np.uint64).view(np.int64)).to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"case": case, "op": case["op"]}
    heads = case["heads"]
    cols = heads * N
    if case["op"] in ("rope", "append"):
        rows = case["rows"]
        s["table"], _ = _angles(case)
        s["axis"] = _axis(case)
        s["pos"] = _positions(case, gen)
        if own:
            from paper_2606_23406_amd import hq
            s["rope"] = hq.Rope(s["table"], interleaved=case["interleaved"], axis=s["axis"])
    if case["op"] == "rope":
        s["x"] = torch.randn((rows, cols), generator=gen, device=DEV).to(_type(case["x"]))
        s["y"] = torch.empty((rows, cols), dtype=_type(case["out"]), device=DEV)
        s["at"] = torch.tensor(s["axis"], device=DEV)
        return s
    block, fmt = case["block"], case["fmt"]
    s["dk"], s["dv"] = _signs(SEED_K, cols), _signs(SEED_V, cols)
    if case["op"] == "append":
        blocks = -(-rows // block) + 1
        s["at"] = torch.tensor(s["axis"], device=DEV)
        s["slots"] = _slots(rows, block, blocks, gen)
        # keys and values as they come out of one projection, side by side with the queries
        wide = torch.randn((rows, (case["group"] + 2) * cols), generator=gen, device=DEV)
        wide[:, case["group"] * cols + 3:(case["group"] + 1) * cols:N] *= 10  # outlier channels of the keys
        wide = wide.to(_type(case["x"]))
        s["q"], s["k"], s["v"] = wide.split([case["group"] * cols, cols, cols], 1)
        s["qo"] = torch.empty((rows, case["group"] * cols), dtype=wide.dtype, device=DEV)
        s["kc"], s["ks"] = _empty(fmt, blocks, heads, block)
        s["vc"], s["vs"] = _empty(fmt, blocks, heads, block)
        s["ko"] = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
        s["vo"] = torch.empty_like(s["ko"])
    else:
        lens, t = _lens(case), case["tokens"]
        batch, nb = case["batch"], -(-t // block)
        blocks = batch * nb + 1
        s["table"] = torch.randperm(blocks, generator=gen, device=DEV)[:batch * nb].view(batch, nb).to(torch.int32)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["scale"] = N ** -0.5
        s["kc"], s["ks"] = _codes(fmt, blocks, heads, block, gen)
        s["vc"], s["vs"] = _codes(fmt, blocks, heads, block, gen)
        rows = batch
        if case["op"] == "tree":
            trees = _trees(case)
            rows = sum(trees)
            s["masks"] = _masks(trees, gen)
            s["starts"] = torch.tensor(np.concatenate(([0], np.cumsum(trees))), dtype=torch.int32, device=DEV)
        shape = (rows, heads * case["group"], N)
        s["q"] = torch.randn(shape, generator=gen, device=DEV).to(_type(case["q"]))
        s["o"] = torch.empty(shape, dtype=_type(case["out"]), device=DEV)
    if own:
        wide = (cols + 511) // 512 * 512
        s["kp"] = _plan(SEED_K, wide)
        s["vp"] = _plan(SEED_V, wide)
        _handles(s, case, blocks)
    return s


def _plan(seed, cols):
    from paper_2606_23406_amd import hq
    return hq.hq_plan(cols=cols, bps=4.0, rht_seed=seed)


def _handles(s, case, blocks):
    """What a program of the library keeps: the caches, and the attention's workspace."""
    from paper_2606_23406_amd import hq
    form = {"int8": hq.HQ_INT8, "e4m3": hq.HQ_E4M3, "mxfp4": hq.HQ_MXFP4}[case["fmt"]]
    s["kh"] = hq.Cache(s["kp"], blocks, case["block"], form, heads=case["heads"], codes=s["kc"], scales=s["ks"])
    s["vh"] = hq.Cache(s["vp"], blocks, case["block"], form, heads=case["heads"], codes=s["vc"], scales=s["vs"])
    if case["op"] == "append":
        return
    args = (s["kh"], case["batch"], case["heads"] * case["group"], s["table"].shape[1])
    size = (hq.hq_cache_window_workspace_bytes(*args, case["window"], case["sinks"]) if case["op"] == "window" else
            hq.hq_cache_tree_workspace_bytes(*args, case["tree"], case["window"], case["sinks"]))
    s["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------ plain form

def _stage(v, h):
    """One butterfly stage (a, b) -> (a + b, a - b) at distance h along the last axis."""
    p = v.unflatten(-1, (-1, 2, h))
    a, b = p[..., 0, :], p[..., 1, :]
    return torch.stack((a + b, a - b), -2).flatten(-3)


def _hadamard(v):
    return functools.reduce(_stage, (1 << i for i in range(7)), v)


def _turn(s, x, transposed=False):
    """[rows, heads * 128] turned by the rows' positions, [rows, heads, 128] in fp32."""
    c = s["case"]
    d = c["dims"]
    x = x.float().unflatten(1, (-1, N))
    pair = torch.arange(d // 2, device=DEV)
    p = s["pos"].long()[:, s["at"]]  # [rows, pairs]
    cos, sin = s["table"][p, 0, pair][:, None], s["table"][p, 1, pair][:, None]
    if transposed:
        sin = -sin
    if c["interleaved"]:
        a, b = x[..., 0:d:2], x[..., 1:d:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :d // 2], x[..., d // 2:d]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., d:]), -1)


def _over(top, amax):
    return torch.where(amax > 0, torch.full_like(amax, top) / amax, torch.zeros_like(amax))


def _cast(y, fmt):
    """8-bit codes and scales of the head vectors y."""
    top, amax = TOP[fmt], y.abs().amax(-1)
    q = y * _over(top, amax)[..., None]
    codes = (q.round().clamp(-top, top).to(torch.int8) if fmt == "int8"
             else q.clamp(-top, top).to(torch.float8_e4m3fn))
    return codes, amax / torch.full_like(amax, top)


def _mx_cast(y):
    """MXFP4 of y: E2M1 code pairs (the even one in the low nibble) and E8M0 bytes per 32."""
    b = y.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    x = torch.where(amax > 0, torch.frexp(amax)[1] - 3, -127).clamp(-127, 127)
    t = torch.ldexp(b.abs(), -x[..., None])
    code = ((t > 0.25).to(torch.uint8) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0))
    code = (code + 8 * torch.signbit(b).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (x + 127).to(torch.uint8)


def _values(codes, scales, fmt):
    """The values that stored head vectors stand for, in the transformed coordinates."""
    if fmt == "int8":
        return codes.float() * scales[..., None]
    if fmt == "e4m3":
        return codes.view(torch.float8_e4m3fn).float() * scales[..., None]
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return torch.ldexp(v.unflatten(-1, (-1, 32)), scales.int()[..., None] - 127).flatten(-2)


def _put(case, x, d, slots, codes, scales):
    """Head vectors x [rows, heads, 128] into the slots of the rows that have one."""
    live = slots >= 0
    y = _hadamard(x[live] * d.view(-1, N))
    new = _mx_cast(y) if case["fmt"] == "mxfp4" else _cast(y, case["fmt"])
    slots = slots[live]
    at = (slots // case["block"], slice(None), slots % case["block"])
    codes[at] = new[0].view(codes.dtype)
    scales[at] = new[1]


def _get(case, d, slots, codes, scales):
    """The slots' rows as bf16, zeros for a row without one."""
    at = (slots.clamp(min=0) // case["block"], slice(None), slots.clamp(min=0) % case["block"])
    y = _hadamard(_values(codes[at], scales[at], case["fmt"])) / N
    y = (y.flatten(-2) * d).to(torch.bfloat16)
    return torch.where(slots[:, None] >= 0, y, torch.zeros_like(y))


def _gathered(s, t, codes, scales):
    """[batch, heads, tokens, 128] values of tokens t [batch, tokens] of each sequence."""
    bt = s["case"]["block"]
    blk = s["table"].long().gather(1, t // bt)
    v = _values(codes[blk, :, t % bt], scales[blk, :, t % bt], s["case"]["fmt"])
    return v.transpose(1, 2)


def _softmax_sum(s, q, t, live):
    """q [batch, heads, rows, 128] over tokens t [batch, tokens], of which a row sees where live [batch, rows or 1, tokens]."""
    q = _hadamard(q * s["dk"].view(1, -1, 1, N))
    k, v = _gathered(s, t, s["kc"], s["ks"]), _gathered(s, t, s["vc"], s["vs"])
    score = torch.matmul(q, k.transpose(-1, -2)) * (s["scale"] / N)
    score = score.masked_fill(~live[:, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return _hadamard(o) * s["dv"].view(1, -1, 1, N) / N


def _plain_window(s):
    c = s["case"]
    n = s["lens"].long()[:, None]
    j = torch.arange(min(c["sinks"] + c["window"], c["tokens"]), device=DEV)[None]
    low = (n - c["window"]).clamp(min=0)
    sinks = low.clamp(max=c["sinks"])
    t = torch.where(j < sinks, j, low + j - sinks)
    q = s["q"].float().unflatten(1, (-1, c["group"]))  # [batch, heads, group, 128]
    o = _softmax_sum(s, q, t.clamp(max=c["tokens"] - 1), (t < n)[:, None])
    return {"out": o.flatten(1, 2).to(_type(c["out"]))}


def _plain_tree(s):
    c = s["case"]
    g, most = c["group"], c["tree"]
    starts = s["starts"].long()
    n, length = starts.diff()[:, None], s["lens"].long()[:, None]
    i = torch.arange(most, device=DEV)
    row = (starts[:-1, None] + i).clamp(max=max(0, len(s["masks"]) - 1))  # [batch, most]
    mask = s["masks"][row]
    if c["window"]:
        ctx = length - n
        j = torch.arange(min(c["sinks"] + c["window"] + most, c["tokens"]), device=DEV)[None]
        low = (ctx - c["window"]).clamp(min=0)  # no row's window begins before
        sinks = low.clamp(max=c["sinks"])
        t = torch.where(j < sinks, j, low + j - sinks)
        above = (mask[..., None] >> torch.arange(most, device=DEV) & 1).sum(-1)  # ancestors with itself
        near = (t[:, None] >= ctx[..., None] + above[..., None] - c["window"]) | (t[:, None] < c["sinks"])
    else:
        t = torch.arange(c["tokens"], device=DEV).expand(c["batch"], -1)
        near = torch.ones((), dtype=torch.bool, device=DEV)
    at = t - (length - n)  # a drafted token's place in its tree
    bit = (mask[..., None] >> at.clamp(0, 63)[:, None] & 1).bool()  # [batch, most, tokens]
    live = torch.where((at < 0)[:, None], near, bit) & (at < n)[:, None]
    q = s["q"].float()[row].unflatten(2, (-1, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [batch, heads, most * g, 128]
    o = _softmax_sum(s, q, t.clamp(max=c["tokens"] - 1), live.repeat_interleave(g, 1))
    o = o.unflatten(2, (most, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [batch, most, heads_q, 128]
    return {"out": o[i < n].to(_type(c["out"]))}


def _written(s):
    c = s["case"]
    if c["fmt"] == "e4m3":
        return {n: s[n].view(torch.float8_e4m3fn) if n in ("kc", "vc") else s[n] for n in ("kc", "ks", "vc", "vs")}
    return {n: s[n] for n in ("kc", "ks", "vc", "vs")}


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if s["op"] == "rope":
        return {"y": _turn(s, s["x"], c["transposed"]).flatten(1).to(_type(c["out"]))}
    if s["op"] == "window":
        return _plain_window(s)
    if s["op"] == "tree":
        return _plain_tree(s)
    got = {"q": _turn(s, s["q"]).flatten(1).to(s["q"].dtype)} if c["group"] else {}
    _put(c, _turn(s, s["k"]), s["dk"], s["slots"], s["kc"], s["ks"])
    _put(c, s["v"].float().unflatten(1, (-1, N)), s["dv"], s["slots"], s["vc"], s["vs"])
    if c["fmt"] == "mxfp4":
        return {**got, "k": _get(c, s["dk"], s["slots"], s["kc"], s["ks"]), "v": _get(c, s["dv"], s["slots"], s["vc"], s["vs"])}
    return {**got, **_written(s)}


def _run_own(s, c):
    from paper_2606_23406_amd import hq
    if s["op"] == "rope":
        return {"y": hq.hq_rope(s["rope"], s["x"], s["pos"], transposed=c["transposed"], out=s["y"])}
    if s["op"] == "window":
        hq.hq_cache_window_attention(s["kp"], s["kh"], s["vp"], s["vh"], s["q"], s["table"], s["lens"], c["window"],
                                     c["sinks"], scale=s["scale"], out=s["o"], workspace=s["ws"])
        return {"out": s["o"]}
    if s["op"] == "tree":
        hq.hq_cache_tree_attention(s["kp"], s["kh"], s["vp"], s["vh"], s["q"], s["masks"], s["starts"], c["tree"],
                                   s["table"], s["lens"], window=c["window"], sinks=c["sinks"], scale=s["scale"],
                                   out=s["o"], workspace=s["ws"])
        return {"out": s["o"]}
    queries = {"q": s["q"], "q_out": s["qo"]} if c["group"] else {}
    hq.hq_cache_append(s["kp"], s["k"], s["kh"], s["vp"], s["v"], s["vh"], s["slots"], s["rope"], s["pos"], **queries)
    got = {"q": s["qo"]} if c["group"] else {}
    if c["fmt"] == "mxfp4":
        return {**got, "k": hq.hq_cache_read(s["kp"], s["kh"], s["slots"], out=s["ko"]),
                "v": hq.hq_cache_read(s["vp"], s["vh"], s["slots"], out=s["vo"])}
    return {**got, **_written(s)}


# ------------------------------------------------------------- in 64 bits

def _sylvester(n):
    """H itself: entry (i, j) is -1 to the number of bits that i and j share."""
    i = np.arange(n)
    shared = i[:, None] & i[None, :]
    odd = np.zeros((n, n), dtype=np.int64)
    for b in range(n.bit_length()):
        odd ^= (shared >> b) & 1
    return torch.from_numpy(1.0 - 2.0 * odd).to(DEV)


def _nearest(v, grid):
    """The grid value nearest to each of v (grid ascending; the ties' rule does not matter here)."""
    mid = (grid[1:] + grid[:-1]) / 2
    return grid[torch.bucketize(v, mid)]


E4M3_GRID = sorted({m * 2.0 ** e for e in range(-9, 6) for m in range(16) if m * 2.0 ** e <= 448})
E2M1_GRID = [0, .5, 1, 1.5, 2, 3, 4, 6]


def _grid(half):
    return torch.tensor(sorted({-v for v in half} | set(half)), dtype=torch.float64, device=DEV)


def _exact_cast(y, fmt):
    """(codes as the numbers they are, or None; scales; the values they stand for)"""
    if fmt == "mxfp4":
        b = y.unflatten(-1, (-1, 32))
        top = b.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2)
        return None, None, (_nearest((b / scale).clamp(-6, 6), _grid(E2M1_GRID)) * scale).flatten(-2)
    s = y.abs().amax(-1, keepdim=True) / TOP[fmt]
    c = y / torch.where(s > 0, s, torch.ones_like(s))
    c = torch.round(c) if fmt == "int8" else _nearest(c, _grid(E4M3_GRID))
    return (None if fmt == "int8" else c), s[..., 0], c * s


def _exact_values(codes, scales, fmt):
    if fmt == "int8":
        return codes.double() * scales.double()[..., None]
    if fmt == "e4m3":
        c = codes.int()
        e, m = (c >> 3) & 15, (c & 7).double()
        mag = torch.where(e > 0, torch.exp2(e.double() - 10) * (8 + m), 2.0 ** -9 * m)
        return torch.where(c >= 128, -mag, mag) * scales.double()[..., None]
    out = torch.empty(codes.shape[:-1] + (N,), dtype=torch.float64, device=DEV)
    mag = torch.tensor(E2M1_GRID, dtype=torch.float64, device=DEV)
    for half, nib in ((0, codes & 15), (1, codes >> 4)):
        nib = nib.long()
        out[..., half::2] = torch.where(nib >= 8, -1.0, 1.0) * mag[nib & 7]
    return out * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _exact_turn(case, s, x, transposed=False):
    """The rotation as complex factors of the pairs, from the frequencies."""
    d = case["dims"]
    _, freq = _angles(case)
    x = x.double().unflatten(1, (-1, N))
    angle = torch.stack([s["pos"][:, a].double() * freq[i] for i, a in enumerate(s["axis"])], 1)
    turn = torch.polar(torch.ones_like(angle), -angle if transposed else angle)[:, None]
    first = x[..., :d]
    ab = first.unflatten(-1, (-1, 2)) if case["interleaved"] else first.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(ab.contiguous()) * turn)
    z = z if case["interleaved"] else z.transpose(-1, -2)
    return torch.cat((z.flatten(-2), x[..., d:]), -1)


def _exact_append(case, s):
    H, heads, block = _sylvester(N), case["heads"], case["block"]
    got = {}
    if case["group"]:
        got["q"] = _exact_turn(case, s, s["q"]).flatten(1)
    live = s["slots"] >= 0
    blk, off = s["slots"][live] // block, s["slots"][live] % block
    for n, x in (("k", _exact_turn(case, s, s["k"])), ("v", s["v"].double().unflatten(1, (-1, N)))):
        d = s["d" + n].double().view(heads, N)
        codes, scales, values = _exact_cast((x * d) @ H, case["fmt"])
        if case["fmt"] == "mxfp4":
            got[n] = (((values @ H) / N) * d).flatten(1) * live[:, None]
            continue
        pool = torch.zeros(s[n + "s"].shape, dtype=torch.float64, device=DEV)
        pool[blk, :, off] = scales[live]
        got[n + "s"], got[n + "c"] = pool, None
        if codes is not None:
            got[n + "c"] = torch.zeros(s[n + "c"].shape, dtype=torch.float64, device=DEV)
            got[n + "c"][blk, :, off] = codes[live]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return {"y": _exact_turn(case, s, s["x"], case["transposed"]).flatten(1)}
    if case["op"] == "append":
        return _exact_append(case, s)
    H, heads, g = _sylvester(N), case["heads"], case["group"]
    dk, dv = s["dk"].double().view(heads, 1, N), s["dv"].double().view(heads, 1, N)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    trees = _trees(case) if case["op"] == "tree" else [1] * case["batch"]
    first = np.concatenate(([0], np.cumsum(trees)))
    for b, n in enumerate(_lens(case)):
        d = trees[b]
        if n == 0 or d == 0:
            continue
        t = torch.arange(n, device=DEV)
        if case["op"] == "window":
            live = ((t >= n - case["window"]) | (t < case["sinks"]))[None]
        else:
            bits = s["masks"][first[b]:first[b + 1]].cpu().numpy().view(np.uint64)
            up = torch.tensor([[bool(int(m) >> j & 1) for j in range(d)] for m in bits], device=DEV)
            live = torch.ones((d, n), dtype=torch.bool, device=DEV)
            if case["window"]:
                depth = up.sum(1)[:, None]
                live = (t >= n - d + depth - case["window"]) | (t < case["sinks"])
            live[:, n - d:] = up
        t = t[live.any(0)]  # nothing else is looked at
        blk, off = s["table"][b].long()[t // case["block"]], t % case["block"]
        k = _exact_values(s["kc"][blk, :, off], s["ks"][blk, :, off], case["fmt"]).transpose(0, 1)
        v = _exact_values(s["vc"][blk, :, off], s["vs"][blk, :, off], case["fmt"]).transpose(0, 1)
        k = (k @ H) / N * dk
        q = s["q"][first[b]:first[b + 1]].double().view(d, heads, g, N).transpose(0, 1).flatten(1, 2)
        score = s["scale"] * (q @ k.transpose(1, 2).contiguous())
        score = score.masked_fill(~live[:, live.any(0)].repeat_interleave(g, 0), -math.inf)
        o = ((torch.softmax(score, -1) @ v) @ H) / N * dv
        out[first[b]:first[b + 1]] = o.view(heads, d, g, N).transpose(0, 1).flatten(1, 2)
    return {"out": out}
