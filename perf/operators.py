"""Positions, storage and reach of a paged cache, as cases that can be timed and compared.

Around the tree attention of a decode round stand four calls that these cases time:
  rope    sage_rope_append: rotary positions with three axes (time, height, width) on queries and keys, and the way of
          the keys and values into their places of the paged cache
  seal    sage_seal_kv: pages that have become full move into a cache of 8 bits (e4m3), with a power-of-two scale for
          each page and KV head
  sealed  sage_tree_attention_sealed: tree attention over such a cache; what is not sealed yet is bf16
  window  sage_tree_attention_window: tree attention over a bf16 cache that sees the last `window` positions and the
          first `sink` ones

Where `own` is true, run() makes the calls as a program makes them: outputs and workspaces kept between calls, everything
on the current stream, no host round trip.  Where it is false, the same is computed from elementary torch operations.

Shapes are those of the repository's workloads: 64 query heads over 8 KV heads (a target of 72B parameters) or fewer query
heads per group (a draft-sized model), head dimension 128, pages of 64 tokens, trees of (depth, width, nodes) =
(8, 2, 24), (6, 3, 36), (4, 6, 48), (3, 10, 60), chains, single tokens, up to 64 nodes.
"""
import heapq
import math

import numpy as np
import torch

own = False

HEAD_DIM, PAGE, CAP = 128, 64, 64
TEMPLATES = [(8, 2, 24), (6, 3, 36), (4, 6, 48), (3, 10, 60)]
THETA, SECTIONS = 1.0e6, (16, 24, 24)      # rotary base; frequencies that belong to time, height and width
SCALE_LO, SCALE_HI = -60, 60               # exponents that a sealed page's scale may have
E4M3_MAX = 448.0


def listed():
    return [
        # --- rotary positions and the cache's new rows
        # Smallest call: one layer of a draft's tree of ten nodes; positions follow from the tree.
        dict(name="rope_draft_tree", kind="rope", layers=1, batch=1, trees="4x3x10", tokens=0, ctx=2000, q_heads=32,
             kv_heads=8),
        # One layer of a batch of sixteen trees of 24 to 60 nodes.
        dict(name="rope_serving16", kind="rope", layers=1, batch=16, trees="mix", tokens=0, ctx=1500, q_heads=64, kv_heads=8),
        # One layer of a prefill: a prompt of text and video frames, positions with three axes, rows of a fused projection.
        dict(name="rope_prefill_video", kind="rope", layers=1, batch=1, trees="", tokens=16384, ctx=0, q_heads=64, kv_heads=8),
        # --- full pages into 8 bits
        # A serving round: each of sixteen sequences has filled one page, in all layers.
        dict(name="seal_round", kind="seal", layers=80, batch=16, ctx=500, full=1, kv_heads=8),
        # After a prefill: a video-length prompt of a draft-sized model, all layers.
        dict(name="seal_prefill", kind="seal", layers=28, batch=1, ctx=16384, full=256, kv_heads=8),
        # --- attention over the 8-bit cache
        # Single-token decoding, one layer at 2k positions.
        dict(name="sealed_token_2k", kind="sealed", layers=1, batch=1, ctx_min=2048, ctx_max=2048, trees="0x1x1", q_heads=32,
             kv_heads=8),
        # One layer of the target at a video-length context with the widest template.
        dict(name="sealed_layer_16k", kind="sealed", layers=1, batch=1, ctx_min=16384, ctx_max=16384, trees="3x10x60",
             q_heads=64, kv_heads=8),
        # One layer of batched serving: sixteen ragged sequences, each with its own template.
        dict(name="sealed_serving16", kind="sealed", layers=1, batch=16, ctx_min=1024, ctx_max=8192, trees="mix", q_heads=64,
             kv_heads=8),
        # A chain of nine over a video-length context, all layers of the target in one launch.
        dict(name="sealed_chain_80", kind="sealed", layers=80, batch=1, ctx_min=16384, ctx_max=16384, trees="8x1x9",
             q_heads=64, kv_heads=8),
        # --- attention with a window and sinks
        # A draft's tree of ten nodes far into a video, with the last 1000 positions in sight.
        dict(name="window_draft", kind="window", layers=1, batch=1, ctx_min=16001, ctx_max=16001, trees="4x3x10", q_heads=32,
             kv_heads=8, window=1000, sink=4),
        # One layer of batched serving: 32 ragged sequences, each with its own template.
        dict(name="window_serving32", kind="window", layers=1, batch=32, ctx_min=1024, ctx_max=8192, trees="mix", q_heads=64,
             kv_heads=8, window=2048, sink=64),
        # All layers of a draft-sized model for four chains.
        dict(name="window_chain_28", kind="window", layers=28, batch=4, ctx_min=8000, ctx_max=16384, trees="8x1x9",
             q_heads=32, kv_heads=8, window=4096, sink=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some_tree(rng):
    if rng.random() < 0.2:
        return "0x1x1"
    depth, width = rng.randint(1, 8), rng.randint(1, 10)
    return "%dx%dx%d" % (depth, width, rng.randint(depth + 1, CAP))


HEADS = [(64, 8), (64, 8), (32, 8), (16, 8), (8, 8), (8, 1), (28, 7), (32, 16)]


def draw(rng):
    kind = rng.choice(["rope", "rope", "seal", "sealed", "sealed", "sealed", "window", "window", "window"])
    q_heads, kv_heads = rng.choice(HEADS)
    if kind == "rope":
        if rng.random() < 0.5:
            batch = _log_int(rng, 1, 40)
            layers = rng.choice([1, 1, _log_int(rng, 1, 80)])
            while layers * batch > 200:
                layers = max(1, layers // 2)
            return dict(kind=kind, layers=layers, batch=batch, trees=rng.choice(["mix", _some_tree(rng)]), tokens=0,
                        ctx=_log_int(rng, 1, 4000), q_heads=q_heads, kv_heads=kv_heads)
        batch = rng.choice([1, 1, 2, 5])
        return dict(kind=kind, layers=1, batch=batch, trees="", tokens=_log_int(rng, 20, 16384 // batch),
                    ctx=rng.choice([0, _log_int(rng, 1, 4000)]), q_heads=q_heads, kv_heads=kv_heads)
    if kind == "seal":
        batch, layers = _log_int(rng, 1, 32), _log_int(rng, 1, 80)
        ctx = _log_int(rng, 64, 16384)
        while batch * layers * ctx * kv_heads > 28 * 16384 * 8:
            layers, batch = max(1, layers // 2), (batch if layers > 1 else max(1, batch // 2))
        return dict(kind=kind, layers=layers, batch=batch, ctx=ctx, full=rng.choice([1, ctx // PAGE, rng.randint(1, ctx // PAGE)]),
                    kv_heads=kv_heads)
    batch = rng.choice([1, 1, _log_int(rng, 1, 40)])
    layers = rng.choice([1, 1, 1, _log_int(rng, 1, 80)])
    ctx_max = _log_int(rng, 64, 32768)
    most = 80 * 16384 * 8 if kind == "sealed" else 28 * 4 * 8192 * 8
    while layers * batch * ctx_max * kv_heads > most:                  # no dearer than the largest listed case
        layers, batch = max(1, layers // 2), (batch if layers > 1 else max(1, batch // 2))
    c = dict(kind=kind, layers=layers, batch=batch, ctx_min=ctx_max if batch == 1 else max(16, ctx_max // rng.randint(1, 8)),
             ctx_max=ctx_max, trees="mix" if batch > 1 and rng.random() < 0.5 else _some_tree(rng), q_heads=q_heads,
             kv_heads=kv_heads)
    if kind == "window":
        c.update(window=_log_int(rng, 30, 4096), sink=rng.choice([0, 1, 4, 16, 64, rng.randint(0, 200)]))
    return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _tree(shape):
    """Parents of a "depth x width x nodes" tree: the chain of first candidates down to `depth`, then the likeliest
    further nodes (a candidate of rank r counts 0.6 ** r), level by level."""
    depth, width, nodes = (int(v) for v in shape.split("x"))
    chosen, heap = {(0,) * i: 1.0 for i in range(min(depth, nodes - 1) + 1)}, []

    def offer(path):
        if len(path) < depth:
            for r in range(width):
                if path + (r,) not in chosen:
                    heapq.heappush(heap, (-chosen[path] * 0.6 ** r, path + (r,)))

    for path in list(chosen):
        offer(path)
    while len(chosen) < nodes and heap:
        score, path = heapq.heappop(heap)
        if path not in chosen:
            chosen[path] = -score
            offer(path)
    order = sorted(chosen, key=lambda p: (len(p), p))
    at = {p: i for i, p in enumerate(order)}
    return [-1] + [at[p[:-1]] for p in order[1:]]


def _trees(shape, batch):
    return [_tree("%dx%dx%d" % TEMPLATES[b % 4] if shape == "mix" else shape) for b in range(batch)]


def _depths(parent):
    d = [0]
    for p in parent[1:]:
        d.append(d[p] + 1)
    return d


def _ancestors(parent):
    a = np.eye(len(parent), dtype=bool)
    for i, p in enumerate(parent):
        if p >= 0:
            a[i] |= a[p]
    return a


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _bytes(n):
    return torch.empty(max(16, n), dtype=torch.uint8, device="cuda")


def _offsets(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _lengths(case):
    """Prefix lengths of a batch, spread over [ctx_min, ctx_max], the same for every seed."""
    r = np.random.RandomState(case["batch"] * 7 + case["ctx_max"])
    lens = r.randint(case["ctx_min"], case["ctx_max"] + 1, case["batch"])
    lens[0] = case["ctx_max"]
    return [int(v) for v in lens]


def _counts(case):
    """Tokens per sequence of a rope case, and their trees (None in a prefill)."""
    if case["trees"]:
        trees = _trees(case["trees"], case["batch"])
        return [len(t) for t in trees], trees
    return [max(1, case["tokens"] - 37 * b) for b in range(case["batch"])], None


def _seal_plan(case):
    """(length, pages sealed before, pages sealed after) of every sequence of a seal case."""
    plan = []
    for b in range(case["batch"]):
        length = max(PAGE, case["ctx"] - (11 * b) % 64)
        after = length // PAGE
        plan.append((length, max(0, after - case["full"]), after))
    return plan


def _table(gen, first, last, spare=1.125):
    """Page tables whose entries [first[b], last[b]) name pages in random order, all others none; (table, pages)."""
    need = [z - a for a, z in zip(first, last)]
    pages = max(1, int(math.ceil(sum(need) * spare)))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(need), max(1, max(last))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, first[b]:last[b]] = order[at:at + n]
        at += n
    return table, pages


def _normal(gen, *shape):
    x = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
    for layer in range(shape[0]):
        x[layer].normal_(generator=gen)
    return x


def _visual(pool, table, first, last):
    """The first two fifths of every sequence are visual tokens, of larger magnitude."""
    ids = torch.cat([table[b, first[b]:max(first[b], int(0.4 * last[b]))] for b in range(table.shape[0])]).long()
    for layer in range(pool.shape[0]):
        pool[layer, ids] *= 1.5


def _exponent(amax):
    """Smallest e with amax <= 448 * 2**e, within the exponents that a scale may have."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, SCALE_LO)).clamp(SCALE_LO, SCALE_HI)


def _sealed(tiles):
    """bf16 tiles [..., 64, 128] as (e4m3 values, exponent bytes)."""
    x = tiles.float()
    e = _exponent(x.abs().amax((-2, -1)))
    y = torch.ldexp(x, -e[..., None, None]).clamp(-E4M3_MAX, E4M3_MAX)
    return y.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _video_positions(n, start):
    """[3, n] positions of a prompt: text, then frames of 8 x 12 patches whose time, height and width count from the
    position they begin at, then text that goes on behind the largest."""
    head = min(n, max(1, n // 10))
    body = n - head - min(n - head, n // 10)
    i = np.arange(body)
    grid = np.stack([i // 96, i % 96 // 12, i % 12]) + start + head
    text = start + np.arange(head)
    after = (grid.max() + 1 if body else start + head) + np.arange(n - head - body)
    return np.concatenate([np.stack([text] * 3), grid, np.stack([after] * 3)], axis=1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    return {"rope": _prepare_rope, "seal": _prepare_seal, "sealed": _prepare_attention, "window": _prepare_attention}[case["kind"]](s, case, gen, seed)


def _handles(s, make):
    """What a program keeps between its calls of the library."""
    if own:
        import paper_2602_00523_b200 as sage
        s.update(status=sage.new_status(), **make(sage))
    return s


def _prepare_rope(s, case, gen, seed):
    layers, batch, hq, hkv = case["layers"], case["batch"], case["q_heads"], case["kv_heads"]
    counts, trees = _counts(case)
    n = sum(counts)
    lengths = [case["ctx"] + 13 * b for b in range(batch)]
    last = [-(-(l + c) // PAGE) for l, c in zip(lengths, counts)]
    table, pages = _table(gen, [l // PAGE for l in lengths], last)
    rows = _normal(gen, layers, n, hq + 2 * hkv, HEAD_DIM)            # the rows of a fused projection
    if trees:
        # text positions run ahead of or behind the cache's: a frame has many tokens and few positions
        base = [l // 3 + 5 + seed % 100 for l in lengths]
        depth = [d for t in trees for d in _depths(t)]
        pos = np.stack([np.repeat(base, counts) + depth] * 3)
        s.update(parent=_i32([p for t in trees for p in t]), next_pos=_i32(base))
    else:
        pos = np.concatenate([_video_positions(c, l // 3 + seed % 100) for c, l in zip(counts, lengths)], axis=1)
        s.update(pos=_i32(pos))
    s.update(q=rows[:, :, :hq], k=rows[:, :, hq:hq + hkv], v=rows[:, :, hq + hkv:], table=table, seq_len=_i32(lengths),
             node_offsets=_i32(_offsets(counts)), positions=torch.from_numpy(pos).cuda(),
             k_pool=_normal(gen, layers, pages, hkv, PAGE, HEAD_DIM), v_pool=_normal(gen, layers, pages, hkv, PAGE, HEAD_DIM),
             out=torch.zeros(layers, n, hq, HEAD_DIM, dtype=torch.bfloat16, device="cuda"))
    slot = np.concatenate([l + np.arange(c) for l, c in zip(lengths, counts)])
    s["slot"] = torch.from_numpy(slot).cuda()                          # logical position of every token
    s["owner"] = torch.from_numpy(np.repeat(np.arange(batch), counts)).cuda()
    return _handles(s, lambda sage: {"policy": sage.make_rope_policy(THETA, SECTIONS)})


def _prepare_seal(s, case, gen, seed):
    layers, hkv = case["layers"], case["kv_heads"]
    plan = _seal_plan(case)
    before, after = [p[1] for p in plan], [p[2] for p in plan]
    last = [l // PAGE + 1 for l, _, _ in plan]
    table, pages = _table(gen, before, last)                           # pages sealed earlier have left the bf16 cache
    table8, pages8 = _table(gen, [0] * len(plan), after)
    k, v = _normal(gen, layers, pages, hkv, PAGE, HEAD_DIM), _normal(gen, layers, pages, hkv, PAGE, HEAD_DIM)
    _visual(k, table, before, last)
    pool8 = lambda: torch.zeros(layers, pages8, hkv, PAGE, HEAD_DIM, dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    exps = lambda: torch.full((layers, pages8, hkv), 127, dtype=torch.uint8, device="cuda")  # noqa: E731
    s.update(k_pool=k, v_pool=v, table=table, seq_len=_i32([p[0] for p in plan]), before=_i32(before), sealed=_i32(before),
             cache={"k": pool8(), "v": pool8(), "k_exp": exps(), "v_exp": exps(), "page_table": table8})
    pairs = [(b, p) for b, (_, a, z) in enumerate(plan) for p in range(a, z)]
    s["pairs"] = torch.tensor(pairs, device="cuda").reshape(-1, 2).T
    return _handles(s, lambda sage: {})


def _prepare_attention(s, case, gen, seed):
    layers, batch, hq, hkv = case["layers"], case["batch"], case["q_heads"], case["kv_heads"]
    trees = _trees(case["trees"], batch)
    lengths, counts = _lengths(case), [len(t) for t in trees]
    n, most = sum(counts), max(counts)
    last = [-(-(l + c) // PAGE) for l, c in zip(lengths, counts)]
    first = [l // PAGE for l in lengths] if case["kind"] == "sealed" else [0] * batch
    table, pages = _table(gen, first, last)
    k, v = _normal(gen, layers, pages, hkv, PAGE, HEAD_DIM), _normal(gen, layers, pages, hkv, PAGE, HEAD_DIM)
    if case["kind"] == "sealed":
        table8, pages8 = _table(gen, [0] * batch, first)
        cache = {"page_table": table8}
        for name in ("k", "v"):
            pool = torch.empty(layers, pages8, hkv, PAGE, HEAD_DIM, dtype=torch.float8_e4m3fn, device="cuda")
            exps = torch.empty(layers, pages8, hkv, dtype=torch.uint8, device="cuda")
            for layer in range(layers):
                x = _normal(gen, 1, pages8, hkv, PAGE, HEAD_DIM)
                _visual(x, table8, [0] * batch, first)
                y, e = _sealed(x[0])
                pool[layer].view(torch.uint8).copy_(y.view(torch.uint8))
                exps[layer] = e
            cache[name], cache[name + "_exp"] = pool, exps
        s.update(cache=cache, sealed=_i32(first))
    else:
        _visual(k, table, first, last)
    s.update(q=_normal(gen, layers, n, hq, HEAD_DIM), k_pool=k, v_pool=v, table=table, seq_len=_i32(lengths),
             parent=_i32([p for t in trees for p in t]), node_offsets=_i32(_offsets(counts)),
             out=torch.zeros(layers, n, hq, HEAD_DIM, dtype=torch.bfloat16, device="cuda"))
    # the trees as matrices, and where the nodes of a padded batch lie
    anc, depth = np.zeros((batch, most, most), bool), np.zeros((batch, most), np.int64)
    row, at = np.zeros((batch, most), np.int64), _offsets(counts)
    for b, t in enumerate(trees):
        anc[b, :len(t), :len(t)], depth[b, :len(t)] = _ancestors(t), _depths(t)
        row[b] = at[b] + np.minimum(np.arange(most), len(t) - 1)
    s.update(ancestors=torch.from_numpy(anc).cuda(), depth=torch.from_numpy(depth).cuda(), row=torch.from_numpy(row).cuda(),
             live=torch.from_numpy(np.arange(most)[None] < np.array(counts)[:, None]).cuda(),
             counts=torch.tensor(counts, device="cuda"))

    def make(sage):
        if case["kind"] == "sealed":
            return {"ws": _bytes(sage.sage_tree_attention_sealed_workspace_size(layers, batch, n, hq, hkv, HEAD_DIM, table.shape[1]))}
        return {"ws": _bytes(sage.sage_tree_attention_window_workspace_size(layers, batch, n, hq, hkv, HEAD_DIM, table.shape[1],
                                                                            case["window"], case["sink"]))}
    return _handles(s, make)


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rope": _own_rope, "seal": _own_seal, "sealed": _own_sealed, "window": _own_window}[kind](s)
    return {"rope": _plain_rope, "seal": _plain_seal, "sealed": _plain_sealed, "window": _plain_window}[kind](s)


def _own_rope(s):
    import paper_2602_00523_b200 as sage
    sage.sage_rope_append(s["q"], s["k"], s["v"], s["policy"], s["k_pool"], s["v_pool"], s["table"], s["seq_len"],
                          s["node_offsets"], pos=s.get("pos"), parent=s.get("parent"), next_pos=s.get("next_pos"),
                          out=s["out"], status=s["status"])
    return [s["out"], s["k_pool"], s["v_pool"]]


def _own_seal(s):
    import paper_2602_00523_b200 as sage
    s["sealed"].copy_(s["before"])                        # every pass starts from the same pages
    sage.sage_seal_kv(s["k_pool"], s["v_pool"], s["table"], s["seq_len"], s["sealed"], s["cache"], status=s["status"])
    return [s["sealed"], s["cache"]]


def _own_sealed(s):
    import paper_2602_00523_b200 as sage
    return sage.sage_tree_attention_sealed(s["q"], s["k_pool"], s["v_pool"], s["table"], s["cache"], s["sealed"], s["seq_len"],
                                           s["parent"], s["node_offsets"], 1.0 / math.sqrt(HEAD_DIM), out=s["out"],
                                           ws=s["ws"], status=s["status"])


def _own_window(s):
    import paper_2602_00523_b200 as sage
    c = s["case"]
    return sage.sage_tree_attention_window(s["q"], s["k_pool"], s["v_pool"], s["table"], s["seq_len"], s["parent"],
                                           s["node_offsets"], 1.0 / math.sqrt(HEAD_DIM), c["window"], c["sink"],
                                           out=s["out"], ws=s["ws"], status=s["status"])


def _plain_rope(s):
    # angles in 64 bits: in 32 a position of a few thousand leaves the first frequencies 2^-12 of a turn off
    half = HEAD_DIM // 2
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(SECTIONS, device="cuda"))
    freq = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = s["positions"][axis].T.double() * freq                     # [tokens, 64]
    cos, sin = angle.cos().float()[None, :, None], angle.sin().float()[None, :, None]
    turn = lambda x: torch.cat([x[..., :half] * cos - x[..., half:] * sin, x[..., half:] * cos + x[..., :half] * sin], -1)  # noqa: E731
    s["out"].copy_(turn(s["q"].float()))
    page, slot = s["table"][s["owner"], s["slot"] // PAGE].long(), s["slot"] % PAGE
    s["k_pool"][:, page, :, slot] = turn(s["k"].float()).to(torch.bfloat16).transpose(0, 1)
    s["v_pool"][:, page, :, slot] = s["v"].transpose(0, 1)
    return [s["out"], s["k_pool"], s["v_pool"]]


def _plain_seal(s):
    b, p = s["pairs"]
    src, dst, cache = s["table"][b, p].long(), s["cache"]["page_table"][b, p].long(), s["cache"]
    k, ke = _sealed(s["k_pool"][:, src])
    v, ve = _sealed(s["v_pool"][:, src])
    cache["k"].view(torch.uint8)[:, dst] = k.view(torch.uint8)
    cache["v"].view(torch.uint8)[:, dst] = v.view(torch.uint8)
    cache["k_exp"][:, dst], cache["v_exp"][:, dst] = ke, ve
    s["sealed"].copy_(s["seq_len"] // PAGE)
    return [s["sealed"], cache]


def _gathered(pool, table):
    """Rows of a sequence in logical order, in 32 bits: [layers, batch, kv heads, positions, head dim]."""
    x = pool[:, table.long().clamp(min=0)].float()                     # [layers, batch, pages, heads, slots, dim]
    return x.transpose(2, 3).flatten(3, 4)


def _unsealed(s, name, table):
    """The same from the 8-bit cache where pages are sealed, from the bf16 one behind them."""
    cache, ids = s["cache"], s["cache"]["page_table"].long().clamp(min=0)
    # (an index of 8-bit floats goes by their bytes)
    x8 = cache[name].view(torch.uint8)[:, ids].view(torch.float8_e4m3fn).float()
    x8 = torch.ldexp(x8, cache[name + "_exp"][:, ids].int()[..., None, None] - 127)
    x8 = x8.transpose(2, 3).flatten(3, 4)
    x = _gathered(s[name + "_pool"], table)
    x8 = torch.nn.functional.pad(x8, (0, 0, 0, x.shape[3] - x8.shape[3]))
    at = torch.arange(x.shape[3], device="cuda")
    return torch.where((at < PAGE * s["sealed"][:, None])[None, :, None, :, None], x8, x)


def _attend(s, k, v, window, sink):
    c = s["case"]
    hq, hkv = c["q_heads"], c["kv_heads"]
    length, depth = s["seq_len"].long(), s["depth"]
    t = torch.arange(k.shape[3], device="cuda")
    slot = t[None] - length[:, None]                                   # tree slot of a key, below 0 in the prefix
    inside = slot.clamp(0, depth.shape[1] - 1)
    node = torch.gather(s["ancestors"], 2, inside[:, None].expand(-1, depth.shape[1], -1))
    sees = torch.where(slot[:, None] < 0, torch.ones_like(node), node & (slot < s["counts"][:, None])[:, None])
    at = torch.where(slot < 0, t[None], length[:, None] + torch.gather(depth, 1, inside))     # a key's position
    if window:
        sees &= ((length[:, None] + depth)[:, :, None] - at[:, None] < window) | (at < sink)[:, None]
    q = s["q"][:, s["row"]].float().unflatten(3, (hkv, hq // hkv))     # [layers, batch, nodes, kv heads, group, dim]
    q = q.permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    x = (q @ k.transpose(3, 4)).mul_(1.0 / math.sqrt(HEAD_DIM)).unflatten(3, (-1, hq // hkv))
    x.masked_fill_(~sees[None, :, None, :, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    x /= x.sum(-1, keepdim=True)
    y = (x.flatten(3, 4) @ v).unflatten(3, (-1, hq // hkv)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    s["out"][:, s["row"][s["live"]]] = y[:, s["live"]].to(torch.bfloat16)
    return s["out"]


def _plain_sealed(s):
    return _attend(s, _unsealed(s, "k", s["table"]), _unsealed(s, "v", s["table"]), 0, 0)


def _plain_window(s):
    return _attend(s, _gathered(s["k_pool"], s["table"]), _gathered(s["v_pool"], s["table"]), s["case"]["window"], s["case"]["sink"])


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    row = HEAD_DIM * 2.0                                               # bytes of a bf16 row
    layers, hkv = case["layers"], case["kv_heads"]
    if case["kind"] == "rope":
        n = sum(_counts(case)[0])
        return {"bytes": layers * n * row * (2 * case["q_heads"] + 4 * hkv), "flops": layers * n * HEAD_DIM * 3.0 * (case["q_heads"] + hkv)}
    if case["kind"] == "seal":
        pages = sum(z - a for _, a, z in _seal_plan(case))
        return {"bytes": 2 * layers * hkv * pages * (PAGE * row * 1.5 + 1), "flops": 2.0 * layers * hkv * pages * PAGE * HEAD_DIM * 3}
    lengths, trees = _lengths(case), _trees(case["trees"], case["batch"])
    kv, flops = 0.0, 0.0
    for l, t in zip(lengths, trees):
        n, pages = len(t), l // PAGE
        if case["kind"] == "sealed":
            kv += 2 * hkv * (pages * (PAGE * row / 2 + 1) + (l - pages * PAGE + n) * row)
            seen = n * (l + 1) + sum(_depths(t))
        else:
            w, sink = case["window"], case["sink"]
            kv += 2 * hkv * row * (min(sink, max(0, l - w + 1)) + min(l, w - 1) + n)
            seen = sum(min(l + d + 1, w + min(sink, max(0, l + d + 1 - w))) for d in _depths(t))
        kv += 2 * n * case["q_heads"] * row
        flops += 4.0 * seen * case["q_heads"] * HEAD_DIM
    return {"bytes": layers * kv, "flops": layers * flops}


# ---------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits, one sequence after the other
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "seal": _exact_seal, "sealed": _exact_attention, "window": _exact_attention}[case["kind"]](s)


def _exact_rope(s):
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    out, kp, vp = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), s["k_pool"].double(), s["v_pool"].double()
    turned = []
    for x in (q, k):
        y = torch.empty_like(x)
        for i in range(64):
            axis = 0 if i < SECTIONS[0] else 1 if i < SECTIONS[0] + SECTIONS[1] else 2
            a = s["positions"][axis].double() * THETA ** (-i / 64.0)
            c, d = torch.cos(a)[None, :, None], torch.sin(a)[None, :, None]
            y[..., i] = x[..., i] * c - x[..., i + 64] * d
            y[..., i + 64] = x[..., i + 64] * c + x[..., i] * d
        turned.append(y)
    out.copy_(turned[0])
    table, start = s["table"].tolist(), s["node_offsets"].tolist()
    for b, length in enumerate(s["seq_len"].tolist()):
        n = start[b + 1] - start[b]
        at = torch.arange(length, length + n, device="cuda")
        page = torch.tensor(table[b], device="cuda")[at // PAGE]
        kp[:, page, :, at % PAGE] = turned[1][:, start[b]:start[b + 1]].transpose(0, 1)
        vp[:, page, :, at % PAGE] = v[:, start[b]:start[b + 1]].transpose(0, 1)
    return [out, kp, vp]


def _exact_seal(s):
    """Every 8-bit value is the nearest multiple of its own step, ties to the even one."""
    cache = {"k": torch.zeros(s["cache"]["k"].shape, device="cuda"), "v": torch.zeros(s["cache"]["v"].shape, device="cuda"),
             "k_exp": None, "v_exp": None, "page_table": None}         # (whole numbers are compared with the other form's)
    t16, t8, before, length = s["table"].tolist(), s["cache"]["page_table"].tolist(), s["before"].tolist(), s["seq_len"].tolist()
    for b in range(len(length)):
        for p in range(before[b], length[b] // PAGE):
            for name in ("k", "v"):
                x = s[name + "_pool"][:, t16[b][p]].double()
                top = x.abs().flatten(2).amax(2).clamp(min=2.0 ** -200)
                scale = 2.0 ** torch.ceil(torch.log2(top / E4M3_MAX) + 0.5)
                for _ in range(2):                                     # down to the smallest that serves (a logarithm may be a step off)
                    scale = torch.where(top <= E4M3_MAX * scale / 2, scale / 2, scale)
                y = x / scale.clamp(2.0 ** SCALE_LO, 2.0 ** SCALE_HI)[..., None, None]
                step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
                cache[name][:, t8[b][p]] = (torch.round(y / step) * step).float()
    return [None, cache]


def _exact_attention(s):
    c = s["case"]
    hq, hkv, sealed = c["q_heads"], c["kv_heads"], c["kind"] == "sealed"
    group = hq // hkv
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    start, table = s["node_offsets"].tolist(), s["table"].tolist()
    parents, lengths = s["parent"].tolist(), s["seq_len"].tolist()
    done = s["sealed"].tolist() if sealed else [0] * len(lengths)
    table8 = s["cache"]["page_table"].tolist() if sealed else None
    for b, length in enumerate(lengths):
        parent = parents[start[b]:start[b + 1]]
        n = len(parent)
        position = [length + d for d in _depths(parent)]
        sees = torch.zeros(n, length + n, dtype=torch.bool)
        for i in range(n):
            sees[i, :length] = True
            j = i
            while j >= 0:
                sees[i, length + j] = True
                j = parent[j]
            if not sealed:
                key = torch.tensor(list(range(length)) + position)
                sees[i] &= (position[i] - key < c["window"]) | (key < c["sink"])
        sees = sees.cuda().repeat_interleave(group, 0)
        for layer in range(c["layers"]):
            kv = []
            for name in ("k", "v"):
                rows = []
                if done[b]:
                    ids = torch.tensor(table8[b][:done[b]], device="cuda")
                    x = s["cache"][name][layer].view(torch.uint8)[ids].view(torch.float8_e4m3fn).to(torch.float64)
                    rows.append(x * 2.0 ** (s["cache"][name + "_exp"][layer][ids].double() - 127)[..., None, None])
                ids = torch.tensor(table[b][done[b]:-(-(length + n) // PAGE)], device="cuda")
                rows.append(s[name + "_pool"][layer][ids].double())
                kv.append(torch.cat(rows).transpose(0, 1).flatten(1, 2)[:, :length + n])
            q = s["q"][layer, start[b]:start[b + 1]].double().unflatten(1, (hkv, group)).transpose(0, 1).flatten(1, 2)
            x = (q @ kv[0].transpose(1, 2)) / math.sqrt(HEAD_DIM)
            p = torch.softmax(x.masked_fill(~sees, -math.inf), -1)
            y = (p @ kv[1]).unflatten(1, (n, group)).transpose(0, 1).flatten(1, 2)
            out[layer, start[b]:start[b + 1]] = y
    return out
