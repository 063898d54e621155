"""Rotary positions with cache append, sealing of pages, attention over sealed pages and with a window, against plain 64-bit
statements of each (cache_reference.py)."""
import numpy as np
import pytest
import torch

import paper_2602_00523_b200 as sage
from cache_reference import DIM, PAGE, Batch, bf16, depths, dev16, dev32, dev_cache, random_tree, rope, seal_tile

pytestmark = pytest.mark.gpu
SCALE = 1.0 / np.sqrt(DIM)
# Half steps of rounding, relative to the value: bf16 2^-8.  What else 32-bit arithmetic adds (scores, exponentials and
# sums of some thousand terms; each a few 2^-22) is far below 2^-12, which stands for all of it.
HALF_BF16, SLOP = 2.0 ** -8, 2.0 ** -12


def clean(status):
    torch.cuda.synchronize()
    return int(status.item()) == 0


def host(t):
    return t.double().cpu().numpy()


# --- rope ------------------------------------------------------------------------------------
def rope_case(seed, counts, lengths, hq, hkv, layers, tree, base=1e6, sections=(16, 24, 24), interleaved=False, far=0, fused=True):
    rng = np.random.default_rng(seed)
    n, batch = sum(counts), len(counts)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = bf16(rng.standard_normal((layers, n, hq + 2 * hkv, DIM)))
    q, k, v = rows[:, :, :hq], rows[:, :, hq:hq + hkv], rows[:, :, hq + hkv:]
    last = [-(-(l + c) // PAGE) for l, c in zip(lengths, counts)]
    pages = sum(last) + 2
    order = rng.permutation(pages)
    table, at = np.full((batch, max(max(last), 1)), -1, np.int32), 0
    for b, z in enumerate(last):
        table[b, :z] = order[at:at + z]
        at += z
    kw, pos = {}, rng.integers(-5, 5000, (3, n)) + far
    if tree:
        parents = [random_tree(rng, c) for c in counts]
        start = rng.integers(0, 4000, batch) + far
        pos = np.stack([np.concatenate([start[b] + np.array(depths(p)) for b, p in enumerate(parents)])] * 3)
        kw = dict(parent=dev32(np.concatenate(parents)), next_pos=dev32(start))
    else:
        kw = dict(pos=dev32(pos))
    pool = bf16(rng.standard_normal((2, layers, pages, hkv, PAGE, DIM)))
    policy = sage.make_rope_policy(base, sections, interleaved=interleaved)
    freq, axis = np.array(policy.inv_freq), np.array(policy.axis)
    wq, wk = rope(q, pos, freq, axis), rope(k, pos, freq, axis)
    wp = pool.copy()
    for b in range(batch):
        for i in range(counts[b]):
            t = lengths[b] + i
            wp[0][:, table[b, t // PAGE], :, t % PAGE] = wk[:, offsets[b] + i]
            wp[1][:, table[b, t // PAGE], :, t % PAGE] = v[:, offsets[b] + i]
    d = dev16(rows)
    dq, dk, dv = d[:, :, :hq], d[:, :, hq:hq + hkv], d[:, :, hq + hkv:]
    if not fused:
        dq, dk, dv = dq.contiguous(), dk.contiguous(), dv.contiguous()
    args = [dq, dk, dv, policy, dev16(pool[0]), dev16(pool[1]), dev32(table), dev32(lengths), dev32(offsets)]
    return args, kw, wq, wp, pool


def near_bf16(got, want):
    # one rounding to bf16 of a 32-bit value that is off by a few 2^-23 of the row's elements (here below 8)
    assert (np.abs(got - want) <= HALF_BF16 * np.abs(want) + 2.0 ** -18).all()


@pytest.mark.parametrize("counts,lengths,hq,hkv,layers,tree", [
    ([1], [0], 8, 8, 1, True), ([1], [63], 8, 1, 2, True), ([10], [2000], 32, 8, 1, True), ([60, 1, 24], [64, 127, 5], 64, 8, 2, True),
    ([64], [100], 28, 7, 3, True), ([1], [0], 4, 2, 1, False), ([130], [0], 16, 8, 1, False), ([70, 0, 200, 3], [61, 9, 64, 0], 64, 8, 2, False),
    ([5], [640], 96, 24, 1, False), ([33] * 40, list(range(40)), 8, 2, 1, False)])
def test_rope_append(counts, lengths, hq, hkv, layers, tree):
    args, kw, wq, wp, pool = rope_case(1, counts, lengths, hq, hkv, layers, tree)
    st = sage.new_status()
    got = sage.sage_rope_append(*args, status=st, **kw)
    assert clean(st)
    near_bf16(host(got), wq)
    gk, gv = host(args[4]), host(args[5])
    near_bf16(gk, wp[0])
    assert (gv == wp[1]).all()
    untouched = (wp[0] == pool[0]).all(-1)
    assert (gk[untouched] == pool[0][untouched]).all()


@pytest.mark.parametrize("far", [10 ** 5, 2 ** 30])
def test_rope_angles_of_far_positions(far):
    """An angle in 32 bits is off by up to 2^-24 of itself: 30 radians at a position of 2^30 and a frequency of 1."""
    args, kw, wq, _, _ = rope_case(2, [9], [30], 8, 2, 1, False, far=far)
    # (the reference's own angle, in 64 bits, is off by 2^-53 of 2^30: 2^-23)
    near = np.abs(host(sage.sage_rope_append(*args, **kw)) - wq)
    assert (near <= HALF_BF16 * np.abs(wq) + 2.0 ** -18).all()


@pytest.mark.parametrize("kw", [dict(sections=(64, 0, 0), base=1e4), dict(sections=(24, 20, 20), interleaved=True), dict(sections=(0, 0, 64))])
def test_rope_policies(kw):
    args, more, wq, _, _ = rope_case(3, [12, 7], [3, 90], 16, 4, 1, False, fused=False, **kw)
    near_bf16(host(sage.sage_rope_append(*args, **more)), wq)


def test_rope_in_place_and_rows_behind_the_last_sequence():
    args, kw, wq, _, _ = rope_case(4, [12, 7], [3, 90], 16, 4, 1, False, fused=False)
    before = args[0].clone()
    args[8] = args[8].clone()
    args[8][2] = 15                               # the second sequence has three tokens, four rows belong to none
    out = sage.sage_rope_append(*args, out=args[0], **kw)
    assert out.data_ptr() == args[0].data_ptr()
    near_bf16(host(out)[:, :15], wq[:, :15])
    assert torch.equal(out[:, 15:], before[:, 15:])


def test_rope_leaves_out_what_does_not_fit():
    args, kw, wq, wp, pool = rope_case(5, [12, 7, 4], [3, 90, 10], 16, 4, 1, False)
    st = sage.new_status()
    args[7][1] = args[6].shape[1] * PAGE - 6      # seven tokens, six places
    args[6][2, 0] = 10 ** 6                       # no such page
    out = torch.zeros(1, 23, 16, DIM, dtype=torch.bfloat16, device="cuda")
    sage.sage_rope_append(*args, out=out, status=st, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == sage.SAGE_STATUS_BAD_PAGE
    near_bf16(host(out)[:, :12], wq[:, :12])
    assert not out[:, 12:19].any()
    first = args[6][0].long().cpu().numpy()
    rest = [p for p in range(pool.shape[2]) if p not in first]
    assert (host(args[4])[:, rest] == pool[0][:, rest]).all()


def test_rope_bad_trees_are_reported():
    args, kw, wq, _, _ = rope_case(6, [12, 7], [3, 90], 16, 4, 1, True)
    kw["parent"][12 + 3] = 5                      # not in front of its child
    st = sage.new_status()
    out = sage.sage_rope_append(*args, status=st, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == sage.SAGE_STATUS_BAD_TREE
    near_bf16(host(out)[:, :12], wq[:, :12])


# --- seal ------------------------------------------------------------------------------------
def seal_case(seed, lengths, before, hkv, layers, spread=None):
    rng = np.random.default_rng(seed)
    batch = len(lengths)
    after = [l // PAGE for l in lengths]
    b = Batch(seed, lengths, [1] * batch, hkv, hkv, layers, first_page=before)
    for x in (b.k, b.v):
        for i in range(batch):
            x[i][:] = bf16(x[i] * (np.exp(rng.standard_normal(x[i].shape[:3] + (1,)) * 2) if spread is None else spread))
    k, v, table = b.pools()
    t8, pages8 = b.tables([0] * batch, after)
    cache = sage.new_sealed_cache(layers, pages8, hkv, dev32(t8))
    return b, after, (dev16(k), dev16(v), dev32(table), dev32(lengths)), cache, t8


@pytest.mark.parametrize("lengths,before,hkv,layers,spread", [
    ([64], [0], 1, 1, None), ([63], [0], 2, 1, None), ([0], [0], 1, 1, None), ([1000, 64, 130, 700], [3, 1, 0, 9], 8, 2, None),
    ([129] * 70, [1, 2, 0] * 23 + [2], 1, 2, None), ([640], [0], 4, 3, 1e-18), ([640], [0], 2, 1, 1e-30), ([256], [1], 2, 1, 1e20),
    ([200], [0], 2, 2, 0.0)])
def test_seal(lengths, before, hkv, layers, spread):
    b, after, args, cache, t8 = seal_case(11, lengths, before, hkv, layers, spread)
    sealed, st = dev32(before), sage.new_status()
    sage.sage_seal_kv(*args, sealed, cache, status=st)
    assert clean(st)
    assert sealed.tolist() == after
    written = np.zeros(cache["k"].shape[1], bool)
    for name, x in (("k", b.k), ("v", b.v)):
        got, exps = host(cache[name]), cache[name + "_exp"].cpu().numpy()
        for i in range(len(lengths)):
            for p in range(before[i], after[i]):
                written[t8[i, p]] = True
                for l in range(layers):
                    for g in range(hkv):
                        y, e = seal_tile(x[i][l, g, p * PAGE:(p + 1) * PAGE])
                        assert exps[l, t8[i, p], g] == e + 127
                        assert (got[l, t8[i, p], g] == y).all()
        assert not got[:, ~written].any() and (exps[:, ~written] == 127).all()


def test_seal_border_values():
    """Largest values on either side of a step of the scale, ties, the smallest numbers, and values that are not finite."""
    b, after, args, cache, t8 = seal_case(12, [640], [0], 1, 1, 1.0)
    x = host(args[0])
    for p, top in enumerate([448.0, 450.0, 3.5, 3.515625, 2.0 ** -52, 448 * 2.0 ** 60, 1e30, 1.0, 1.0]):
        x[0, args[2][0, p].item(), 0, 5, 7] = bf16(top)
    tie = args[2][0, 7].item()
    x[0, tie, 0] = 0
    x[0, tie, 0, 0, :6] = [448.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9]
    strange = args[2][0, 8].item()
    x[0, strange, 0, 0, 0], x[0, strange, 0, 0, 1] = np.nan, np.inf
    sage.sage_seal_kv(dev16(x), *args[1:], dev32([0]), cache)
    got, exps = host(cache["k"]), cache["k_exp"].cpu().numpy()
    for p in range(10):
        if p == 8:
            continue
        y, e = seal_tile(bf16(x[0, args[2][0, p].item(), 0]))
        assert exps[0, t8[0, p], 0] == e + 127 and (got[0, t8[0, p], 0] == y).all()
    assert np.isnan(got[0, t8[0, 8], 0, 0, 0]) and got[0, t8[0, 8], 0, 0, 1] == 448.0


def test_seal_reports_and_leaves_bad_sequences():
    b, after, args, cache, t8 = seal_case(13, [320, 320, 320, 320], [1, 1, 6, 1], 2, 1)
    sealed, st = dev32([1, 1, 6, 1]), sage.new_status()      # the third says more than it has
    args[2][0, 3] = 10 ** 6                                  # no such page of the bf16 cache
    cache["page_table"][1, 2] = -7                           # ... nor of the 8-bit one
    sage.sage_seal_kv(*args, sealed, cache, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == sage.SAGE_STATUS_BAD_PAGE
    assert sealed.tolist() == [1, 1, 6, 5]
    y, e = seal_tile(b.v[3][0, 1, 64:128])
    assert (host(cache["v"])[0, t8[3, 1], 1] == y).all()


# --- attention -------------------------------------------------------------------------------
def near(got, want, size, per_p):
    """per_p: how far a probability may be from its own value, relative; the output is rounded to bf16 once more."""
    assert np.isfinite(got).all()
    over = np.abs(got - want) - (HALF_BF16 * np.abs(want) + (per_p + SLOP) * size)
    assert over.max() <= 0, f"{over.max()} over the bound"


WINDOWED = [
    # lengths, nodes, heads, layers, window, sink
    ([0], [1], (8, 8), 1, 1, 0), ([0], [64], (8, 1), 1, 3, 0), ([1], [1], (8, 8), 1, 1, 1), ([500], [1], (32, 8), 1, 100, 4),
    ([500], [10], (32, 8), 1, 64, 64), ([500], [64], (64, 8), 1, 5, 0), ([500], [64], (64, 8), 1, 5, 3), ([500], [33], (8, 8), 1, 1, 0),
    ([511, 512, 513, 64, 63], [1, 2, 64, 7, 17], (16, 8), 2, 128, 65), ([700], [20], (28, 7), 1, 10 ** 9, 0), ([700], [20], (8, 2), 1, 200, 10 ** 9),
    ([3], [40], (8, 2), 1, 2, 10), ([130, 0, 900, 2], [5, 60, 24, 1], (64, 8), 1, 191, 130), ([1500] * 9, [17] * 9, (8, 1), 1, 640, 1),
    ([6000], [9], (8, 1), 1, 4096, 16)]


def window_args(b, width=None):
    k, v, table = b.pools(width)
    return [dev16(b.q), dev16(k), dev16(v), dev32(table), dev32(b.lengths), dev32(b.parent), dev32(b.offsets), SCALE]


@pytest.mark.parametrize("lengths,nodes,heads,layers,window,sink", WINDOWED)
def test_window_attention(lengths, nodes, heads, layers, window, sink):
    b = Batch(21, lengths, nodes, *heads, layers)
    st = sage.new_status()
    got = sage.sage_tree_attention_window(*window_args(b), window, sink, status=st)
    assert clean(st)
    near(host(got), *b.want(SCALE, window, sink), HALF_BF16)


def test_window_attention_reads_no_page_out_of_sight():
    """Table entries between sinks and window may name nothing, and the pages there may hold NaN."""
    b = Batch(22, [2000, 900], [9, 30], 16, 4)
    args = window_args(b)
    table = args[3]
    table[0, 1:(2000 - 300 + 1) // PAGE] = -1
    table[1, 1:(900 - 300 + 1) // PAGE] = 10 ** 6
    st = sage.new_status()
    got = sage.sage_tree_attention_window(*args, 300, 7, status=st)
    assert clean(st)
    near(host(got), *b.want(SCALE, 300, 7), HALF_BF16)


def test_window_attention_as_wide_as_the_cache_is_tree_attention():
    b = Batch(23, [1200, 77], [30, 60], 64, 8, 2)
    args = window_args(b)
    near(host(sage.sage_tree_attention_window(*args, 10 ** 6, 0)), *b.want(SCALE), HALF_BF16)
    near(host(sage.sage_tree_attention(*args)), *b.want(SCALE), HALF_BF16)


SEALED = [
    # lengths, nodes, heads, layers, sealed pages
    ([0], [1], (8, 8), 1, [0]), ([63], [1], (8, 1), 1, [0]), ([64], [1], (8, 8), 1, [1]), ([65], [64], (64, 8), 1, [1]), ([200], [1], (32, 8), 1, [2]),
    ([500], [10], (32, 8), 1, [7]), ([500], [60], (64, 8), 1, [7]), ([500], [64], (64, 8), 2, [0]), ([511, 512, 513, 64, 63], [1, 2, 64, 7, 17], (16, 8), 2, [7, 8, 3, 0, 0]),
    ([700], [20], (28, 7), 1, [10]), ([130, 0, 900, 2], [5, 60, 24, 1], (64, 8), 1, [2, 0, 14, 0]), ([1500] * 9, [17] * 9, (8, 1), 1, [23] * 9),
    ([6000], [9], (8, 1), 1, [93]), ([6000], [9], (8, 1), 1, [40])]


def sealed_args(b, cache, width=None):
    k, v, table = b.pools(width)
    return [dev16(b.q), dev16(k), dev16(v), dev32(table), dev_cache(cache), dev32(b.first), dev32(b.lengths), dev32(b.parent), dev32(b.offsets),
            SCALE]


def near_sealed(b, got, spread=1.0):
    want, size = b.want(SCALE)
    # Probabilities: an e4m3 number and what is left over as e5m2, 2^-4 and then 2^-3 of the rest.  Queries: off by 2^-17 of the
    # row's largest element at most, so a score by 2^-17 max|q| sum|k| / sqrt(d), and a probability relatively by twice that.
    most_q = np.abs(b.q).max()
    most_k = max(np.abs(k).sum(-1).max() for k in b.k)
    per_p = 2.0 ** -7 + 2 * 2.0 ** -17 * most_q * most_k * SCALE
    # ... and probabilities below the formats' range: half of e5m2's smallest step, 2^-17, against a reference 2^3 below the maximum
    # of the first page and 2^5 below later ones: 2^-20 of the row's largest at most.  Held to 2^-23 here, where a row's maximum is not the first page's.
    floor = 2.0 ** -23 * max(k.shape[2] for k in b.k) * max(np.abs(v).max() for v in b.v)
    assert np.isfinite(got).all()
    over = np.abs(got - want) - (HALF_BF16 * np.abs(want) + (per_p + SLOP) * size + floor)
    assert over.max() <= 0, f"{over.max()} over the bound"


@pytest.mark.parametrize("lengths,nodes,heads,layers,sealed", SEALED)
def test_sealed_attention(lengths, nodes, heads, layers, sealed):
    b = Batch(31, lengths, nodes, *heads, layers)
    cache = b.seal(sealed)
    st = sage.new_status()
    got = sage.sage_tree_attention_sealed(*sealed_args(b, cache), status=st)
    assert clean(st)
    near_sealed(b, host(got))
