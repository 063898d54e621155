"""The operators around the paged cache where they can go wrong: ways of cutting a launch, scales and scores that spread, values that are
not finite, strides, streams, captured graphs, offsets beyond 32 bits, reported errors, and a run of them as a decode loop uses them."""
import numpy as np
import pytest
import torch

import paper_2602_00523_b200 as sage
from cache_reference import DIM, PAGE, Batch, attention, bf16, depths, dev16, dev32, dev_cache, random_tree, rope, seal_tile, visible
from test_gpu_cache_operators import HALF_BF16, SCALE, SLOP, clean, host, near, near_bf16, near_sealed, sealed_args, window_args

pytestmark = pytest.mark.gpu


# --- ways of cutting a launch: whole items, slices with a merge of their own, slices as a cluster, full waves and a cut rest ---------
CUTS = [
    # lengths, nodes, heads, layers (two blocks fit on each of 148 multiprocessors)
    ([130] * 2, [3, 5], (8, 8), 20),            # 320 items: more than a wave
    ([700] * 2, [3, 5], (8, 8), 24),            # 384 items of 11 pages: a wave whole, 88 items behind it
    ([900] * 3, [9, 9, 9], (16, 8), 13),        # 312 items, 16 behind the wave
    ([500] * 3, [3, 60, 17], (64, 8), 3),       # trees of one to four row tiles in one launch
    ([1700], [12], (8, 1), 1),                  # one item
    ([4000], [2], (8, 1), 1),                   # ... of more pages than slices
    ([260, 1300, 64], [20, 1, 40], (8, 1), 12),
]


@pytest.mark.parametrize("lengths,nodes,heads,layers", CUTS)
def test_cuts_of_sealed_launches(lengths, nodes, heads, layers):
    b = Batch(41, lengths, nodes, *heads, layers)
    cache = b.seal([max(0, l // PAGE - i % 2) for i, l in enumerate(lengths)])
    st = sage.new_status()
    got = sage.sage_tree_attention_sealed(*sealed_args(b, cache), status=st)
    assert clean(st)
    near_sealed(b, host(got))


@pytest.mark.parametrize("lengths,nodes,heads,layers", CUTS)
def test_cuts_of_window_launches(lengths, nodes, heads, layers):
    b = Batch(42, lengths, nodes, *heads, layers)
    st = sage.new_status()
    got = sage.sage_tree_attention_window(*window_args(b), 333, 70, status=st)
    assert clean(st)
    near(host(got), *b.want(SCALE, 333, 70), HALF_BF16)


@pytest.mark.parametrize("width", [7, 40, 700, 6000])
def test_the_width_of_the_page_table_changes_no_more_than_the_cut(width):
    """It is all that the host knows of the lengths: from one slice to many that are empty."""
    b = Batch(43, [400, 130], [9, 30], 16, 4)
    cache = b.seal([6, 1])
    st = sage.new_status()
    got = sage.sage_tree_attention_sealed(*sealed_args(b, cache, width), status=st)
    assert clean(st)
    near_sealed(b, host(got))
    got = sage.sage_tree_attention_window(*window_args(Batch(44, [400, 130], [9, 30], 16, 4), width), 10 ** 6, status=st)
    assert clean(st)
    near(host(got), *Batch(44, [400, 130], [9, 30], 16, 4).want(SCALE), HALF_BF16)


# --- scores and scales ------------------------------------------------------------------------
@pytest.mark.parametrize("spread", [0.0, 1e-3, 6.0, 40.0])
def test_spread_scores(spread):
    """From equal probabilities to one key that takes everything; references move in most steps."""
    b = Batch(45, [1500, 300], [9, 20], 16, 4, spread=spread)
    near(host(sage.sage_tree_attention_window(*window_args(b), 1000, 5)), *b.want(SCALE, 1000, 5), HALF_BF16)
    cache = b.seal([23, 4])
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


@pytest.mark.parametrize("order", ["up", "down"])
def test_scores_that_grow_from_page_to_page(order):
    b = Batch(46, [1200], [6], 8, 2)
    ramp = np.linspace(0.05, 8.0, 1200)[:, None]
    b.k[0][:, :, :1200] = bf16(np.abs(b.k[0][:, :, :1200]) * (ramp if order == "up" else ramp[::-1]))
    b.q = bf16(np.abs(b.q))                     # all scores positive: they grow with the keys
    near(host(sage.sage_tree_attention_window(*window_args(b), 10 ** 6)), *b.want(SCALE), HALF_BF16)
    cache = b.seal([18])
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


def test_scales_of_keys_and_values_differ_from_page_to_page():
    """Exponents of neighbouring pages 2^-6 to 2^6 apart, the largest in the middle of the walk."""
    rng = np.random.default_rng(1)
    b = Batch(47, [1300, 700], [9, 33], 16, 4, 2)
    for i in range(2):
        pages = -(-b.lengths[i] // PAGE)
        for x in (b.k, b.v):
            f = np.repeat(2.0 ** rng.integers(-6, 7, pages), PAGE)[:b.lengths[i]]
            x[i][:, :, :b.lengths[i]] = bf16(x[i][:, :, :b.lengths[i]] * f[:, None])
        b.k[i][:] = bf16(b.k[i] / 30)           # scores of a few units
    cache = b.seal([20, 10])
    assert len(set(cache["v_exp"][0].flatten().tolist())) > 8
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


@pytest.mark.parametrize("size", [1e-15, 1e15])
def test_values_of_any_size(size):
    b = Batch(48, [600], [9], 16, 4)
    b.v[0][:] = bf16(b.v[0] * size)
    cache = b.seal([9])
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


@pytest.mark.parametrize("size", [1e-20, 1e18])
def test_queries_of_any_size(size):
    b = Batch(49, [600], [9], 16, 4)
    b.q = bf16(b.q * size)
    b.k[0][:] = bf16(b.k[0] / size)
    cache = b.seal([9])
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


def test_queries_with_outliers():
    b = Batch(50, [900], [20], 16, 4)
    b.q[..., 5] *= 64
    for k in b.k:
        k[..., 5] /= 64
    b.q, b.k = bf16(b.q), [bf16(k) for k in b.k]
    cache = b.seal([14])
    near_sealed(b, host(sage.sage_tree_attention_sealed(*sealed_args(b, cache))))


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_queries_that_are_not_finite_spoil_their_own_rows_only(bad):
    for which in ("window", "sealed"):
        b = Batch(51, [900, 77], [20, 9], 16, 4)
        q = b.q.copy()
        q[0, 3, 2, 17] = bad                    # node 3 of the first sequence, head 2
        cache = b.seal([14, 1]) if which == "sealed" else None
        b_args = sealed_args(b, cache) if which == "sealed" else window_args(b)
        b_args[0] = dev16(q)
        got = host(sage.sage_tree_attention_sealed(*b_args) if which == "sealed" else sage.sage_tree_attention_window(*b_args, 10 ** 6))
        assert np.isnan(got[0, 3, 2]).all()
        got[0, 3, 2] = b.want(SCALE)[0][0, 3, 2]
        near_sealed(b, got)


# --- rows and memory that are not the call's ----------------------------------------------------
@pytest.mark.parametrize("which", ["window", "sealed"])
def test_rows_behind_the_last_sequence_stay(which):
    b = Batch(52, [300, 200], [10, 7], 64, 8, capacity=64)
    cache = b.seal([4, 3]) if which == "sealed" else None
    args = sealed_args(b, cache) if which == "sealed" else window_args(b)
    args[0][:, 17:] = float("nan")
    out = torch.full_like(args[0], 7.0)
    if which == "sealed":
        sage.sage_tree_attention_sealed(*args, out=out)
        near_sealed(b, host(out)[:, :17])
    else:
        sage.sage_tree_attention_window(*args, 100, 9, out=out)
        near(host(out)[:, :17], *b.want(SCALE, 100, 9), HALF_BF16)
    assert (out[:, 17:] == 7.0).all()


def test_layers_at_a_distance():
    """Pools that are every other layer of larger ones, both forms."""
    b = Batch(53, [300, 90], [10, 7], 16, 4, layers=3)
    args = window_args(b)
    for i in (1, 2):
        wide = torch.full((6,) + args[i].shape[1:], float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[::2] = args[i]
        args[i] = wide[::2]
    near(host(sage.sage_tree_attention_window(*args, 100, 9)), *b.want(SCALE, 100, 9), HALF_BF16)
    cache = b.seal([4, 1])
    args = sealed_args(b, cache)
    for n in ("k", "v"):
        wide = torch.full((6,) + args[4][n].shape[1:], 127, dtype=torch.uint8, device="cuda")
        wide[1::2] = args[4][n].view(torch.uint8)
        args[4][n] = wide[1::2].view(torch.float8_e4m3fn)
    near_sealed(b, host(sage.sage_tree_attention_sealed(*args)))


def test_the_cache_as_bytes_or_as_another_mapping():
    from types import MappingProxyType
    b = Batch(54, [300], [10], 16, 4)
    args = sealed_args(b, b.seal([4]))
    first = sage.sage_tree_attention_sealed(*args)
    args[4] = MappingProxyType({n: t.view(torch.uint8) if n in "kv" else t for n, t in args[4].items()})
    assert torch.equal(first, sage.sage_tree_attention_sealed(*args))
    with pytest.raises(KeyError):
        args[4] = {"k": args[4]["k"]}
        sage.sage_tree_attention_sealed(*args)


def test_offsets_beyond_32_bits():
    """Pools of more than 2^31 elements a layer, the sequence's pages at both ends; appended to, sealed and attended to."""
    pages, hkv = 32768 + 40, 8
    pool = lambda dtype: torch.empty(2, pages, hkv, PAGE, DIM, dtype=dtype, device="cuda")  # noqa: E731
    k, v, k8, v8 = pool(torch.bfloat16), pool(torch.bfloat16), pool(torch.uint8), pool(torch.uint8)
    b = Batch(55, [130], [5], 16, 8, layers=2)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    # the prefix by rope_append without a turn, from every token's own rows
    zero = sage.make_rope_policy(inv_freq=[0.0] * 64)
    rows = lambda x: dev16(np.swapaxes(x[0], 1, 2))  # noqa: E731
    total = 135
    q = torch.zeros(2, total, 16, DIM, dtype=torch.bfloat16, device="cuda")
    st = sage.new_status()
    sage.sage_rope_append(q, rows(b.k), rows(b.v), zero, k, v, table, dev32([0]), dev32([0, total]),
                          pos=torch.zeros(3, total, dtype=torch.int32, device="cuda"), status=st)
    args = [dev16(b.q), k, v, table, dev32([130]), dev32(b.parent), dev32(b.offsets), SCALE]
    near(host(sage.sage_tree_attention_window(*args, 100, 3, status=st)), *b.want(SCALE, 100, 3), HALF_BF16)
    exps = [torch.zeros(2, pages, hkv, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = {"k": k8, "v": v8, "k_exp": exps[0], "v_exp": exps[1],
             "page_table": torch.tensor([[pages - 5, pages - 6]], dtype=torch.int32, device="cuda")}
    sealed = dev32([0])
    sage.sage_seal_kv(k, v, table, dev32([130]), sealed, cache, status=st)
    assert sealed.tolist() == [2]
    b.seal([2])
    table[0, :2] = -1
    got = sage.sage_tree_attention_sealed(dev16(b.q), k, v, table, cache, sealed, dev32([130]), dev32(b.parent), dev32(b.offsets), SCALE, status=st)
    assert clean(st)
    near_sealed(b, host(got))


# --- streams and graphs ------------------------------------------------------------------------
def test_another_stream():
    b = Batch(56, [700], [20], 32, 8)
    cache = b.seal([10])
    w_args, s_args = window_args(Batch(56, [700], [20], 32, 8)), sealed_args(b, cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = sage.sage_tree_attention_window(*w_args, 300, 5), sage.sage_tree_attention_sealed(*s_args)
    with torch.cuda.stream(side):
        inside = sage.sage_tree_attention_window(*w_args, 300, 5), sage.sage_tree_attention_sealed(*s_args)
    given = (sage.sage_tree_attention_window(*w_args, 300, 5, stream=side), sage.sage_tree_attention_sealed(*s_args, stream=side))
    torch.cuda.synchronize()
    for other in (inside, given):
        assert torch.equal(first[0], other[0]) and torch.equal(first[1], other[1])


def test_results_are_the_same_every_time():
    b = Batch(57, [3000, 200, 1000], [9, 60, 33], 64, 8)
    cache = b.seal([46, 3, 15])
    args = sealed_args(b, cache)
    first = sage.sage_tree_attention_sealed(*args)
    for _ in range(20):
        assert torch.equal(first, sage.sage_tree_attention_sealed(*args))


def test_captured_graphs_that_share_a_workspace():
    """Two graphs captured with one workspace, replayed one after the other with new lengths and queries."""
    b = Batch(58, [900, 3000], [9, 30], 32, 8)
    cache = b.seal([14, 46])
    args = sealed_args(b, cache)
    need = sage.sage_tree_attention_sealed_workspace_size(1, 2, 39, 32, 8, DIM, args[3].shape[1])
    ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(args[0]) for _ in range(2)]
    sage.sage_tree_attention_sealed(*args, out=outs[0], ws=ws)          # (attributes are set outside a capture)
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sage.sage_tree_attention_sealed(*args, out=out, ws=ws)
        graphs.append(g)
    graphs[0].replay()
    graphs[1].replay()
    assert torch.equal(outs[0], outs[1])
    near_sealed(b, host(outs[1]))
    args[0].copy_(dev16(bf16(-b.q)))
    b.q = bf16(-b.q)
    graphs[0].replay()
    near_sealed(b, host(outs[0]))


# --- errors --------------------------------------------------------------------------------------
def test_bad_sequences_are_reported_and_leave_the_others():
    for what in ("sealed", "negative", "length", "tree"):
        b = Batch(59, [300, 200, 260], [10, 7, 3], 16, 4)
        cache = b.seal([4, 2, 4])
        args = sealed_args(b, cache)
        if what == "sealed":
            args[5][1] = 4                      # more than 200 positions fill
        elif what == "negative":
            args[5][1] = -1
        elif what == "length":
            args[6][1] = 10 ** 6
        else:
            args[7][10 + 5] = 6                 # a parent behind its child
        st, out = sage.new_status(), torch.zeros_like(args[0])
        sage.sage_tree_attention_sealed(*args, out=out, status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == (sage.SAGE_STATUS_BAD_TREE if what == "tree" else sage.SAGE_STATUS_BAD_PAGE)
        got, (want, size) = host(out), b.want(SCALE)
        keep = [i for i in range(20) if not 10 <= i < 17]
        got[:, 10:17] = want[:, 10:17]
        assert keep and np.isfinite(got).all()
        near_sealed(b, got)


@pytest.mark.parametrize("where", ["bf16", "sealed"])
def test_bad_pages_are_reported(where):
    b = Batch(60, [300, 200], [10, 7], 16, 4)
    args = sealed_args(b, b.seal([4, 2]))
    for bad in (-3, 10 ** 8):
        if where == "bf16":
            args[3][1, 2] = bad
        else:
            args[4]["page_table"][1, 0] = bad
        st = sage.new_status()
        got = sage.sage_tree_attention_sealed(*args, status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == sage.SAGE_STATUS_BAD_PAGE
        want, _ = b.want(SCALE)
        assert np.abs(host(got)[:, :10] - want[:, :10]).max() < 0.1


@pytest.mark.parametrize("layers", [1, 40])
def test_a_wait_that_runs_out_is_reported(layers):
    """The copies are never issued, so the first wait of every other warp runs out; the kernel returns, and the next call is sound."""
    b = Batch(61, [300], [10], 16, 8, layers)
    cache = b.seal([4])
    args = sealed_args(b, cache)
    st = sage.new_status()
    try:
        sage.sage_debug_attention_waits(2_000_000, True)
        sage.sage_tree_attention_sealed(*args, status=st)
        torch.cuda.synchronize()
    finally:
        sage.sage_debug_attention_waits()
    assert int(st.item()) == sage.SAGE_STATUS_TIMEOUT
    st.zero_()
    got = sage.sage_tree_attention_sealed(*args, status=st)
    assert clean(st)
    near_sealed(b, host(got))


def test_python_calls_check_their_tensors():
    b = Batch(62, [300], [10], 16, 4)
    args = sealed_args(b, b.seal([4]))

    def refused(error, at, value, match=None):
        bad = list(args)
        bad[at] = value
        with pytest.raises(error, match=match):
            sage.sage_tree_attention_sealed(*bad)

    refused(ValueError, 0, args[0].float(), "element type")
    refused(ValueError, 0, args[0][:, ::2], "contiguous")
    refused(ValueError, 1, args[1][:, :, :, :, ::2].contiguous(), "head dimension|size")
    refused(ValueError, 1, args[1].transpose(1, 2), "size|gaps")
    refused(ValueError, 3, args[3].long(), "element type")
    refused(ValueError, 5, args[5].repeat(2), "size")
    refused(ValueError, 6, args[6].cpu(), "device tensors")
    refused(ValueError, 7, args[7][:5].contiguous(), "size")
    refused(ValueError, 4, dict(args[4], k_exp=args[4]["k_exp"].int()), "element type")
    refused(ValueError, 4, dict(args[4], v=args[4]["v"][:, :1].contiguous()), "size")
    refused(sage.SageError, 9, 0.0)
    with pytest.raises(sage.SageError) as e:
        sage.sage_tree_attention_window(*window_args(Batch(63, [5000], [60], 64, 8)), 10 ** 6, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.code == sage.SAGE_ERR_WORKSPACE
    with pytest.raises(sage.SageError) as e:
        sage.sage_tree_attention_window(*window_args(b), 0)
    assert e.value.code == sage.SAGE_ERR_INVALID_ARG
    with pytest.raises(OverflowError):
        sage.sage_tree_attention_window(*window_args(b), 2 ** 40)


# --- all of them, as a decode loop uses them ------------------------------------------------------
def test_a_run_of_rounds():
    """Prefill with positions of three axes, then rounds of: the tree's rows get their positions and places, attention over sealed and bf16
    pages, acceptance, compaction, sealing.  The bf16 cache keeps four pages per sequence, used in turn; nothing else holds the prefix."""
    rng = np.random.default_rng(5)
    hq, hkv, layers, batch, ring, rounds = 16, 4, 2, 2, 4, 12
    policy = sage.make_rope_policy(1e6, (16, 24, 24))
    freq, axis = np.array(policy.inv_freq), np.array(policy.axis)
    width = 12
    table = np.array([[b * ring + p % ring for p in range(width)] for b in range(batch)], np.int32)
    k, v = (torch.zeros(layers, batch * ring, hkv, PAGE, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = sage.new_sealed_cache(layers, batch * width, hkv, dev32(rng.permutation(batch * width).reshape(batch, width)))
    sealed, seq_len, st = dev32([0] * batch), dev32([0] * batch), sage.new_status()
    rk, rv = [np.zeros((layers, hkv, 0, DIM)) for _ in range(batch)], [np.zeros((layers, hkv, 0, DIM)) for _ in range(batch)]
    next_pos, tb = [0] * batch, dev32(table)

    def rows(n):
        return (bf16(rng.standard_normal((layers, n, h, DIM))) for h in (hq, hkv, hkv))

    def appended(new, pos, counts, offs, starts):
        """The turned keys as the cache holds them: within a rounding of the reference's own (which roundings fall the other way depends on
        the last bits of 32- and 64-bit products, and what follows is compared with the same keys)."""
        want, pool, got = rope(new, pos, freq, axis), host(k), np.zeros_like(new)
        for b in range(batch):
            for i in range(counts[b]):
                t = starts[b] + i
                got[:, offs[b] + i] = pool[:, table[b, t // PAGE], :, t % PAGE]
        near_bf16(got, want)
        return got

    def round_reference(b):
        """What sealing leaves of the reference's cache: full pages as their 8-bit values."""
        for p in range(ref_sealed[b], rk[b].shape[2] // PAGE):
            for x in (rk[b], rv[b]):
                for l in range(layers):
                    for g in range(hkv):
                        y, e = seal_tile(x[l, g, p * PAGE:(p + 1) * PAGE])
                        x[l, g, p * PAGE:(p + 1) * PAGE] = y * 2.0 ** e
            ref_sealed[b] = p + 1

    ref_sealed = [0] * batch
    # prefill in two chunks, text and a frame
    for counts in ([100, 130], [70, 0]):
        q, nk, nv = rows(sum(counts))
        pos = np.stack([np.concatenate([next_pos[b] + np.arange(c) // d for b, c in enumerate(counts)]) for d in (1, 3, 5)])
        offs = np.concatenate([[0], np.cumsum(counts)])
        got = sage.sage_rope_append(dev16(q), dev16(nk), dev16(nv), policy, k, v, tb, seq_len, dev32(offs), pos=dev32(pos), status=st)
        near_bf16(host(got), rope(q, pos, freq, axis))
        turned = appended(nk, pos, counts, offs, [x.shape[2] for x in rk])
        for b in range(batch):
            rk[b] = np.concatenate([rk[b], np.swapaxes(turned[:, offs[b]:offs[b + 1]], 1, 2)], 2)
            rv[b] = np.concatenate([rv[b], np.swapaxes(nv[:, offs[b]:offs[b + 1]], 1, 2)], 2)
            next_pos[b] += counts[b]
        seq_len += dev32(counts)
        sage.sage_seal_kv(k, v, tb, seq_len, sealed, cache, status=st)
        for b in range(batch):
            round_reference(b)
    for r in range(rounds):
        parents = [random_tree(rng, int(rng.integers(1, 40))) for _ in range(batch)]
        counts = [len(p) for p in parents]
        offs = np.concatenate([[0], np.cumsum(counts)])
        q, nk, nv = rows(sum(counts))
        flat = np.concatenate(parents)
        args = dict(parent=dev32(flat), next_pos=dev32(next_pos))
        tq = sage.sage_rope_append(dev16(q), dev16(nk), dev16(nv), policy, k, v, tb, seq_len, dev32(offs), status=st, **args)
        pos = np.stack([np.concatenate([next_pos[b] + np.array(depths(p)) for b, p in enumerate(parents)])] * 3)
        near_bf16(host(tq), rope(q, pos, freq, axis))
        rq, turned = host(tq), appended(nk, pos, counts, offs, [x.shape[2] for x in rk])
        out = host(sage.sage_tree_attention_sealed(tq, k, v, tb, cache, sealed, seq_len, args["parent"], dev32(offs), SCALE, status=st))
        draft = rng.integers(0, 3, len(flat))
        target = rng.integers(0, 3, len(flat))
        a = sage.sage_accept(args["parent"], dev32(draft), dev32(target), dev32(offs), 9, status=st)
        path, path_len = a["path"].tolist(), a["path_len"].tolist()
        sage.sage_compact_kv(k, v, tb, seq_len, a["path"], a["path_len"], status=st)
        sage.sage_seal_kv(k, v, tb, seq_len, sealed, cache, status=st)
        assert clean(st)
        for b in range(batch):
            L, s = rk[b].shape[2], slice(offs[b], offs[b + 1])
            kk = np.concatenate([rk[b], np.swapaxes(turned[:, s], 1, 2)], 2)
            vv = np.concatenate([rv[b], np.swapaxes(nv[:, s], 1, 2)], 2)
            for l in range(layers):
                want, size = attention(rq[l, s], kk[l], vv[l], visible(parents[b], L), SCALE)
                # (bounds as in near_sealed; no query or key is above 5)
                bound = HALF_BF16 * np.abs(want) + (2.0 ** -7 + 2 * 2.0 ** -17 * 5 * DIM * 5 * SCALE + SLOP) * size + 2.0 ** -23 * 300 * 5
                assert (np.abs(out[l, s] - want) <= bound).all()
            took = L + np.array(path[b][:path_len[b]])
            rk[b], rv[b] = np.concatenate([rk[b], kk[:, :, took]], 2), np.concatenate([rv[b], vv[:, :, took]], 2)
            next_pos[b] += path_len[b]
            round_reference(b)
        assert seq_len.tolist() == [x.shape[2] for x in rk] and sealed.tolist() == [x.shape[2] // PAGE for x in rk]
    assert sum(sealed.tolist()) > 2 + 2         # (a page has been filled and sealed within the rounds)


def test_rope_refuses_to_turn_rows_in_place_that_lie_apart():
    rows = torch.zeros(1, 1, 6, DIM, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(1, 2, 6, DIM, dtype=torch.bfloat16, device="cuda")
    pool, table = torch.zeros(1, 2, 1, PAGE, DIM, dtype=torch.bfloat16, device="cuda"), dev32([[0, 1]])
    args = [sage.make_rope_policy(), pool, pool.clone(), table, dev32([0]), dev32([0, 1])]
    pos = dev32([[1], [1], [1]])
    sage.sage_rope_append(rows[:, :, :4], rows[:, :, 4:5], rows[:, :, 5:], *args, pos=pos)
    with pytest.raises(ValueError, match="contiguous"):
        sage.sage_rope_append(wide[:, :, :4], wide[:, :, 4:5], wide[:, :, 5:], *args, pos=dev32([[1, 1]] * 3), out=wide.view(1, 3, 4, DIM)[:, :2])
    with pytest.raises(ValueError, match="size"):
        sage.sage_rope_append(rows[:, :, :4], rows[:, :, 4:5], rows[:, :, 5:], *args, pos=dev32([[1, 1]] * 3))
    with pytest.raises(sage.SageError):
        sage.sage_rope_append(rows[:, :, :4], rows[:, :, 4:5], rows[:, :, 5:], *args)
    with pytest.raises(sage.SageError):
        sage.sage_rope_append(rows[:, :, :4], rows[:, :, 4:5], rows[:, :, 5:], *args, pos=pos, parent=dev32([-1]), next_pos=dev32([0]))


def test_calls_on_several_streams_at_once():
    """Windowed, sealed and plain tree attention, appending and sealing side by side, each with its own workspace."""
    b = Batch(64, [1500, 200], [20, 9], 32, 8)
    w_args = window_args(b)
    s = Batch(65, [1500, 200], [20, 9], 32, 8)
    s_args = sealed_args(s, s.seal([23, 3]))
    f = Batch(66, [640, 300], [1, 1], 8, 8)
    fk, fv, ft = f.pools()
    pools = [dev16(fk), dev16(fv), dev32(ft), dev32([640, 300])]

    def seal():
        cache = sage.new_sealed_cache(1, 16, 8, dev32(np.arange(20).reshape(2, 10) % 16))
        sage.sage_seal_kv(*pools, dev32([0, 0]), cache)
        return cache["k"].view(torch.uint8)

    calls = [lambda: sage.sage_tree_attention_window(*w_args, 700, 5), lambda: sage.sage_tree_attention_sealed(*s_args),
             lambda: sage.sage_tree_attention(*w_args), seal, lambda: sage.sage_tree_attention_window(*w_args, 10 ** 6)]
    alone = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        got = []
        for c, st in zip(calls, streams):
            with torch.cuda.stream(st):
                got.append(c())
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(alone, got))


def test_scale_bytes_out_of_range_are_read_as_the_nearest():
    b = Batch(67, [300], [3], 8, 2)
    args = sealed_args(b, b.seal([4]))
    out = []
    for low, high in ((67, 187), (0, 255)):
        for name in ("k_exp", "v_exp"):
            args[4][name].fill_(low)
        args[4]["v_exp"][:, args[4]["page_table"][0, 1]] = high
        out.append(sage.sage_tree_attention_sealed(*args))
    assert torch.equal(out[0], out[1]) and torch.isfinite(out[0].float()).all()


def test_rope_trees_of_more_than_64_nodes_are_reported():
    q = torch.ones(1, 70, 4, DIM, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(1, 4, 4, PAGE, DIM, dtype=torch.bfloat16, device="cuda")
    st, out = sage.new_status(), torch.zeros_like(q)
    sage.sage_rope_append(q, q, q, sage.make_rope_policy(), pool, pool.clone(), dev32([[0, 1, 2]]), dev32([5]), dev32([0, 65]),
                          parent=dev32(np.arange(70) - 1), next_pos=dev32([3]), out=out, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == sage.SAGE_STATUS_BAD_TREE and not out.any() and not pool.any()


def test_first_calls_inside_a_capture():
    """In a process of its own, since attributes are set once: nothing that a first call does breaks a capture."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import sys, torch
sys.path[:0] = [%r, %r]
import numpy as np
import paper_2602_00523_b200 as sage
from cache_reference import Batch
from test_gpu_cache_operators import SCALE, host, near_sealed, sealed_args
b = Batch(68, [900], [9], 16, 4)
args = sealed_args(b, b.seal([14]))
out = torch.empty_like(args[0])
need = sage.sage_tree_attention_sealed_workspace_size(1, 1, 9, 16, 4, 128, args[3].shape[1])
ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    sage.sage_tree_attention_sealed(*args, out=out, ws=ws)
g.replay()
torch.cuda.synchronize()
near_sealed(b, host(out))
print("sound")
""" % (root, os.path.join(root, "tests"))
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "sound" in got.stdout, got.stderr[-2000:]


@pytest.mark.parametrize("lengths,heads,layers", [([300, 200], (16, 4), 1), ([4000, 5000], (64, 8), 1), ([700, 700], (8, 8), 24), ([130, 130], (8, 8), 20)])
def test_rows_of_a_reported_sequence_stay_however_the_launch_is_cut(lengths, heads, layers):
    for at, value in ((5, -1), (6, -2)):        # sealed, length
        b = Batch(69, lengths, [10, 7], *heads, layers)
        args = sealed_args(b, b.seal([l // PAGE for l in lengths]))
        args[at][1] = value
        st, out = sage.new_status(), torch.full_like(args[0], 3.0)
        sage.sage_tree_attention_sealed(*args, out=out, status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == sage.SAGE_STATUS_BAD_PAGE
        assert (out[:, 10:] == 3.0).all() and not (out[:, :10] == 3.0).all(-1).any()
