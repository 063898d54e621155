"""Blocks that read more than 32 pages: page ids and scales are looked up 32 at a time, the next ones ahead.  The pools are small and
their pages used many times over, in another order by every sequence, with scales that differ from page to page."""
import numpy as np
import pytest

import paper_2602_00523_b200 as sage
from cache_reference import DIM, PAGE, attention, bf16, dev16, dev32, dev_cache, e4m3, random_tree, visible
from test_gpu_cache_operators import HALF_BF16, SCALE, SLOP, clean, host

pytestmark = pytest.mark.gpu
POOL = 150


def walk(seed, lengths, sealed, hkv, g=1):
    """Pools, tables and arguments; keys(b) and values(b) of sequence b as float64 [hkv, T, d]."""
    rng = np.random.default_rng(seed)
    batch = len(lengths)
    parents = [random_tree(rng, int(rng.integers(1, 9))) for _ in lengths]
    offsets = np.concatenate([[0], np.cumsum([len(p) for p in parents])]).astype(np.int32)
    k, v = (bf16(rng.standard_normal((1, POOL, hkv, PAGE, DIM))) for _ in range(2))
    width = max(-(-(l + len(p)) // PAGE) for l, p in zip(lengths, parents))
    table, table8 = rng.integers(0, POOL, (2, batch, width)).astype(np.int32)
    cache = {"page_table": table8}
    for name, spread in (("k", 2), ("v", 6)):
        cache[name] = e4m3(rng.standard_normal((1, POOL, hkv, PAGE, DIM)) * 64)
        cache[name + "_exp"] = (121 + rng.integers(-spread, spread + 1, (1, POOL, hkv))).astype(np.uint8)
    q = bf16(rng.standard_normal((1, int(offsets[-1]), hkv * g, DIM)) * 0.5)

    def rows(pool, name, b):
        got = []
        for p in range(-(-(lengths[b] + len(parents[b])) // PAGE)):
            if sealed is not None and p < sealed[b]:
                at = table8[b, p]
                got.append(cache[name][0, at] * 2.0 ** (cache[name + "_exp"][0, at].astype(float) - 127)[:, None, None])
            else:
                got.append(pool[0, table[b, p]])
        return np.concatenate(got, 1)[:, :lengths[b] + len(parents[b])]

    args = [dev16(q), dev16(k), dev16(v), dev32(table)]
    tail = [dev32(lengths), dev32(np.concatenate(parents)), dev32(offsets), SCALE]
    return q, parents, offsets, lambda b: rows(k, "k", b), lambda b: rows(v, "v", b), cache, args, tail


def compare(got, q, parents, offsets, lengths, keys, values, which, window=None, sink=0):
    most_q = np.abs(q).max()
    for b in which:
        s = slice(offsets[b], offsets[b + 1])
        kk, vv = keys(b), values(b)
        want, size = attention(q[0, s], kk, vv, visible(parents[b], lengths[b], window, sink), SCALE)
        # probabilities: off by 2^-8 of their value, sealed or not, and by what the split of the queries does to the scores
        per_p = HALF_BF16 + 2 * 2.0 ** -17 * most_q * np.abs(kk).sum(-1).max() * SCALE
        floor = 2.0 ** -27 * kk.shape[1] * np.abs(vv).max() * 2.0 ** 12        # (value scales lie up to 2^12 apart)
        assert np.isfinite(got[0, s]).all()
        assert (np.abs(got[0, s] - want) <= HALF_BF16 * np.abs(want) + (per_p + SLOP) * size + floor).all()
        # in the norm: the output's own rounding is 2^-8 / sqrt(3) in the mean of squares, probabilities that all err one way 2^-8
        off = np.linalg.norm(got[0, s] - want, axis=(0, 2)) / np.linalg.norm(want, axis=(0, 2))
        assert off.max() <= 1.2 * 2.0 ** -8


RNG = np.random.default_rng(3)
LAUNCHES = [
    # 320 items and more, left whole but for what does not fill a wave: 70 to 100 pages each
    ([int(x) for x in RNG.integers(70 * 64, 100 * 64, 40)], 8, 1),
    ([int(x) for x in RNG.integers(40 * 64, 72 * 64, 38)], 8, 4),
    # one sequence in slices of more than 32 pages
    ([70001], 8, 1),
]


@pytest.mark.parametrize("lengths,hkv,g", LAUNCHES)
@pytest.mark.parametrize("bf16_pages", [0, 3, 37])
def test_long_walks_over_sealed_pages(lengths, hkv, g, bf16_pages):
    """bf16_pages: how many full ones are not sealed, so that the sealed pages' batches of 32 begin elsewhere than the walk's."""
    sealed = [l // PAGE - (bf16_pages + i % 2 if bf16_pages else 0) for i, l in enumerate(lengths)]
    q, parents, offsets, keys, values, cache, args, tail = walk(101, lengths, sealed, hkv, g)
    st = sage.new_status()
    got = sage.sage_tree_attention_sealed(*args, dev_cache(cache), dev32(sealed), *tail, status=st)
    assert clean(st)
    compare(host(got), q, parents, offsets, lengths, keys, values, sorted({0, 1, len(lengths) // 2, len(lengths) - 1} & set(range(len(lengths)))))


@pytest.mark.parametrize("lengths,hkv,g", LAUNCHES)
def test_long_walks_in_a_window(lengths, hkv, g):
    q, parents, offsets, keys, values, cache, args, tail = walk(102, lengths, None, hkv, g)
    window = max(lengths) - 3 * PAGE if len(lengths) > 1 else 60000
    st = sage.new_status()
    got = sage.sage_tree_attention_window(*args, *tail, window, 70, status=st)
    assert clean(st)
    compare(host(got), q, parents, offsets, lengths, keys, values, sorted({0, 1, len(lengths) // 2, len(lengths) - 1} & set(range(len(lengths)))), window, 70)
