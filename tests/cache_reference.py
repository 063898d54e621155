"""Plain 64-bit statements of the operators around the paged cache, and inputs for their tests.  Everything is a numpy array
on the host; nothing is shared with the library."""
import numpy as np
import torch

PAGE, DIM = 64, 128


def bf16(x):
    """Nearest bf16 values of x, as float64."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.float32).to(torch.bfloat16).double().numpy()


def e4m3(x):
    """Nearest e4m3 values (ties to even, cut off at 448): multiples of 2^-9, or of an eighth of the value's binade."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** -6))
    step = np.ldexp(1.0, e - 4)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def exponent(amax):
    """Smallest e in [-60, 60] with amax <= 448 * 2^e (60 where there is none)."""
    for e in range(-60, 61):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return 60


def seal_tile(x):
    """(values, exponent) of a tile: values stand for themselves times 2^exponent."""
    e = exponent(np.abs(x).max())
    return e4m3(x * 2.0 ** -e), e


def rope(x, pos, inv_freq, axis, scale=1.0):
    """x [..., tokens, heads, 128], pos [3, tokens]."""
    out = np.empty_like(x)
    for i in range(64):
        a = pos[axis[i]].astype(np.float64) * inv_freq[i]
        c, s = np.cos(a)[:, None] * scale, np.sin(a)[:, None] * scale
        out[..., i] = x[..., i] * c - x[..., i + 64] * s
        out[..., i + 64] = x[..., i + 64] * c + x[..., i] * s
    return out


def depths(parent):
    d = []
    for p in parent:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def ancestors(parent, i):
    got = {i}
    while parent[i] >= 0:
        i = parent[i]
        got.add(i)
    return got


def visible(parent, L, window=None, sink=0):
    """[nodes, L + nodes] booleans."""
    n, d = len(parent), depths(parent)
    sees = np.zeros((n, L + n), bool)
    for i in range(n):
        mine = ancestors(parent, i)
        for t in range(L + n):
            at = t if t < L else L + d[t - L]
            ok = t < L or (t - L) in mine
            if ok and window is not None:
                ok = L + d[i] - at < window or at < sink
            sees[i, t] = ok
    return sees


def attention(q, k, v, sees, scale):
    """q [n, Hq, d], k and v [Hkv, T, d], sees [n, T].  Returns the outputs and, for tolerances, sum p |v| / sum p."""
    n, hq, d = q.shape
    g = hq // k.shape[0]
    out, size = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    for h in range(hq):
        s = q[:, h] @ k[h // g].T * scale
        s = np.where(sees, s, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h], size[:, h] = p @ v[h // g], p @ np.abs(v[h // g])
    return out, size


def random_tree(rng, n, width=4):
    return [-1] + [int(rng.integers(max(0, i - width), i)) for i in range(1, n)]


class Batch:
    """A batch of sequences with trees: q, and the keys and values of every position, [layer][sequence][head][T][d] in bf16
    values; `table` places bf16 pages in random order, with spare ones that hold NaN (so do rows past a sequence's end)."""

    def __init__(self, seed, lengths, nodes, hq, hkv, layers=1, spread=1.0, first_page=None, capacity=0, parents=None):
        rng = np.random.default_rng(seed)
        self.rng, self.lengths, self.hq, self.hkv, self.layers = rng, list(lengths), hq, hkv, layers
        self.parents = parents or [random_tree(rng, n) for n in nodes]
        self.nodes = [len(p) for p in self.parents]
        self.offsets = np.concatenate([[0], np.cumsum(self.nodes)]).astype(np.int32)
        self.total = int(self.offsets[-1])
        rows = max(self.total, capacity)
        self.q = bf16(rng.standard_normal((layers, rows, hq, DIM)) * spread)
        self.k = [bf16(rng.standard_normal((layers, hkv, l + n, DIM))) for l, n in zip(lengths, self.nodes)]
        self.v = [bf16(rng.standard_normal((layers, hkv, l + n, DIM))) for l, n in zip(lengths, self.nodes)]
        self.parent = np.full(rows, -1, np.int32)
        self.parent[:self.total] = np.concatenate(self.parents)
        self.first = list(first_page) if first_page is not None else [0] * len(self.lengths)
        self.last = [-(-(l + n) // PAGE) for l, n in zip(lengths, self.nodes)]

    def tables(self, first, last, width=None, extra=3):
        need = [z - a for a, z in zip(first, last)]
        pages = sum(need) + extra
        order = self.rng.permutation(pages).astype(np.int32)
        table = np.full((len(need), width or max(1, max(last))), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, first[b]:last[b]] = order[at:at + n]
            at += n
        return table, pages

    def pools(self, width=None):
        """bf16 pools (values) and page table of the pages from `first` on."""
        table, pages = self.tables(self.first, self.last, width)
        got = []
        for x in (self.k, self.v):
            pool = np.full((self.layers, pages, self.hkv, PAGE, DIM), np.nan)
            for b in range(len(self.lengths)):
                for p in range(self.first[b], self.last[b]):
                    rows = x[b][:, :, p * PAGE:(p + 1) * PAGE]
                    pool[:, table[b, p], :, :rows.shape[2]] = rows
            got.append(pool)
        return got[0], got[1], table

    def seal(self, sealed, width=None):
        """The first sealed[b] pages in 8 bits: a host cache (values and exponent bytes), and k, v with what they stand for."""
        table, pages = self.tables([0] * len(sealed), sealed, width)
        cache = {"page_table": table}
        for name, x in (("k", self.k), ("v", self.v)):
            pool = np.full((self.layers, pages, self.hkv, PAGE, DIM), np.nan)
            exps = np.full((self.layers, pages, self.hkv), 127, np.uint8)
            for b, n in enumerate(sealed):
                for p in range(n):
                    for l in range(self.layers):
                        for g in range(self.hkv):
                            y, e = seal_tile(x[b][l, g, p * PAGE:(p + 1) * PAGE])
                            pool[l, table[b, p], g], exps[l, table[b, p], g] = y, e + 127
                            x[b][l, g, p * PAGE:(p + 1) * PAGE] = y * 2.0 ** e
            cache[name], cache[name + "_exp"] = pool, exps
        self.first = list(sealed)
        return cache

    def want(self, scale, window=None, sink=0):
        out, size = np.zeros((self.layers, self.total, self.hq, DIM)), np.zeros((self.layers, self.total, self.hq, DIM))
        for b, L in enumerate(self.lengths):
            sees = visible(self.parents[b], L, window, sink)
            a, z = self.offsets[b], self.offsets[b + 1]
            for l in range(self.layers):
                out[l, a:z], size[l, a:z] = attention(self.q[l, a:z], self.k[b][l], self.v[b][l], sees, scale)
        return out, size


# --- to the device -------------------------------------------------------------------------
def dev16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.float32).to(torch.bfloat16).cuda()


def dev8(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.float32).to(torch.float8_e4m3fn).cuda()


def dev32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def dev_cache(c):
    return {"k": dev8(c["k"]), "v": dev8(c["v"]), "k_exp": torch.from_numpy(c["k_exp"]).cuda(),
            "v_exp": torch.from_numpy(c["v_exp"]).cuda(), "page_table": dev32(c["page_table"])}
