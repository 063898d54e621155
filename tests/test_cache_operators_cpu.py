"""The operators around the paged cache without a GPU: what they refuse, their host arithmetic, and the rules that their kernels'
sources keep."""
import ctypes
import glob
import os
import re

import numpy as np
import pytest
import torch

import paper_2602_00523_b200 as sage
from cache_reference import e4m3, exponent, rope, visible

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_00523_b200", "csrc", "cache")
WAIT = "after_previous_kernel();"
FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: the calls below fail validation first
LAYER = 16 * 8 * 64 * 128               # elements of a layer of 16 pages and 8 heads


def kernels():
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\([^)]*\)\s*)?(\w+)\s*\(", text):
            at = text.index("{", m.end())
            depth, end = 1, at + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
            found.append((m.group(1), text[at:end]))
    return found


KERNELS = kernels()


def test_all_kernels_are_found():
    assert {"rope_append_kernel", "seal_pages_kernel", "count_sealed_kernel", "tree_attention_paged_kernel"} <= {n for n, _ in KERNELS}


@pytest.mark.parametrize("name,body", KERNELS, ids=[n for n, _ in KERNELS])
def test_kernels_wait_for_the_one_in_front(name, body):
    """Each is launched while the kernel before it still runs: none ends, reads global memory or holds tensor memory before it has waited."""
    assert body.count(WAIT) == 1
    ahead = body[:body.index(WAIT)]
    assert not re.search(r"\breturn\b", ahead)
    assert not re.search(r"p\.\w+\s*\[|node_offsets|seq_len|page_table|part_|range_of|atomic|report_status|tcgen05", ahead)


# --- refusals at the C entry points ---------------------------------------------------------
def cache_struct(**kw):
    c = sage.SageSealedCache(FAKE, FAKE, LAYER, FAKE, FAKE, 16, FAKE, 4)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def refusals(call, args, changes):
    for at, value, code in changes:
        bad = list(args)
        for i, v in zip(at, value) if isinstance(at, tuple) else [(at, value)]:
            bad[i] = v
        assert call(*bad) == code, (at, value)


INVALID, UNSUPPORTED, WORKSPACE = sage.SAGE_ERR_INVALID_ARG, sage.SAGE_ERR_UNSUPPORTED, sage.SAGE_ERR_WORKSPACE


def test_window_attention_refuses():
    #       q     k     v     stride  nl pages table width len  parent offs  b  n  hq hk d    p   scale win sink out  ws    bytes
    args = [FAKE, FAKE, FAKE, LAYER, 1, 16, FAKE, 4, FAKE, FAKE, FAKE, 1, 8, 8, 8, 128, 64, 0.1, 100, 4, FAKE, FAKE, 1 << 30, None, None]
    refusals(sage.lib().sage_tree_attention_window, args, [
        (0, None, INVALID), (1, None, INVALID), (2, None, INVALID), (6, None, INVALID), (8, None, INVALID), (9, None, INVALID),
        (10, None, INVALID), (20, None, INVALID), (4, 0, INVALID), (5, 0, INVALID), (7, 0, INVALID), (11, -1, INVALID), (12, 0, INVALID),
        (17, 0.0, INVALID), (17, float("nan"), INVALID), (18, 0, INVALID), (18, -5, INVALID), (19, -1, INVALID), (3, LAYER + 4, INVALID),
        (0, ctypes.c_void_p(0x1008), INVALID), (15, 64, UNSUPPORTED), (16, 16, UNSUPPORTED), ((13, 14), (6, 2), UNSUPPORTED),
        ((13, 14), (7, 2), UNSUPPORTED), ((3, 4), (LAYER - 8, 2), INVALID), (21, None, WORKSPACE), (22, 8, WORKSPACE), (7, 1 << 25, UNSUPPORTED)])
    ok = list(args)
    ok[11] = 0
    assert sage.lib().sage_tree_attention_window(*ok) == sage.SAGE_OK


def test_sealed_attention_refuses():
    ref = ctypes.byref(cache_struct())
    #       q     k     v     stride  nl pages table width cache sealed len   parent offs  b  n  hq hk d    p   scale out   ws    bytes
    args = [FAKE, FAKE, FAKE, LAYER, 1, 16, FAKE, 4, ref, FAKE, FAKE, FAKE, FAKE, 1, 8, 8, 8, 128, 64, 0.1, FAKE, FAKE, 1 << 30, None, None]
    changes = [(i, None, INVALID) for i in (0, 1, 2, 6, 8, 9, 10, 11, 12, 20)]
    changes += [(19, -1.0, INVALID), (17, 64, UNSUPPORTED), (18, 32, UNSUPPORTED), ((15, 16), (6, 2), UNSUPPORTED), (21, None, WORKSPACE), (22, 8, WORKSPACE)]
    for kw, code in [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k_exp=None), INVALID), (dict(v_exp=None), INVALID),
                     (dict(page_table=None), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages_per_seq=0), INVALID),
                     (dict(layer_stride=-16), INVALID), (dict(layer_stride=LAYER + 8), INVALID), (dict(k=ctypes.c_void_p(0x1004)), INVALID),
                     (dict(max_pages_per_seq=1 << 25), UNSUPPORTED)]:
        changes.append((8, ctypes.byref(cache_struct(**kw)), code))
    changes.append(((4, 8), (2, ctypes.byref(cache_struct(layer_stride=LAYER - 16))), INVALID))
    refusals(sage.lib().sage_tree_attention_sealed, args, changes)
    ok = list(args)
    ok[13] = 0
    assert sage.lib().sage_tree_attention_sealed(*ok) == sage.SAGE_OK


def test_seal_refuses():
    ref = ctypes.byref(cache_struct())
    #       k     v     stride nl pages table width len  cache sealed b hk d    p
    args = [FAKE, FAKE, LAYER, 1, 16, FAKE, 4, FAKE, ref, FAKE, 1, 8, 128, 64, None, None]
    changes = [(i, None, INVALID) for i in (0, 1, 5, 7, 8, 9)]
    changes += [(10, -1, INVALID), (11, 0, INVALID), (12, 64, UNSUPPORTED), (13, 128, UNSUPPORTED), ((2, 3), (LAYER - 8, 2), INVALID),
                (8, ctypes.byref(cache_struct(k=None)), INVALID), (8, ctypes.byref(cache_struct(layer_stride=8)), INVALID)]
    refusals(sage.lib().sage_seal_kv, args, changes)
    ok = list(args)
    ok[10] = 0
    assert sage.lib().sage_seal_kv(*ok) == sage.SAGE_OK


def test_rope_refuses():
    def rows(**kw):
        r = sage.SageRopeRows(FAKE, FAKE, FAKE, 1024, 128, 1024, 128, 1024, 128)
        for name, value in kw.items():
            setattr(r, name, value)
        return ctypes.byref(r)

    def policy(**kw):
        p = sage.make_rope_policy()
        for name, value in kw.items():
            getattr(p, name)[3] = value
        return ctypes.byref(p)

    #       rows    policy    nl n  hq hk d   pos   parent next  out   k     v     stride pages p  table width len  offs  b
    args = [rows(), policy(), 1, 8, 8, 8, 128, FAKE, None, None, FAKE, FAKE, FAKE, LAYER, 16, 64, FAKE, 4, FAKE, FAKE, 1, None, None]
    refusals(sage.lib().sage_rope_append, args, [
        (0, None, INVALID), (1, None, INVALID), (0, rows(k=None), INVALID), (0, rows(q_token_stride=132), INVALID), (0, rows(v_layer_stride=-8), INVALID),
        (7, None, INVALID), (8, FAKE, INVALID), ((7, 8), (None, FAKE), INVALID), ((7, 9), (None, FAKE), INVALID), (10, None, INVALID),
        (11, None, INVALID), (16, None, INVALID), (18, None, INVALID), (19, None, INVALID), (6, 64, UNSUPPORTED), (15, 16, UNSUPPORTED),
        (1, policy(axis=3), INVALID), (1, policy(inv_freq=float("nan")), INVALID), (1, policy(inv_freq=1e300), INVALID), (20, -1, INVALID),
        ((2, 13), (2, LAYER - 8), INVALID)])
    for at, value in ((20, 0), (3, 0)):
        ok = list(args)
        ok[at] = value
        assert sage.lib().sage_rope_append(*ok) == sage.SAGE_OK


def test_workspace_queries():
    w = sage.sage_tree_attention_window_workspace_size
    assert w(1, 1, 60, 64, 8, 128, 257, 1000, 4) >= 16
    assert w(1, 1, 60, 64, 8, 128, 257, 2 ** 40, 2 ** 40) >= 16
    for bad in [(0, 1, 60, 64, 8, 128, 257, 1000, 4), (1, 1, 60, 64, 7, 128, 257, 1000, 4), (1, 1, 60, 64, 8, 128, 257, 0, 4), (1, 1, 60, 64, 8, 128, 257, 9, -1)]:
        assert w(*bad) == 0
    s = sage.sage_tree_attention_sealed_workspace_size
    assert s(1, 1, 60, 64, 8, 128, 257) >= 60 * 64 * 130 * 4 and s(1, 0, 60, 64, 8, 128, 257) == 0


# --- refusals of the Python calls ---------------------------------------------------------
def test_python_calls_want_device_tensors():
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    i = lambda *shape: z(*shape, dtype=torch.int32)  # noqa: E731
    q, pool, ws = z(1, 4, 8, 128), z(1, 3, 8, 64, 128), z(16, dtype=torch.uint8)
    cache = sage.new_sealed_cache(1, 3, 8, i(1, 2))
    assert cache["k"].dtype == torch.float8_e4m3fn and cache["k"].shape == (1, 3, 8, 64, 128) and cache["v_exp"].shape == (1, 3, 8)
    with pytest.raises(ValueError, match="device tensors only"):
        sage.sage_tree_attention_window(q, pool, pool, i(1, 2), i(1), i(4), i(2), 0.1, 5, 1, ws=ws)
    with pytest.raises(ValueError, match="device tensors only"):
        sage.sage_tree_attention_sealed(q, pool, pool, i(1, 2), cache, i(1), i(1), i(4), i(2), 0.1, ws=ws)
    with pytest.raises(ValueError, match="device tensors only"):
        sage.sage_seal_kv(pool, pool, i(1, 2), i(1), i(1), cache)
    with pytest.raises(ValueError, match="device tensors only"):
        sage.sage_rope_append(q, q, q, sage.make_rope_policy(), pool, pool, i(1, 2), i(1), i(2), pos=i(3, 4))


def test_rope_policy():
    p = sage.make_rope_policy(1e6, (16, 24, 24))
    assert np.allclose(p.inv_freq, 1e6 ** (-np.arange(64) / 64.0), rtol=1e-15)
    assert list(p.axis) == [0] * 16 + [1] * 24 + [2] * 24 and p.scale == 1.0
    mixed = list(sage.make_rope_policy(1e6, (24, 20, 20), interleaved=True).axis)
    assert mixed[:7] == [0, 1, 2, 0, 1, 2, 0] and [mixed.count(a) for a in range(3)] == [24, 20, 20] and mixed[60:] == [0] * 4
    for bad in [(16, 24), (16, 24, 25), (-1, 32, 33)]:
        with pytest.raises(ValueError):
            sage.make_rope_policy(1e6, bad)
    with pytest.raises(ValueError):
        sage.make_rope_policy(inv_freq=[1.0] * 63)


# --- the reference itself ------------------------------------------------------------------
def test_reference_rounds_to_e4m3_as_the_type_does():
    x = np.concatenate([np.linspace(-448, 448, 4001), np.logspace(-4, 2.6, 4001), [2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875]])
    x = torch.from_numpy(x).float()
    assert (torch.from_numpy(e4m3(x.double().numpy())).float() == x.to(torch.float8_e4m3fn).float()).all()


def test_reference_exponents():
    assert [exponent(v) for v in (448.0, 448.1, 224.0, 3.5, 3.51, 0.0, 1e30)] == [0, 1, -1, -7, -6, -60, 60]


def test_reference_rotation_is_a_rotation():
    """Scores depend on differences of positions only, and lengths stay."""
    rng = np.random.default_rng(0)
    p = sage.make_rope_policy(1e6, (16, 24, 24))
    q, k = rng.standard_normal((2, 1, 1, 128))
    at = lambda x, t: rope(x, np.array([[t], [2 * t], [3 * t]]), np.array(p.inv_freq), np.array(p.axis))  # noqa: E731
    assert abs((at(q, 7) * at(k, 3)).sum() - (at(q, 107) * at(k, 103)).sum()) < 1e-9
    assert abs((at(q, 7) ** 2).sum() - (q ** 2).sum()) < 1e-9


def test_reference_window():
    sees = visible([-1, 0, 0, 1], 5, window=3, sink=1)
    # node 3 (depth 2, position 7) sees position 5 on, its ancestors 0, 1 and itself, and the sink
    assert sees[3].tolist() == [True, False, False, False, False, True, True, False, True]
    assert sees[0].tolist() == [True, False, False, True, True, True, False, False, False]
