"""Workspaces of the attention over sealed pages and with a window: one serves calls of all sizes."""
import pytest
import torch

import paper_2602_00523_b200 as sage
from cache_reference import DIM, Batch
from test_gpu_cache_operators import HALF_BF16, SCALE, clean, host, near, near_sealed, sealed_args, window_args

pytestmark = pytest.mark.gpu


def test_a_workspace_for_the_largest_trees_serves_smaller_ones():
    """Eight sequences, 64 pages each: trees of 64 nodes are not cut, some smaller ones are, into partial results of tens of megabytes."""
    need = {n: sage.sage_tree_attention_sealed_workspace_size(1, 8, 8 * n, 64, 8, DIM, 64) for n in range(1, 65)}
    more = [n for n in need if need[n] > need[64]]
    assert more
    for n in (more[0], more[-1]):
        b = Batch(91, [700, 30, 64, 129, 300, 5, 90, 400], [n] * 8, 64, 8)
        cache = b.seal([l // 64 for l in b.lengths])
        ws = torch.empty(need[64], dtype=torch.uint8, device="cuda")
        st = sage.new_status()
        got = sage.sage_tree_attention_sealed(*sealed_args(b, cache, 64), ws=ws, status=st)
        assert clean(st)
        near_sealed(b, host(got))


@pytest.mark.parametrize("lengths,nodes,heads,layers", [([4000], [60], (64, 8), 1), ([700] * 2, [3, 5], (8, 8), 24), ([500] * 3, [3, 60, 17], (64, 8), 3)])
@pytest.mark.parametrize("share", [0.0, 0.4, 0.9])
def test_any_workspace_of_sixteen_bytes_or_more_will_do(lengths, nodes, heads, layers, share):
    """Less than a launch asks for: what lies behind stays as it was."""
    b = Batch(92, lengths, nodes, *heads, layers)
    args = window_args(b)
    need = sage.sage_tree_attention_window_workspace_size(layers, len(lengths), sum(nodes), *heads, DIM, args[3].shape[1], 10 ** 6, 0)
    room = max(16, int(need * share))
    ws = torch.full((room + 4096,), 77, dtype=torch.uint8, device="cuda")
    st = sage.new_status()
    got = sage.sage_tree_attention_window(*args, 10 ** 6, 0, ws=ws[:room], status=st)
    assert clean(st)
    near(host(got), *b.want(SCALE), HALF_BF16)
    assert (ws[room:] == 77).all()
    for few in (0, 15):
        with pytest.raises(sage.SageError) as e:
            sage.sage_tree_attention_window(*args, 10 ** 6, 0, ws=ws[:few])
        assert e.value.code == sage.SAGE_ERR_WORKSPACE
