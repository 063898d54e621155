"""Rules that the sources of the kernels around the paged cache keep, where a GPU cannot be made to show them."""
from test_cache_operators_cpu import KERNELS


def test_a_block_that_gives_up_leaves_nothing_in_flight():
    """A wait that runs out in one warp may find the copies of another on their way and products unfinished, whichever warp it is: what is in
    flight is waited for behind the barrier at which all warps have ended, ahead of the tensor memory's release, and nowhere else."""
    body = dict(KERNELS)["tree_attention_paged_kernel"]
    end = body[body.rindex("if (sh->abort)"):]
    assert body[:body.rindex("if (sh->abort)")].rstrip().endswith("__syncthreads();")
    drain, release = end[:end.index("tcgen05.dealloc")], end[end.index("tcgen05.dealloc"):]
    for bar in ("full[", "q_ready", "o_full"):
        assert f"mbar_wait_quiet(&sh->{bar}" in drain
    assert drain.count("__syncthreads();") == 1 and drain.index("__syncthreads();") > drain.rindex("mbar_wait_quiet")
    assert "mbar_wait_quiet" not in body[:body.rindex("if (sh->abort)")] and "mbar_wait_quiet" not in release
