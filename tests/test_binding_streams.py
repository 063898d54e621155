"""What a call allocates itself belongs to the stream that it goes to."""
import contextlib

import numpy as np
import pytest
import torch

import paper_2602_00523_b200 as sage
from paper_2602_00523_b200 import binding
from cache_reference import Batch, bf16, dev32, dev_cache


class Native:
    """Stands for the marshalling: says which outputs are missing, notes what it is given, launches nothing."""

    def __init__(self):
        self.given = []

    def __getattr__(self, name):
        def call(*args):
            self.given += [a for a in args if isinstance(a, torch.Tensor)]
            for a in args:
                if isinstance(a, dict):
                    if not a:
                        return None
                    self.given += a.values()
            return 0
        return call


def calls(device):
    """One call of every function that allocates, with nothing of its own passed in."""
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
    q, pool = torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16, device=device), torch.zeros(1, 3, 8, 64, 128, dtype=torch.bfloat16, device=device)
    cache = sage.new_sealed_cache(1, 3, 8, i(1, 2))
    logits, alpha = torch.zeros(4, 512, device=device), torch.zeros(4, device=device)
    policy = sage.make_policy([0.3, 0.5, 0.7])
    return {
        "sage_expand_topk": lambda s: sage.sage_expand_topk(logits, 4, 4, parent=i(4), rank=i(4), node_offsets=i(2), root_token=i(1), stream=s),
        "sage_select_tree": lambda s: sage.sage_select_tree(alpha, policy, handover=True, stream=s),
        "sage_build_ancestor_mask": lambda s: sage.sage_build_ancestor_mask(i(4), i(2), stream=s),
        "sage_tree_attention": lambda s: sage.sage_tree_attention(q, pool, pool, i(1, 2), i(1), i(4), i(2), 0.1, stream=s),
        "sage_tree_attention_window": lambda s: sage.sage_tree_attention_window(q, pool, pool, i(1, 2), i(1), i(4), i(2), 0.1, 5, 1, stream=s),
        "sage_tree_attention_sealed": lambda s: sage.sage_tree_attention_sealed(q, pool, pool, i(1, 2), cache, i(1), i(1), i(4), i(2), 0.1, stream=s),
        "sage_rope_append": lambda s: sage.sage_rope_append(q, q, q, sage.make_rope_policy(), pool, pool, i(1, 2), i(1), i(2), pos=i(3, 4), stream=s),
        "sage_accept": lambda s: sage.sage_accept(i(4), i(4), i(4), i(2), 4, stream=s),
    }


@pytest.mark.parametrize("name", list(calls("cpu")))
def test_allocations_are_made_under_the_stream_that_is_given(name, monkeypatch):
    call, native, under, side, inside, outside = calls("cpu")[name], Native(), [], object(), [], []

    @contextlib.contextmanager
    def stream(s):
        under.append(s)
        yield
        under.pop()

    for f in ("empty", "empty_like", "zeros", "full"):
        real = getattr(torch, f)

        def made(*a, _real=real, **kw):
            t = _real(*a, **kw)
            (inside if under == [side] else outside).append(t)
            return t
        monkeypatch.setattr(torch, f, made)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "Stream", object)
    monkeypatch.setattr(binding, "_native", native)
    call(side)
    mine = [t for t in inside if any(t is g for g in native.given)]
    assert mine and len(mine) == len(inside)
    inside.clear(), outside.clear(), native.given.clear()
    call(None)
    assert not inside and outside


def owner(t):
    """The stream whose memory a tensor lies in."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


@pytest.mark.gpu
def test_outputs_and_workspaces_lie_in_the_memory_of_the_stream(monkeypatch):
    """... and come out right when the current stream is given new memory of the same sizes, and fills it, while they run."""
    b = Batch(81, [3000], [60], 64, 8)
    k, v, table = b.pools()
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()  # noqa: E731
    args = [up(b.q), up(k), up(v), dev32(table), dev32(b.lengths), dev32(b.parent), dev32(b.offsets), 0.09]
    s = Batch(82, [3000], [60], 64, 8)
    cache = dev_cache(s.seal([46]))
    k, v, table = s.pools()
    s_args = [up(bf16(s.q)), up(k), up(v), dev32(table), cache, dev32(s.first), dev32(s.lengths), dev32(s.parent), dev32(s.offsets), 0.09]
    for call, a in ((sage.sage_tree_attention, args), (lambda *x, **kw: sage.sage_tree_attention_window(*x, 2000, 3, **kw), args),
                    (sage.sage_tree_attention_sealed, s_args)):
        want = call(*a)
        torch.cuda.synchronize()
        seen, real = [], torch.empty
        monkeypatch.setattr(torch, "empty", lambda *x, **kw: seen.append(real(*x, **kw)) or seen[-1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(*a, stream=side)
        monkeypatch.undo()
        sizes = [t.numel() for t in seen]
        assert sizes and {owner(t) for t in seen + [got]} == {side.cuda_stream}
        seen.clear()
        for n in sizes + [got.numel() * 2]:
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


class Handle:
    """A stream of another library: no more than its handle."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.gpu
def test_streams_that_are_not_torch_s():
    parent, offsets = torch.tensor([-1, 0, 0, 1], dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (torch.cuda.default_stream(), side):
        got = sage.sage_build_ancestor_mask(parent, offsets, stream=Handle(stream))
        torch.cuda.synchronize()
        assert owner(got) == stream.cuda_stream and got.tolist() == [1, 3, 5, 11]
