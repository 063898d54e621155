"""A sealed cache that is not a dict: what it hands out lives until the call has been made."""
import weakref
from collections.abc import Mapping

import pytest
import torch

import paper_2602_00523_b200 as sage
from cache_reference import Batch, dev32
from test_gpu_cache_operators import SCALE, sealed_args

pytestmark = pytest.mark.gpu


class HandsOut(Mapping):
    """New tensors at every look."""

    def __init__(self, tensors):
        self.tensors, self.out = tensors, []

    def __getitem__(self, name):
        t = self.tensors[name].view(self.tensors[name].shape)
        self.out.append(weakref.ref(t))
        return t

    def __iter__(self):
        return iter(self.tensors)

    def __len__(self):
        return len(self.tensors)


class Stream:
    """Asked for its handle last, right ahead of the launch."""

    def __init__(self, cache):
        self.cache, self.alive = cache, None

    @property
    def cuda_stream(self):
        self.alive = [r() is not None for r in self.cache.out]
        return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("which", ["attention", "seal"])
def test_tensors_of_another_mapping_live_until_the_launch(which):
    b = Batch(97, [300], [10], 16, 4)
    args = sealed_args(b, b.seal([4]))
    want = sage.sage_tree_attention_sealed(*args)
    cache = HandsOut(args[4])
    stream = Stream(cache)
    if which == "attention":
        args[4] = cache
        out, ws = torch.empty_like(want), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
        sage.sage_tree_attention_sealed(*args, out=out, ws=ws, stream=stream)
        assert torch.equal(out, want)
    else:
        sage.sage_seal_kv(args[1], args[2], args[3], dev32([300]), dev32([4]), cache, stream=stream)
    assert len(stream.alive) == 5 and all(stream.alive)
    assert not any(r() is not None for r in cache.out)
