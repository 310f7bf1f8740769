"""The tree decoding example over 4-bit caches: rotary positions, write, attention, validation and commit run together."""
import pytest

from test_gpu_tree_decode import LENGTHS, decode, example, start  # noqa: F401

pytestmark = pytest.mark.gpu


def test_greedy_trees_give_the_plain_decoding(example):
    """At temperature 0 a tree changes how many tokens a step gives, not which."""
    kw = dict(temperature=0.0, cache_dtype=example.torch.uint8)
    plain, taken = decode(start(example, (), **kw), 32)
    assert all(t == [1] * len(LENGTHS) for t in taken)
    assert decode(start(example, (3, 2, 1), **kw), 32)[0] == plain
    mine, taken = decode(start(example, (2, 1, 1, 1), self_draft=True, **kw), 32)
    assert mine == plain
    assert sum(map(sum, taken)) > 4.5 * len(taken) * len(LENGTHS)   # the target's own best tokens: paths of 5 nodes
