"""The tree decoding example (examples/tree_decode.py): the tree speculation operators run together."""
import importlib.util
import os

import numpy as np
import pytest

import synth
from conftest import ROOT
from oracle.model import Transformer

pytestmark = pytest.mark.gpu

LENGTHS = (150, 1, 37)
MODELS = synth.scaled(synth.TINY, batch=len(LENGTHS), prompt_len=max(LENGTHS))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def start(example, widths, **kw):
    torch = example.torch
    d = example.build(MODELS, widths, slots=512, **kw)
    d.prefill(torch.from_numpy(synth.prompts(MODELS)).cuda(), torch.tensor(LENGTHS, dtype=torch.int32, device="cuda"))
    return d


def decode(d, n):
    """(the first n tokens of each sequence, the tokens of each step)."""
    out, taken = [[] for _ in LENGTHS], []
    while min(map(len, out)) < n:
        emitted, m = d.step()
        taken.append(m.tolist())
        for o, e, k in zip(out, emitted.tolist(), taken[-1]):
            assert all(x >= 0 for x in e[:k]) and all(x == -1 for x in e[k:])
            o += e[:k]
    assert int(d.status) == 0
    assert d.lens.tolist() == [l - 1 + sum(t[b] for t in taken) for b, l in enumerate(LENGTHS)]
    return [o[:n] for o in out], taken


@pytest.mark.parametrize("cache", ["float8_e4m3fn", "bfloat16"])
def test_greedy_trees_give_the_plain_decoding(example, cache):
    """At temperature 0 a tree changes how many tokens a step gives, not which."""
    kw = dict(temperature=0.0, cache_dtype=getattr(example.torch, cache))
    plain, taken = decode(start(example, (), **kw), 32)
    assert all(t == [1] * len(LENGTHS) for t in taken)
    assert decode(start(example, (3, 2, 1), **kw), 32)[0] == plain
    mine, taken = decode(start(example, (2, 1, 1, 1), self_draft=True, **kw), 32)
    assert mine == plain
    assert np.mean(taken) > 4.5                # the target's own best tokens: paths of 5 nodes


def test_sampled_trees_run(example):
    a = decode(start(example, (3, 2, 1), temperature=0.7, seed=5), 16)
    b = decode(start(example, (3, 2, 1), temperature=0.7, seed=5), 16)
    assert a == b
    assert all(0 <= x < MODELS.target.vocab for o in a[0] for x in o)


def test_logits_against_the_oracle(example):
    """fp32 models over a bf16 cache: K and V are rounded by 2^-9 of themselves at most, which reaches the logits through
    two layers' attention, each one of the four parts of the residual; 2^-6 of their norm is eight times one rounding."""
    torch = example.torch
    d = start(example, (), cache_dtype=torch.bfloat16)
    got = d.target.forward(d.tokens, d.lens, d.depth, d.mask).cpu().numpy()[:, 0]
    model = Transformer(MODELS.target, synth.model_weights(MODELS, "target"))
    for b, n in enumerate(LENGTHS):
        want = model.forward_full(synth.prompts(MODELS)[b, :n])[0][-1]
        assert np.linalg.norm(got[b] - want) < 2.0 ** -6 * np.linalg.norm(want)
