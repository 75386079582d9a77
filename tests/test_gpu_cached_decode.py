"""examples/cached_decode.py: the cache and attention calls with drafting and verification, as one loop."""
import importlib.util
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "cached_decode.py")
    spec = importlib.util.spec_from_file_location("cached_decode", path)
    m = importlib.util.module_from_spec(spec)
    sys.modules["cached_decode"] = m
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_drafts_change_no_token(lib, example, cache):
    """The same tokens with and without drafts, in fewer steps with; the log probabilities are those of the
    tokens that came out."""
    shape = example.Shape(cache=cache)
    g = torch.Generator("cuda").manual_seed(1)
    prompt = torch.randint(0, shape.vocab, (3, 40), generator=g, device="cuda", dtype=torch.int32)
    prompt = torch.cat((prompt, prompt[:, :20]), 1)
    got = {}
    for draft in (False, True):
        model = example.Decoder(shape, 3, example.context_of(60, 32, shape))
        got[draft] = model.decode(prompt, 32, draft=draft)
    plain, drafted = got[False], got[True]
    # What the two ways round differently could turn a choice whose lead is as small as that; up to such a
    # one the tokens are the same.
    compared = 0
    for a, b, la, lb, ga, gb in zip(plain[0], drafted[0], plain[3], drafted[3], plain[4], drafted[4]):
        n = min(len(la), len(lb))
        close = [i for i in range(n) if min(ga[i], gb[i]) < 1e-3]
        n = close[0] if close else n
        assert a[: 60 + n] == b[: 60 + n]
        assert all(abs(x - y) < 0.05 for x, y in zip(la[:n], lb[:n])) and all(x <= 0 for x in la)
        compared += n
    assert compared >= 32
    assert plain[2] == 0 and drafted[1] <= plain[1]
