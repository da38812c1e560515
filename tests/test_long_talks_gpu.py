"""The example of talks behind a shared prefix whose sessions keep a part of their tokens."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def talks():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    sys.path.insert(0, at)
    try:
        import long_talks
        yield long_talks
    finally:
        sys.path.remove(at)


def test_talks_that_keep_all(talks):
    """With room for everything, the hidden states are those of a decoder without a cache (to bf16's roundings
    of three layers: a few 2^-8 of each layer's output)."""
    r = talks.run(steps=12, limit=10000)
    assert r["evicted"] == 0 and r["held"] == r["said"]
    assert r["apart"] < 3 * 4 * 2.0 ** -8


def test_talks_that_evict(talks):
    r = talks.run()
    assert r["evicted"] > 0 and max(r["held"]) <= 96 + 8 and min(r["said"]) > max(r["held"])
    assert r["apart"] == r["apart"] and r["apart"] < float("inf")
