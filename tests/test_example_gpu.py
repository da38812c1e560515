"""The example of voice turns: KV that was written, evicted, loaded back and read by later steps gives
what a computation without a cache gives."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_voice_turns():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        import voice_turns
    finally:
        sys.path.pop(0)
    r = voice_turns.run(sessions=5, turns=3)
    assert r["pages_out"] > 0 and r["pages_in"] > 0
    # four layers of bf16 values (2^-8 each), rounded at different places in the two runs
    assert r["error"] < 4 * 4 * 2.0 ** -8
