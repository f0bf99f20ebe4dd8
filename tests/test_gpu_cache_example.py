"""The example that runs the cache's calls and the verification together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# Logits have a standard deviation of 3.  A hidden state goes through about a dozen roundings to bf16 (2^-8 / sqrt 3 each): 0.8 %, 0.025 of a logit; the
# difference of two logits over some 150 tokens stays within 6 times sqrt 2 of that, 0.2, and the verified logits are rounded once more (at 16: 0.06 each).
# A row of the cache in the wrong place moves logits by their standard deviation.
TOLERANCE = 0.4


def test_every_committed_token_is_the_models_choice():
    print("example", flush=True)
    spec = importlib.util.spec_from_file_location("cached_decode", os.path.join(ROOT, "examples", "cached_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    got, short, c = example.main(say=lines.append)
    print("\n".join(lines), flush=True)
    assert all(len(x) >= 40 for x in got) and max(map(max, short)) <= TOLERANCE
    assert not c.refs.any() and not c.held.any() and (c.page_table == -1).all()
