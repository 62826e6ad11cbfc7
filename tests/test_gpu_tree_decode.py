"""The example that decodes with trees of drafted tokens: the same tokens as token by token, in fewer passes."""
import importlib.util
import os

import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("seed,requests", [(0, 3), (3, 1), (5, 6)])
def test_trees_give_the_tokens_of_token_by_token_decoding(seed, requests):
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    plain, trees, ahead, passes = example.main(count=32, requests=requests, seed=seed)
    assert passes < 24
    for x, y, a in zip(plain, trees, ahead):
        differ = [i for i in range(32) if x[i] != y[i]]
        # logits are of size sqrt(512), their inputs rounded at 2^-11 in a dozen places: a choice that is ahead by more stands
        assert not differ or a[differ[0]] < 0.1, (differ[0], a[differ[0]])
