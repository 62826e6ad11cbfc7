"""A plan of a step that no request has rows in: no adapter array is asked for, and any other plan asks for it.  (Without a GPU a call that is not
refused ends at its launch.)"""
import pytest

import paper_2306_03078_amd  # noqa: F401
from test_host_block import NULL, SHAPE, plan


def test_only_a_plan_of_no_requests_goes_without_adapters():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("addresses that nothing may read")
    assert plan(requests=0, adapter=None) not in (NULL, SHAPE)
    assert plan(requests=1, adapter=None) == NULL and plan(requests=130, q_start=None, adapter=None) == NULL
    assert plan(requests=0, q_start=None, adapter=None) == SHAPE
