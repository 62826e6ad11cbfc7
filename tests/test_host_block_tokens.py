"""Tokens of a call that scores rows are [rows, given]: [given, rows] has as many elements and would be read in another order."""
import pytest
import torch

import paper_2306_03078_amd.block_binding as K
from test_host_block_streams import Tensor, handles, world  # noqa: F401


@pytest.mark.parametrize("given,shape,fits", [(1, (3,), True), (1, (3, 1), True), (1, (1, 3), True), (2, (3, 2), True), (2, (6,), True), (3, (3, 3), True),
                                              (2, (2, 3), False), (2, (6, 1), False), (2, (1, 6), False), (1, (2,), False), (1, (4, 1), False)])
def test_shapes_of_tokens(world, given, shape, fits):  # noqa: F811
    got, _, one = world
    scores = handles(one)[3]
    scores.given = given
    logits, tokens = Tensor((3, 64)), Tensor(shape, torch.int32)
    if fits:
        K.spqr_token_logprobs(scores, logits, tokens)
        assert len(got) == 1
    else:
        with pytest.raises(ValueError):
            K.spqr_token_logprobs(scores, logits, tokens)
        assert got == []
