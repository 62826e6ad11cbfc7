"""Log probabilities of logits (or scores, where the scale is large) between 2^20 and the end of binary32, of masks by large numbers, and of rows that
hold no number.

Tolerance as in test_gpu_scores: what an exponential's argument is off by goes by its distance from the row's largest score, whatever that
one's size."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402
from test_gpu_scores import TYPES, check, draw  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("rows,vocab", [(2, 600), (3, 20000), (600, 9000), (1, 100000)])
@pytest.mark.parametrize("power", [20, 23, 24, 25, 28, 30, 31, 32, 33, 40, 64, 99, 100, 101, 125])
def test_logits_of_any_size(power, rows, vocab):
    """Logits near 1.1 * 2^power of both signs, with a few of the type's steps between them, so that some are equal and some are near."""
    g = torch.Generator(device="cuda").manual_seed(power)
    for dtype in ("f32", "bf16"):
        step = 1.1 * 2.0 ** power * torch.finfo(TYPES[dtype]).eps
        near = 1.1 * 2.0 ** power + step * torch.randint(0, 3, (rows, vocab), generator=g, device="cuda").double()
        tokens = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda", dtype=torch.int32)
        for sign in (1.0, -1.0):
            check((sign * near).to(TYPES[dtype]), tokens, 5)
            mixed = torch.where(torch.rand(rows, vocab, generator=g, device="cuda") < 0.5, -sign * near, sign * near)
            check(mixed.to(TYPES[dtype]), tokens, 5)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [1e4, 3.3e6, 1e9, 1e12, 1e25])
def test_large_scales(scale, dtype):
    for rows, vocab in ((2, 20000), (300, 3000)):
        logits, tokens = draw(rows, vocab, dtype, seed=11, size=300.0)
        check(logits, tokens(2), 7, scale=scale)


@pytest.mark.parametrize("rows,vocab", [(2, 600), (3, 20000), (600, 9000), (1, 100000)])
@pytest.mark.parametrize("mask", [-1e7, -1e9, -1.1e10, -1e12, -1e20, -1e29, -1e31, -3e38])
def test_masks_by_large_numbers(mask, rows, vocab):
    """Tokens forbidden by a number, whole stretches of them too: those that are left count as if the others were not there."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    for dtype in ("f32", "bf16"):
        for kind in ("half", "front", "back", "all"):
            logits, tokens = draw(rows, vocab, dtype, seed=rows)
            if kind == "half":
                logits[torch.rand(rows, vocab, generator=g, device="cuda") < 0.5] = mask
            elif kind == "front":
                logits[:, :-7] = mask
            elif kind == "back":
                logits[:, 7:] = mask
            else:
                logits[:] = mask
            check(logits, tokens(2), 5)
            check(logits, tokens(2), 9, scale=0.37)
