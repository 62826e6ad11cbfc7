"""Attention with scales at the ends of their range: zero (every key that a row sees counts the same), the smallest numbers."""
import numpy as np
import pytest
import test_gpu_attention as A

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


def uniform_check(p, step_of, S, scale):
    """The same as with queries of zero, whose check knows the bound of a mean."""
    import torch
    out = S.spqr_tree_attention(step_of(scale=scale), p.q)
    p.q = torch.zeros_like(p.q)
    p.check(out)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, -1e-40])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,kind", [
    ([0], [1], 2, 1, 64, "chain"), ([37, 0, 64], [3, 5, 1], 4, 2, 128, "tree"), ([0, 10, 0], [64, 3, 1], 4, 2, 128, "any"), ([0, 0], [5, 1], 2, 2, 96, "none"),
    ([2000, 31], [2, 1], 40, 8, 96, "chain"), ([5000, 3], [33, 4], 2, 1, 256, "tree")])
def test_no_score_counts(S, dtype, scale, cached, fresh, heads, kv, D, kind):
    p = A.Problem(cached, fresh, heads, kv, D, 16, dtype, kind)
    uniform_check(p, lambda **more: p.step(S, **more), S, scale)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_no_score_counts_in_shared_tiles(S, D):
    p = A.Problem([900], [70], 4, 1, D, 16, "float16", "tree")
    uniform_check(p, lambda **more: A.roomy(p, S, **more), S, 0.0)


def test_a_scale_of_zero_is_no_default(S):
    p = A.Problem([20], [2], 2, 1, 64, 16, "float16", "chain")
    assert p.step(S, scale=0).desc.scale == 0.0 and p.step(S).desc.scale == np.float32(0.125)
