"""Many rows a request over caches of 70 MB and more, with the tables that each request needs of them: what takes 256 rows at a time.
(The cases of test_gpu_attention.py, whose own pools are as large only counted once a request.)"""
import math

import numpy as np
import pytest
import test_gpu_attention as A

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


def in_a_large_pool(p, S, **more):
    import torch
    pages = max(p.pages, -(-(70 << 20) // (4 * p.kv * p.D * p.page)))
    k, v = (torch.full((1, pages) + tuple(p.k.shape[2:]), math.nan, dtype=p.dtype, device="cuda:0") for _ in range(2))
    k[:, :p.pages], v[:, :p.pages] = p.k, p.v
    wide = np.full((len(p.cached), -(-pages // len(p.cached)) + p.table.shape[1]), -1)
    wide[:, :p.table.shape[1]] = p.table
    p.k, p.v, p.pages, p.table = k, v, pages, wide
    step = p.step(S, **more)
    rows = (4 if p.D < 256 else 2) * 64
    # as many rows of partial results, twice a workgroup of 256, as a chunk of `rows` has
    assert step.workspace.numel() >= 2 * 256 * rows * (p.D + 2) * 4
    return step


@pytest.fixture(autouse=True)
def large_pools(monkeypatch):
    monkeypatch.setattr(A, "roomy", in_a_large_pool)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,kind", [
    ([700, 0, 129], [20, 40, 1], 8, 2, 128, "tree"), ([333], [256], 4, 2, 128, "tree"), ([90, 2000], [33, 2], 16, 2, 64, "any"),
    ([1000, 31], [30, 65], 12, 4, 96, "chain"), ([500, 7], [70, 18], 8, 2, 256, "tree"), ([3000], [100], 8, 1, 256, "any"),
    ([0, 64], [64, 70], 71, 1, 64, "tree")])
def test_many_rows_over_long_prefixes(S, dtype, cached, fresh, heads, kv, D, kind):
    A.test_many_rows_over_long_prefixes(S, dtype, cached, fresh, heads, kv, D, kind)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_pages_missing_and_values_masked_under_many_rows(S, D):
    A.test_pages_missing_and_values_masked_under_many_rows(S, D)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,group,fresh,page", [(64, 71, 3, 16), (96, 16, 5, 32), (128, 8, 40, 64), (256, 8, 9, 128)])
def test_tiles_shared_by_many_rows(S, dtype, D, group, fresh, page):
    A.test_tiles_shared_by_many_rows(S, dtype, D, group, fresh, page)


def test_values_that_are_not_finite_come_through_shared_tiles(S):
    A.test_values_that_are_not_finite_come_through_shared_tiles(S)


@pytest.mark.parametrize("D", [64, 256])
def test_many_requests_of_many_rows(S, D):
    A.test_many_requests_of_many_rows(S, D)
