"""Scores whose last binary32 place is as large as what the softmax tells apart, up to the largest that 16-bit elements give: equal ones
share, smaller ones have nothing, nothing overflows."""
import math

import pytest
import test_gpu_attention as A

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


SHAPES = [([100], [1], 2, 1, 64, False), ([1500, 40], [2, 1], 4, 2, 128, False), ([700], [9], 8, 2, 96, False), ([600, 7], [17, 3], 4, 1, 256, False),
          ([9000], [1], 4, 4, 128, False), ([900], [40], 4, 1, 128, True), ([900], [70], 2, 1, 64, True), ([700], [40], 4, 1, 256, True)]


def problem(cached, fresh, heads, kv, D, dtype):
    """Rows see cached keys only.  Scores are q[0] k[0] + q[1] k[1]; values are around 1000."""
    import torch
    p = A.Problem(cached, fresh, heads, kv, D, 16, dtype, "none")
    p.q.zero_()
    p.k.zero_()
    p.v.copy_((1000.0 + p.v.float()).to(p.dtype))
    assert torch.isfinite(p.v).all()
    return p


def places(p, r):
    import torch
    ids = torch.from_numpy(p.table[r, [j // p.page for j in range(p.cached[r])]]).cuda()
    return ids, torch.arange(p.cached[r], device="cuda:0") % p.page


def mean_check(p, out, r, keys):
    """The mean of the values of `keys`, each weight rounded by 2^-11 or 2^-8 at most, the mean once more, sums in binary32."""
    import torch
    ids, row = places(p, r)
    u = 2.0 ** -11 if p.dtype == torch.float16 else 2.0 ** -8
    group = p.heads // p.kv
    for i in range(p.kv):
        want = p.v[0, ids[keys], i, row[keys]].double().mean(0)
        got = out[p.q_start[r]:p.q_start[r + 1], i * group:(i + 1) * group].double()
        off = (got - want).abs()
        assert bool((off <= (2 * u + 2.0 ** -16) * want.abs()).all()), f"request {r} kv head {i}: {float((off / want.abs()).max())}"


@pytest.mark.parametrize("dtype,size", [("float16", 300.0), ("float16", 5000.0), ("float16", 40000.0), ("float16", 65504.0), ("bfloat16", 3000.0), ("bfloat16", 6e4),
                                        ("bfloat16", 1e9), ("bfloat16", 1e18)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,pool", SHAPES)
def test_equal_scores_share(S, dtype, size, sign, cached, fresh, heads, kv, D, pool):
    """All keys the same; then every third one far below the others."""
    import torch
    p = problem(cached, fresh, heads, kv, D, dtype)
    high, low = (size, size / 2) if sign > 0 else (size / 2, size)
    p.q[..., 0] = sign * size
    step = A.roomy(p, S) if pool else p.step(S)
    for some in (False, True):
        for r, c in enumerate(cached):
            ids, row = places(p, r)
            low_ones = (torch.arange(c, device="cuda:0") % 3 == 1) & some
            p.k[0, ids, :, row, 0] = torch.where(low_ones, low, high).to(p.dtype)[:, None]
        out = S.spqr_tree_attention(step, p.q)
        for r, c in enumerate(cached):
            keys = torch.arange(c, device="cuda:0")
            mean_check(p, out, r, keys[keys % 3 != 1] if some else keys)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("power", [20, 22, 23, 24, 25, 26, 27, 28, 30])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,pool", SHAPES)
def test_scores_that_grow_by_a_few_powers_of_two(S, dtype, power, cached, fresh, heads, kv, D, pool):
    """2^power and a little more from tile to tile (in powers of two, by less than 32): results stay among the values."""
    import torch
    p = problem(cached, fresh, heads, kv, D, dtype)
    p.q[..., 0], p.q[..., 1] = 2.0 ** (power - power // 2), 4.0
    step = A.roomy(p, S, scale=math.log(2)) if pool else p.step(S, scale=math.log(2))
    for turn in (1.0, 2.0, 3.75, 4.0, 7.0):
        for r, c in enumerate(cached):
            ids, row = places(p, r)
            p.k[0, ids, :, row, 0] = 2.0 ** (power // 2)
            p.k[0, ids, :, row, 1] = (turn * (torch.arange(c, device="cuda:0") // 32 % 37)).to(p.dtype)[:, None]
        out = S.spqr_tree_attention(step, p.q)
        for r in range(len(cached)):
            ids, row = places(p, r)
            for i in range(kv):
                v = p.v[0, ids, i, row].double()
                got = out[p.q_start[r]:p.q_start[r + 1], i * (heads // kv):(i + 1) * (heads // kv)].double()
                assert bool((got >= v.amin(0) * (1 - 2.0 ** -6)).all()) and bool((got <= v.amax(0) * (1 + 2.0 ** -6)).all())
