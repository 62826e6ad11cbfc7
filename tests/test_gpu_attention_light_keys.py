"""Keys of little weight beside one that has nearly all: each counts little, all together they count."""
import math

import pytest
import test_gpu_attention as A

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


def check(p, S, step, heavy):
    """Against 64 bits.  Probabilities in binary16 are multiples of 2^-24 from below 2^-14 on, of at most 2^15 where a sum of 2^7
    and more is theirs (the largest score's is at least 2^7): off by 2^-11 of themselves or by half of 2^-24 of those 2^7, which is
    2^-32 of the largest.  Scores: two exact products in binary32, 2^-20 in the exponent."""
    import torch
    out = S.spqr_tree_attention(step, p.q).double()
    for r, c in enumerate(p.cached):
        ids = torch.from_numpy(p.table[r, [j // p.page for j in range(c)]]).cuda()
        row = torch.arange(c, device="cuda:0") % p.page
        K, V = (x[0][ids, :, row].double() for x in (p.k, p.v))
        for t in range(p.q_start[r], p.q_start[r + 1]):
            for h in range(p.heads):
                k, v = K[:, h // (p.heads // p.kv)], V[:, h // (p.heads // p.kv)]
                s = p.q[t, h].double() @ k.T
                assert heavy < 0 or int(s.argmax()) == heavy
                e = torch.exp(s - s.max())
                z = e.sum()
                want = e @ v / z
                bound = (2.0 ** -11 + 2.0 ** -19) * (e @ v.abs()) / z + 2.0 ** -11 * want.abs() + 2.0 ** -32 * v.abs().sum(0) / z + 2.0 ** -25
                ratio = ((out[t, h] - want).abs() / bound).max()
                assert float(ratio) <= 1, f"request {r} row {t} head {h}: {float(ratio)} of the bound"


def one_heavy_key(cached, fresh, heads, kv, D, gap, at=0, seed=0):
    """Scores of zero for all cached keys but one, whose score is `gap` powers of two above and whose value is zero; the others'
    values are around 1000.  New keys are seen by nobody."""
    import torch
    p = A.Problem(cached, fresh, heads, kv, D, 16, "float16", "none", seed=seed)
    p.q.zero_()
    p.q[..., 0] = 4.0
    p.k.zero_()
    p.v.copy_((1000.0 + 100.0 * torch.randn(p.v.shape, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(seed))).half())
    for r in range(len(cached)):
        place = (0, p.table[r, at // 16], slice(None), at % 16)
        p.k[place][:, 0] = gap * math.log(2) / 4
        p.v[place] = 0.0
    return p


@pytest.mark.parametrize("gap", [17.3, 25.3, 27.8])
@pytest.mark.parametrize("cached,fresh,heads,kv,D", [([600], [1], 2, 2, 64), ([600, 333], [1, 1], 2, 1, 128), ([600], [5], 8, 2, 128), ([500], [8], 5, 1, 96),
                                                     ([600], [10], 3, 1, 256)])
def test_one_key_has_nearly_all(S, gap, cached, fresh, heads, kv, D):
    p = one_heavy_key(cached, fresh, heads, kv, D, gap)
    check(p, S, p.step(S, scale=1.0), 0)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("gap", [17.3, 26.3])
def test_one_key_has_nearly_all_in_shared_tiles(S, D, gap):
    p = one_heavy_key([600], [40], 2, 1, D, gap)
    check(p, S, A.roomy(p, S, scale=1.0), 0)


def test_scores_that_grow_by_less_than_the_reference_follows(S):
    """Probabilities at their largest: each tile's scores a little less than what would move the reference above the last ones'."""
    p = one_heavy_key([600], [1], 1, 1, 64, 0.0)
    for step in (7.9, 8.1, 1.0):
        for j in range(600):
            p.k[0, p.table[0, j // 16], :, j % 16, 0] = 0.0 if j < 128 else step * math.log(2) / 4 + (j // 128) * 0.01
        p.v[p.v == 0] = 1000.0
        check(p, S, p.step(S, scale=1.0), -1)
