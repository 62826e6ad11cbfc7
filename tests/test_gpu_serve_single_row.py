"""A step of one row: the distance to a next row, which there is not, is no reason to refuse it."""
import pytest
import test_gpu_attention as A

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("extra", [1, 3, 5])
@pytest.mark.parametrize("flat", [False, True])
def test_one_row_out_of_a_wider_tensor(extra, flat):
    import torch
    import paper_2306_03078_amd.serve_binding as S
    p = A.Problem([40], [1], 4, 2, 64, 16, "float16", "chain")
    step = p.step(S)
    want = S.spqr_tree_attention(step, p.q)
    p.check(want)
    shape = (1, 256) if flat else (1, 4, 64)
    q, out = (torch.full((1, 256 + extra), 9.0, dtype=torch.float16, device="cuda:0") for _ in range(2))
    q[:, :256] = p.q.view(1, 256)
    rows = [x[:, :256] if flat else x[:, :256].as_strided(shape, (256 + extra, 64, 1)) for x in (q, out)]
    S.spqr_tree_attention(step, rows[0], out=rows[1])
    assert torch.equal(rows[1].reshape(1, 4, 64), want) and bool((out[:, 256:] == 9).all())
    step.slot.fill_(5)
    step.position.zero_()
    kv = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda:0")
    assert torch.equal(S.spqr_cache_store(step, rows[0], kv, kv), p.q)
