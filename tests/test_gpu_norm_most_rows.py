"""Norms of more rows than one launch has threads for (2^32 in a direction of its grid)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def test_norms_of_two_to_the_29_rows():
    rows = (1 << 29) + 77
    x = torch.empty(rows, 1, dtype=torch.float16, device="cuda")
    x.view(-1)[:] = 3.0
    x[::1000003] = -5.0
    x[-1] = 7.0
    h = K.SpQRResidualNorm(1, norm_x=None, skip=2.0)
    out = torch.zeros_like(x)
    K.spqr_residual_norm(h, x, out=out)
    assert torch.equal(out, 2 * x)


def test_norms_of_two_to_the_22_wide_rows():
    """In place (70 GB): x + x, a norm of nothing."""
    if torch.cuda.mem_get_info()[0] < 90e9:
        pytest.skip("needs 90 GB of device memory")
    rows, width = (1 << 22) + 3, 8193
    x = torch.ones(rows, width, dtype=torch.float16, device="cuda")
    x[::1001, 5], x[-1], x[-1, -1] = 3.0, 2.0, 9.0
    h = K.SpQRResidualNorm(width, norm_x=None, skip=2.0, out_dtype=None)
    K.spqr_residual_norm(h, x, sum=x)
    x[::1001, 5] -= 4.0
    assert (x[-1, :-1] == torch.where(torch.arange(width - 1, device="cuda") == 5, 4.0 - 4.0 * ((rows - 1) % 1001 == 0), 4.0)).all() and x[-1, -1] == 18.0
    for a in range(0, rows - 1, 1 << 18):
        assert bool((x[a:min(a + (1 << 18), rows - 1)] == 2.0).all())
