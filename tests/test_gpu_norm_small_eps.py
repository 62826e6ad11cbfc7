"""Norms whose eps is below binary32's smallest normal number: zeros stay zeros, and rows whose squares eps outweighs are divided by its root.

Tolerance as in test_gpu_norm.  The rows' squares (1e-42 of 2e-39) are held to 2^-150 each, 1e-3 of themselves, 1e-6 of what the root is taken of:
half of that reaches the result, 2^-20 with room."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
SUBNORMAL = 2.0 ** -149


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", [1, 7, 8, 64, 77, 1000, 8192, 8193, 40000])
def test_zeros_with_the_smallest_eps(width, kind):
    z = torch.zeros(3, width, device="cuda")
    for eps in (SUBNORMAL, 1e-40, 2.0 ** -126):
        h = K.SpQRResidualNorm(width, norm_y=kind, norm_x=kind, out_dtype="float32", eps=eps)
        s, out = K.spqr_residual_norm(h, z, z)
        assert not s.any() and not out.any()


@pytest.mark.parametrize("width", [7, 8, 64, 77, 1000, 8192, 8193])
def test_small_values_with_a_small_eps(width):
    g = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn(3, width, generator=g, device="cuda") * 1e-21
    h = K.SpQRResidualNorm(width, out_dtype="float32", eps=2e-39)
    out = K.spqr_residual_norm(h, x)[1]
    want = x.double() / (x.double().square().mean(1, keepdim=True) + h.desc.eps).sqrt()
    assert ((out - want).abs() <= 2.0 ** -20 * want.abs()).all()
