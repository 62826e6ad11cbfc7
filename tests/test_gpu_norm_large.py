"""Norms of values as large as the header allows: magnitude * sqrt(width) just below 1.8e19, whatever the width.  Bounds as in test_gpu_norm."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402
from test_gpu_norm import close, reference  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", [1, 7, 8, 77, 1024, 4099, 8192, 8193, 40000, 65536])
def test_the_largest_values(width, kind):
    g = torch.Generator(device="cuda").manual_seed(width)
    sign = 1.0 - 2.0 * torch.randint(0, 2, (5, width), generator=g, device="cuda").float()
    y = sign * (1.799e19 / math.sqrt(width))
    y[1:3] *= 0.5 + 0.5 * torch.rand(2, width, generator=g, device="cuda")
    case = dict(norm_y=kind, norm_x="rms")
    h = K.SpQRResidualNorm(width, norm_y=kind, norm_x="rms", out_dtype="float32")
    _, out, _, e = reference(case, None, y, None, {}, h.desc.eps, 0.0, 1.0, 1.0)
    close(K.spqr_residual_norm(h, y=y)[1], out, e)
