"""Norms of more rows than there are workgroups, so that a workgroup takes rows in turn: odd widths, several rows a workgroup (the last one's not all
there), one gate for all rows, sums in place.  Bounds as in test_gpu_norm; and each row gives what it gives in a call of few rows, bit by bit."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402
from test_gpu_norm import CASES, TYPES, run  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
SHAPES = [(65601, 64), (65603, 63), (33001, 130), (16401, 255), (8201, 511), (5003, 1001), (2051, 2047), (1100, 4095), (1030, 8191), (2051, 2048)]


@pytest.mark.parametrize("rows,width", SHAPES)
def test_against_64_bits(rows, width):
    for i in (1, 2, 5):
        run(CASES[i], rows, width, seed=i)
        run(CASES[i], rows, width, seed=i, gate_shape=1)
    run(CASES[0], rows, width, in_place=True)
    run(CASES[6], rows, width, in_place=True, pad=3)


@pytest.mark.parametrize("rows,width", SHAPES)
def test_every_type_gives_what_few_rows_give(rows, width):
    g = torch.Generator(device="cuda").manual_seed(width)
    make = lambda t, r=rows: (torch.randn(r, width, generator=g, device="cuda") * 2).to(TYPES[t])  # noqa: E731
    weight, bias = make("f32", 1)[0], make("f32", 1)[0]
    for x_type in TYPES:
        for y_type in TYPES:
            x, y, one = make(x_type), make(y_type), make(y_type, 1)[0]
            h = K.SpQRResidualNorm(width, norm_y="layer", norm_x="rms", act="sigmoid", y_weight=weight, y_bias=bias, x_weight=weight, out_dtype=TYPES[y_type])
            for gate in (y, one):
                s, out = K.spqr_residual_norm(h, x, y, gate)
                for at in (0, rows // 2, rows - 40):
                    few = K.spqr_residual_norm(h, x[at:at + 40], y[at:at + 40], gate if gate is one else gate[at:at + 40])
                    assert torch.equal(s[at:at + 40], few[0]) and torch.equal(out[at:at + 40], few[1])
