"""Norms around a block with its gate and the residual sum, against 64 bits.

Tolerance.  A norm's sums have at most 64 terms in a row, then 10 halvings and 16 partial sums: 90 roundings of 2^-24 (half a step), halved by
the square root for sums of squares; what is left (mean, products, sums, exponential of up to 50) is under 38.  So 128 * 2^-24 of the
magnitudes that meet in an element, the same again through the second norm's statistics, and half a step of the result's type."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = 128 * 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def reference(case, x, y, gate, w, eps, offset, skip, scale):
    """s, out, and bounds of their errors before the last rounding, in 64 bits."""
    def weight(side, name):
        v = w.get(f"{side}_{name}")
        return (0.0 if name == "bias" else 1.0) if v is None else v.double() + (offset if name == "weight" else 0.0)

    def norm(v, e, side):
        kind = case["norm_" + side]
        if kind is None:
            return v, e
        mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        e = e + (UNIT * v.abs().mean(1, keepdim=True) + e.mean(1, keepdim=True) + UNIT * v.abs() if kind == "layer" else 0.0)
        u = v - mean
        var = (u * u).mean(1, keepdim=True)
        r = 1.0 / (var + eps).sqrt()
        off = (e * e).mean(1, keepdim=True).sqrt()                       # of the root mean square
        out = u * r * weight(side, "weight") + weight(side, "bias")
        return out, (e * r + u.abs() * r * (off * r + UNIT)) * abs(weight(side, "weight")) + UNIT * abs(weight(side, "bias"))

    s, e = 0.0, 0.0
    if y is not None:
        s, e = norm(y.double(), torch.zeros_like(y.double()), "y")
        if gate is not None:
            g = gate.double()
            g = {None: g, "sigmoid": torch.sigmoid(g), "silu": g * torch.sigmoid(g), "tanh": torch.tanh(g)}[case["act"]]
            s, e = s * g, e * g.abs() + UNIT * (s * g).abs()
        s, e = s * scale, (e + UNIT * s.abs()) * abs(scale)
    if x is not None:
        s, e = s + skip * x.double(), e + UNIT * (abs(skip) * x.double().abs())
    out, e_out = norm(s, e, "x")
    return s, out, e, e_out


def close(got, want, bound):
    assert got.shape == want.shape
    off = (got.double() - want).abs()
    allowed = bound + half(got.dtype) * want.abs() + 1e-40 + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    bad = ~(off <= allowed)
    assert not bad.any(), (int(bad.sum()), float((off / allowed).max()))


def run(case, rows, width, seed=0, pad=0, skip=0.9, scale=0.7, offset=0.0, eps=1e-5, gate_shape=None, in_place=False, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def tensor(dtype, size=1.0, r=rows):
        return (torch.randn(r, width + pad, generator=g, device="cuda") * size).to(TYPES[dtype])[:, :width]
    x = tensor(case["x"], spread) if case.get("x") else None
    y = tensor(case["y"], spread) if case.get("y") else None
    gate = None
    if case.get("gate"):
        gate = tensor(case["gate"], 2.0)
        if gate_shape == 1:
            gate = gate[0].clone()
    w = {}
    for side in "yx":
        if case["norm_" + side]:
            w[side + "_weight"] = (1 + 0.2 * torch.randn(width, generator=g, device="cuda")).to(TYPES[case.get("w", "f32")])
            if case["norm_" + side] == "layer":
                w[side + "_bias"] = torch.randn(width, generator=g, device="cuda").to(TYPES[case.get("w", "f32")])
    h = K.SpQRResidualNorm(width, norm_y=case["norm_y"], norm_x=case["norm_x"], act=case.get("act"), out_dtype=TYPES[case["out"]], weight_offset=offset, eps=eps,
                           skip=skip, scale=scale, **w)
    s, out, e, e_out = reference(case, x, y, gate, w, h.desc.eps, h.desc.weight_offset, h.desc.skip, h.desc.scale)
    total, got = K.spqr_residual_norm(h, x, y, gate, sum=x if in_place else None)
    if x is not None and y is not None:
        assert total.dtype == x.dtype
        close(total, s, e)
    else:
        assert total is None
    close(got, out, e_out)
    return h


CASES = [dict(x="f32", y="f32", out="f16", norm_y=None, norm_x="rms"),
         dict(x="bf16", y="f16", out="f16", norm_y="rms", norm_x="rms", gate="f32", act="silu", w="bf16"),
         dict(x="f16", y="bf16", out="f32", norm_y="layer", norm_x="layer", gate="f16", act="sigmoid", w="f16"),
         dict(x=None, y="f16", out="bf16", norm_y=None, norm_x="layer"),
         dict(x="f32", y=None, out="f16", norm_y=None, norm_x="rms"),
         dict(x=None, y="f32", out="f16", norm_y=None, norm_x=None, gate="f32", act="silu"),
         dict(x="f32", y="f32", out="f32", norm_y="rms", norm_x="layer", gate="bf16", act="tanh")]


@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 500, 511, 512, 1000, 1025, 4096, 4097, 8192, 8193, 16384, 16391, 22016, 40000, 65536])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_widths(width, case):
    run(CASES[case], 3, width, seed=width)


@pytest.mark.parametrize("rows", [1, 2, 5, 31, 32, 33, 700, 5000])
@pytest.mark.parametrize("width", [64, 130, 1024, 2048])
def test_rows(rows, width):
    for i, case in enumerate(CASES[:3]):
        run(case, rows, width, seed=rows + i)


@pytest.mark.parametrize("pad", [1, 3, 8, 64])
def test_rows_of_wider_tensors_at_any_address(pad):
    for i, case in enumerate(CASES):
        run(case, 37, 1000, seed=i, pad=pad)
        run(case, 1, 333, seed=i, pad=pad)


def test_one_gate_for_all_rows_and_sums_in_place():
    for i in (1, 2, 6):
        run(CASES[i], 50, 768, seed=i, gate_shape=1)
    run(CASES[0], 50, 768, in_place=True)
    run(CASES[1], 1, 4096, in_place=True)


def test_offsets_scales_and_wide_values():
    run(CASES[1], 9, 512, offset=1.0, skip=1.0, scale=-2.0)
    run(CASES[0], 9, 512, skip=0.0, scale=1.0, spread=1e8)
    run(CASES[0], 9, 512, spread=1e-12, eps=1e-30)
    run(CASES[0], 9, 512, spread=1e-3, eps=1.0)


def test_a_mean_far_from_zero():
    """Squares about the mean, not about zero: a spread of 1 about 3000."""
    g = torch.Generator(device="cuda").manual_seed(1)
    y = 3000 + torch.randn(5, 2000, generator=g, device="cuda")
    case = dict(norm_y=None, norm_x="layer")
    h = K.SpQRResidualNorm(2000, norm_x="layer", out_dtype="float32")
    _, out, _, e = reference(case, None, y, None, {}, h.desc.eps, 0.0, 1.0, 1.0)
    close(K.spqr_residual_norm(h, y=y)[1], out, e)


def test_rows_that_hold_infinities_or_nan_reach_no_other_row():
    g = torch.Generator(device="cuda").manual_seed(2)
    for width in (40, 200, 3000):
        x, y = (torch.randn(40, width, generator=g, device="cuda") for _ in range(2))
        h = K.SpQRResidualNorm(width, norm_y="rms", norm_x="rms")
        s, out = K.spqr_residual_norm(h, x, y)
        bad = torch.zeros(40, dtype=torch.bool, device="cuda")
        bad[[3, 17, 38]] = True
        x2, y2 = x.clone(), y.clone()
        x2[3, 5], y2[17, 0], y2[38, width - 1] = math.nan, math.inf, -math.inf
        s2, out2 = K.spqr_residual_norm(h, x2, y2)
        assert torch.equal(s2[~bad], s[~bad]) and torch.equal(out2[~bad], out[~bad])
        assert out2[3].isnan().all() and out2[17].isnan().any() and out2[38].isnan().any()


def test_zeros_and_no_rows():
    h = K.SpQRResidualNorm(77, norm_y="layer", norm_x="rms")
    z = torch.zeros(4, 77, device="cuda")
    s, out = K.spqr_residual_norm(h, z, z)
    assert not s.any() and not out.any()
    s, out = K.spqr_residual_norm(h, z[:0], z[:0])
    assert s.shape == (0, 77) and out.shape == (0, 77)


def test_what_is_not_written_stays():
    h = K.SpQRResidualNorm(100, norm_x="rms")
    x, y = torch.randn(3, 100, device="cuda"), torch.randn(3, 100, device="cuda")
    wide, total = torch.full((5, 133), 7.0, dtype=torch.float16, device="cuda"), torch.full((5, 104), 9.0, device="cuda")
    K.spqr_residual_norm(h, x, y, sum=total[1:4, 2:102], out=wide[1:4, 1:101])
    s, out = K.spqr_residual_norm(h, x, y)
    assert torch.equal(wide[1:4, 1:101], out) and torch.equal(total[1:4, 2:102], s)
    wide[1:4, 1:101], total[1:4, 2:102] = 7.0, 9.0
    assert (wide == 7).all() and (total == 9).all()
    only = K.SpQRResidualNorm(100, norm_x=None, out_dtype=None)
    total, nothing = K.spqr_residual_norm(only, x, y)
    assert nothing is None and torch.equal(total, x + y)


def test_refusals_of_the_binding():
    h = K.SpQRResidualNorm(64, norm_x="rms")
    x = torch.zeros(3, 64, device="cuda")
    for args, more in (((x.cpu(), x), {}), ((x, x[:2]), {}), ((x.double(), x), {}), ((x[:, ::2], x), {}), ((None, None), {}), ((x, None, x), {}),
                       ((x, x, x[:2]), {}), ((x, x, x[0, :63]), {}), ((x, x), dict(sum=x.half())), ((x, x), dict(out=x)), ((x.t().contiguous().t(), x), {})):
        with pytest.raises(ValueError):
            K.spqr_residual_norm(h, *args, **more)


def test_another_stream_and_a_captured_call():
    h = K.SpQRResidualNorm(2048, norm_y="rms", norm_x="rms")
    x, y, x2, y2 = (torch.randn(20, 2048, device="cuda") for _ in range(4))
    want, want2 = (tuple(t.clone() for t in K.spqr_residual_norm(h, *v)) for v in ((x, y), (x2, y2)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = K.spqr_residual_norm(h, x, y)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    total, out = torch.empty_like(x), torch.empty_like(x, dtype=torch.float16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.spqr_residual_norm(h, x, y, sum=total, out=out)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(total, want[0]) and torch.equal(out, want[1])
        eager = K.spqr_residual_norm(h, x2, y2)
        assert torch.equal(eager[1], want2[1])
    x.copy_(x2)
    y.copy_(y2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(total, want2[0]) and torch.equal(out, want2[1])


@pytest.mark.parametrize("rows,stride", [(3, 1 << 31), (4200, (1 << 20) + 8)])
def test_offsets_beyond_32_bits(rows, stride):
    """Rows far from each other give what they give side by side, bit by bit; what lies between them stays."""
    width = 1024
    g = torch.Generator(device="cuda").manual_seed(rows)
    norm = K.SpQRResidualNorm(width, norm_y="layer", act="sigmoid", out_dtype="bfloat16")
    far = torch.empty((rows - 1) * stride + 4 * width, dtype=torch.bfloat16, device="cuda")
    place = lambda at: torch.as_strided(far, (rows, width), (stride, 1), at * width)  # noqa: E731
    x, y, gate = (torch.randn(rows, width, device="cuda", generator=g).bfloat16() for _ in range(3))
    want_sum, want = K.spqr_residual_norm(norm, x, y, gate)
    for at, t in enumerate((x, y, gate)):
        place(at).copy_(t)
    place(3).fill_(7.0)
    got_sum, got = K.spqr_residual_norm(norm, place(0), place(1), place(2), sum=place(0), out=place(3))
    assert torch.equal(got_sum, want_sum) and torch.equal(got, want)
    assert torch.equal(place(1), y) and torch.equal(place(2), gate)
