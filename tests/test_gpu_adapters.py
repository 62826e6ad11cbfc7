"""Low-rank adapters of many requests beside shared projections: the plan against plain rules, the sums against 64 bits.

Tolerance.  A x is a sum of n products in binary32: at most n roundings of sums that random signs keep near S = sqrt(sum (a x)^2), so
10 * 2^-24 * sqrt(n) * S with room (the roundings' own signs are random too: their sum is sqrt(n) of one).  Where it meets B it is held to
2^-22 of its row's largest element; the sum over ranks has `rank` roundings; then the scale, y, and half a step of the result's type."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd as P  # noqa: E402
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def plain_plan(rows, slots, adapter, q_start):
    """count, tile, row by the rules of the header."""
    q = q_start if q_start is not None else list(range(rows + 1))
    q = [min(max(v, 0), rows) for v in q]
    groups = [[] for _ in range(slots + 1)]
    for r, a in enumerate(adapter):
        groups[a if 0 <= a < slots else slots] += list(range(q[r], q[r + 1]))
    most = min(rows, rows // 64 + slots + 1)
    tile, row = [], []
    for s, g in enumerate(groups):
        for i in range(0, len(g), 64):
            part = g[i:i + 64]
            tile.append([s if s < slots else -1, len(part)])
            row.append(part + [-1] * (64 - len(part)))
    count = len(tile)
    tile += [[-1, 0]] * (most - count)
    row += [[-1] * 64] * (most - count)
    return count, tile, row


def check_plan(rows, slots, adapter, q_start=None):
    plan = K.SpQRAdapterPlan(rows, slots)
    plan.tile.fill_(77)
    plan.row.fill_(77)
    K.spqr_adapter_plan(plan, ints(adapter), None if q_start is None else ints(q_start))
    count, tile, row = plain_plan(rows, slots, adapter, q_start)
    assert plan.count.tolist() == [count] and plan.tile.tolist() == tile and plan.row.tolist() == row
    return plan


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 129, 300, 1000, 5000])
@pytest.mark.parametrize("slots", [1, 2, 7, 300, 4096])
def test_plan_of_rows(rows, slots):
    rng = np.random.default_rng([rows, slots])
    check_plan(rows, slots, rng.integers(-2, slots + 2, rows).tolist())
    check_plan(rows, slots, [slots - 1] * rows)
    check_plan(rows, slots, [-1] * rows)
    check_plan(rows, slots, [int(a) for a in np.sort(rng.integers(0, slots, rows))[::-1]])


@pytest.mark.parametrize("requests", [1, 3, 64, 255, 256, 257, 1024])
def test_plan_of_requests(requests):
    rng = np.random.default_rng(requests)
    for longest in (1, 5, 256):
        fresh = rng.integers(0, longest + 1, requests)
        q = np.concatenate([[0], np.cumsum(fresh)]).tolist()
        for behind in (0, 1, 200):                       # rows of no request
            rows = max(1, q[-1] + behind)
            check_plan(rows, 9, rng.integers(-1, 10, requests).tolist(), q)
    check_plan(100, 3, [1] * requests, [0] * (requests + 1))     # no rows at all


def test_plan_of_one_long_request_and_of_bounds_outside_the_step():
    check_plan(100001, 2, [1], [0, 100001])
    check_plan(50, 4, [0, 1, 2], [-5, 20, 40, 90])
    plan = K.SpQRAdapterPlan(40, 4)
    K.spqr_adapter_plan(plan, ints([0, 1, 2, 1]), ints([30, 5, 70, -9, 40]))        # no ascending ones: cut to what there is room for
    row = plan.row.tolist()
    assert 0 <= plan.count.item() <= len(row) and all(-1 <= v < 40 for r in row for v in r)
    K.spqr_adapter_plan(plan, ints([0] * 1024), ints([0, 40] * 512 + [0]))
    assert 0 <= plan.count.item() <= len(row) and all(-1 <= v < 40 for r in plan.row.tolist() for v in r)


def bank(width, ms, ranks, slots, dtype="f16", seed=0, mixed=True, per_projection=False, rows=1, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    A = [(size * torch.randn(slots, r, width, generator=g, device="cuda") * width ** -0.5).to(TYPES[dtype]) for r in ranks]
    B = [(torch.randn(slots, m, r, generator=g, device="cuda") * r ** -0.5).to(TYPES[dtype]) for m, r in zip(ms, ranks)]
    rank = scale = None
    if mixed:
        of = [ints([(r * (s + 1 + p)) // slots if s % 3 else r for s in range(slots)]) for p, r in enumerate(ranks)]
        rank = of if per_projection else ints([min(int(v[s]) for v in of) for s in range(slots)])
        scale = 0.5 + torch.rand(slots, generator=g, device="cuda")
        # what lies behind an adapter's rank does not count, whatever it is
        for p in range(len(ms)):
            for s in range(slots):
                k = int((rank[p] if per_projection else rank)[s])
                A[p][s, k:] = math.nan if s % 2 else math.inf
                B[p][s, :, k:] = math.nan
    b = K.SpQRAdapters(A, B, rank=rank, scale=scale, rows=rows)
    b.plain = A, B, rank if isinstance(rank, list) else [rank] * len(ms), [scale] * len(ms)
    return b


def reference(b, adapter_of_row, x, ys):
    """Of each projection: the result, and a bound of its error before the last rounding."""
    A, B, rank, scale = b.plain
    found = []
    for p in range(len(A)):
        out = ys[p].double().clone() if ys is not None else torch.zeros(x.shape[0], B[p].shape[1], dtype=torch.float64, device="cuda")
        bound = torch.zeros_like(out)
        for a in sorted(set(v for v in adapter_of_row if 0 <= v < b.slots)):
            at = torch.tensor([t for t, v in enumerate(adapter_of_row) if v == a], device="cuda")
            k = A[p].shape[1] if rank[p] is None else int(rank[p][a])
            f = 1.0 if scale[p] is None else float(scale[p][a])
            X, Ak, Bk = x[at].double(), A[p][a, :k].double(), B[p][a, :, :k].double()
            v = X @ Ak.T
            if k:
                e = 10 * U * math.sqrt(X.shape[1]) * ((X * X) @ (Ak * Ak).T).sqrt() + 4 * U * v.abs().amax(1, keepdim=True)
                bound[at] = f * (e @ Bk.abs().T + k * U * (v.abs() @ Bk.abs().T)) + 2 * U * out[at].abs()
            out[at] += f * (v @ Bk.T)
        found.append((out, bound + 2 * U * out.abs()))
    return found


def close(got, want, bound):
    allowed = bound + torch.finfo(got.dtype).eps / 2 * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 1e-38)
    off = (got.double() - want).abs()
    bad = ~(off <= allowed)
    assert not bad.any(), (int(bad.sum()), float((off / allowed).max()))


def run(width, ms, ranks, slots, adapter, q_start=None, rows=None, dtype="f16", y="f32", seed=0, pad=0, in_place=False, base=True, mixed=True,
        per_projection=False, size=1.0):
    rows = rows or (len(adapter) if q_start is None else q_start[-1])
    b = bank(width, ms, ranks, slots, dtype, seed, mixed, per_projection, rows, size)
    plan = K.SpQRAdapterPlan(rows, slots)
    K.spqr_adapter_plan(plan, ints(adapter), None if q_start is None else ints(q_start))
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(rows, width + pad, generator=g, device="cuda").to(TYPES[dtype])[:, :width]
    ys = [torch.randn(rows, m + pad, generator=g, device="cuda").to(TYPES[y])[:, :m] for m in ms] if base else None
    of_row = list(adapter) if q_start is None else [a for a, lo, hi in zip(adapter, q_start, q_start[1:]) for _ in range(lo, hi)]
    of_row += [None] * (rows - len(of_row))
    want = reference(b, [-1 if v is None else v for v in of_row], x, ys)
    kept = [t.clone() for t in ys] if base else None
    outs = ys if in_place else [torch.full((rows, m + 2 * pad), 3.5, dtype=TYPES[y], device="cuda")[:, pad:pad + m] for m in ms]
    got = K.spqr_adapters(b, plan, x, ys, outs=outs)
    live = torch.tensor([v is not None for v in of_row], device="cuda")
    none = torch.tensor([v is not None and not 0 <= v < slots for v in of_row], device="cuda")
    for p, (out, bound) in enumerate(want):
        close(got[p][live], out[live], bound[live])
        before = kept[p] if in_place else torch.full_like(got[p], 3.5)
        assert torch.equal(got[p][~live], before[~live])                # rows of no request stay
        if base:
            assert torch.equal(got[p][none], kept[p][none])             # rows of no adapter: y, bit for bit
        else:
            assert not got[p][none].any()
    return b, plan, x, ys, got


@pytest.mark.parametrize("dtype,y", [("f16", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rank", [1, 3, 8, 15, 16, 17, 32, 33, 64, 65, 100, 128, 256])
def test_ranks(rank, dtype, y):
    rng = np.random.default_rng(rank)
    run(256, [96, 200], [rank, max(1, rank // 2)], 5, rng.integers(-1, 6, 50).tolist(), dtype=dtype, y=y, seed=rank, per_projection=rank % 2 == 0)


@pytest.mark.parametrize("width", [1, 2, 7, 8, 31, 32, 33, 100, 127, 128, 129, 500, 1025, 4096, 4099, 11008])
def test_widths(width):
    run(width, [64], [16], 3, [0, 1, 2, -1, 1, 1, 0], seed=width)
    run(width, [64, 64], [20, 20], 3, [0] * 70 + [2] * 20, seed=width, dtype="bf16", y="f16")


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 4097])
def test_outputs(m):
    run(128, [m], [16], 4, [3, 3, 0, -1, 1], seed=m)
    run(128, [m, 2 * m, 5], [40, 40, 40], 4, [0] * 33 + [1] * 66 + [-1] * 9, seed=m, y="f16")


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 32, 33, 48, 49, 63, 64, 65, 100, 128, 200, 500, 2000])
def test_rows(rows):
    rng = np.random.default_rng(rows)
    run(200, [160], [24], 2, [1] * rows, seed=rows)
    run(200, [160], [24], 6, rng.integers(-1, 6, rows).tolist(), seed=rows, dtype="bf16", y="f16")


@pytest.mark.parametrize("count", [1, 2, 3, 4, 5, 6, 7, 8])
def test_projections(count):
    run(320, [48 + 16 * p for p in range(count)], [8 + 9 * p for p in range(count)], 4, [0, 1, 2, 3, 3, 3, -1], seed=count, per_projection=True)


@pytest.mark.parametrize("pad", [1, 3, 8])
def test_rows_of_wider_tensors_at_any_address(pad):
    run(333, [77, 64], [12, 33], 3, [0] * 20 + [2] * 5 + [-1], pad=pad, seed=pad)
    run(333, [77], [12], 3, [1], pad=pad, seed=pad, dtype="bf16", y="bf16")


def test_in_place_and_without_a_base():
    run(512, [128, 256], [16, 16], 3, [0, 1, 1, 2, -1, 0], in_place=True)
    run(512, [128, 256], [16, 16], 3, [0, 1, 1, 2, -1, 0], base=False)
    run(512, [128], [16], 3, [0] * 100 + [-1] * 100, in_place=True, y="f16", dtype="bf16")
    b, plan, x, _, _ = run(512, [128], [16], 3, [0, 1], base=False)
    assert K.spqr_adapters(b, plan, x)[0].dtype == torch.float32


def test_requests_of_a_step_with_rows_behind_the_last():
    run(256, [64, 96], [16, 16], 4, [3, -1, 0, 3, 9], q_start=[0, 5, 6, 6, 100, 120], rows=150)
    run(256, [64, 96], [16, 16], 4, [3, -1, 0, 3, 9], q_start=[0, 5, 6, 6, 100, 120], rows=150, in_place=True)
    run(256, [64], [16], 4, [1], q_start=[0, 0], rows=20)


def test_adapters_of_no_rank_and_a_full_bank():
    g = torch.Generator(device="cuda").manual_seed(0)
    A, B = torch.full((2, 8, 64), math.nan, dtype=torch.float16, device="cuda"), torch.full((2, 32, 8), math.nan, dtype=torch.float16, device="cuda")
    plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(3, 2), ints([0, 1, 0]))
    x, y = torch.randn(3, 64, generator=g, device="cuda").half(), torch.randn(3, 32, generator=g, device="cuda")
    for rank in ([0, 0], [-5, 0]):
        assert torch.equal(K.spqr_adapters(K.SpQRAdapters([A], [B], rank=ints(rank), rows=3), plan, x, [y])[0], y)
    run(64, [32], [8], 2, [0, 1, 0], mixed=False)


def test_values_far_from_one():
    """A x beyond what binary16 holds, and far below it."""
    for size in (3e4, 1e-4):
        run(1024, [64], [16], 2, [0, 1, 1], size=size, mixed=False)
        run(1024, [64], [16], 2, [0, 1, 1], size=size, mixed=False, dtype="bf16")


def test_a_row_with_an_infinity_reaches_no_other():
    b, plan, x, ys, got = run(256, [64], [16], 2, [0] * 20 + [1] * 20, mixed=False)
    x2 = x.clone()
    x2[7, 3], x2[30, 0] = math.inf, math.nan
    again = K.spqr_adapters(b, plan, x2, ys)[0]
    rest = torch.ones(40, dtype=torch.bool, device="cuda")
    rest[[7, 30]] = False
    assert torch.equal(again[rest], got[0][rest]) and not again[7].isfinite().any() and again[30].isnan().all()


def test_the_same_calls_give_the_same_bits():
    b, plan, x, ys, got = run(8192, [1024], [32], 20, [int(v) for v in np.random.default_rng(3).integers(-1, 20, 90)], dtype="bf16")
    for _ in range(3):
        assert torch.equal(K.spqr_adapters(b, plan, x, ys)[0], got[0])


def test_beside_the_shared_projection_out_of_a_graph_on_another_stream():
    import spqr_synth as synth
    fs = [synth.make_matrix(256, 512, w_bits=3, beta1=16, beta2=16, group_axis=1, outlier_rate=0.01, outlier_structure="uniform", seed=(7, i)) for i in range(2)]
    matrices = [P.SpQRMatrix.from_logical(f) for f in fs]
    b = bank(512, [256, 256], [16, 16], 4, rows=40)
    plan = K.SpQRAdapterPlan(40, 4)
    adapter, x = ints([0, 1, 1, -1] * 10), torch.randn(40, 512, device="cuda").half()
    ys = [torch.empty(40, 256, device="cuda") for _ in range(2)]
    need = max(256, P.spqr_workspace_bytes(matrices, 40))
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        K.spqr_adapter_plan(plan, adapter)
        P.spqr_gemm_fused_ws(matrices, x, scratch, outs=ys)
        K.spqr_adapters(b, plan, x, ys, outs=ys)

    def eager():
        step()
        torch.cuda.synchronize()
        return [y.clone() for y in ys]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        graph = torch.cuda.CUDAGraph()
        eager()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for turn in range(3):
        adapter.copy_(ints([turn, -1, 3, 3 - turn] * 10))
        x.normal_()
        torch.cuda.synchronize()
        want = eager()
        plan.row.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(ys, want):
            assert (a - c).abs().max() <= 1e-5 * c.abs().max()   # a captured fused product may add its parts in another order


def test_slots_are_refilled():
    """Other adapters in some slots: their rows change, the others' do not."""
    b, plan, x, ys, got = run(300, [100, 64], [24, 24], 5, [0, 1, 2, 3, 4, -1, 2], mixed=False)
    other = bank(300, [100, 64], [24, 24], 2, seed=9, mixed=False)
    A, B, _, _ = other.plain
    rank = ints([24, 5])
    for p in range(2):
        A[p][1, 5:], B[p][1, :, 5:] = math.nan, math.inf
    b.load(2, A, B, rank)
    for p in range(2):
        b.plain[0][p][2:4], b.plain[1][p][2:4] = A[p], B[p]
    b.plain[2][:] = [ints([24, 24, 24, 5, 24])] * 2
    again = K.spqr_adapters(b, plan, x, ys)
    for p, (out, bound) in enumerate(reference(b, [0, 1, 2, 3, 4, -1, 2], x, ys)):
        close(again[p], out, bound)
        assert torch.equal(again[p][[0, 1, 4, 5]], got[p][[0, 1, 4, 5]]) and not torch.equal(again[p][[2, 3, 6]], got[p][[2, 3, 6]])
    for first, count in ((-1, 2), (4, 2)):
        with pytest.raises(ValueError):
            b.load(first, A, B)
    b.load(5, [a[:0] for a in A], [v[:0] for v in B])


def test_refusals_of_the_binding():
    b = bank(64, [32], [8], 2, rows=4, mixed=False)
    plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(4, 2), ints([0, 1, 0, -1]))
    x, y = torch.zeros(4, 64, dtype=torch.float16, device="cuda"), torch.zeros(4, 32, device="cuda")
    for args, more in (((x.float(), [y]), {}), ((x[:3], [y]), {}), ((x, [y[:3]]), {}), ((x, [y, y]), {}), ((x, [y]), dict(outs=[y.half()])), ((x.cpu(), [y]), {}),
                       ((x, [y.double()]), {}), ((x[:, ::2], [y]), {})):
        with pytest.raises(ValueError):
            K.spqr_adapters(b, plan, *args, **more)
    with pytest.raises(ValueError):
        K.spqr_adapter_plan(plan, ints([0, 1, 0]))
    with pytest.raises(ValueError):
        K.spqr_adapter_plan(plan, ints([0, 1]), ints([0, 1]))
    with pytest.raises(ValueError):
        K.spqr_adapter_plan(plan, torch.zeros(4, device="cuda"))
    large = K.spqr_adapter_plan(K.SpQRAdapterPlan(5000, 2), ints([0] * 5000))
    with pytest.raises(P.SpQRError):
        K.spqr_adapters(b, large, torch.zeros(5000, 64, dtype=torch.float16, device="cuda"))
    with pytest.raises(P.SpQRError):
        K.spqr_adapters(b, K.SpQRAdapterPlan(4, 3), x, [y])


def some_bank(g, slots, rank, width, ms, rows, workspace=None, dtype=torch.float16):
    make = lambda *shape: (torch.randn(shape, device="cuda", generator=g) * 0.1).to(dtype)  # noqa: E731
    return K.SpQRAdapters([make(slots, rank, width) for _ in ms], [make(slots, m, rank) for m in ms], rows=rows, workspace=workspace)


@pytest.mark.parametrize("rows,rank", [(3, 16), (130, 40), (130, 200)])
def test_offsets_beyond_32_bits(rows, rank):
    """Rows far from each other give what they give side by side, bit by bit, in place; a row of no adapter too."""
    width, ms, stride = 260, [200, 500], 1 << (31 if rows == 3 else 25)
    g = torch.Generator(device="cuda").manual_seed(rank)
    bank = some_bank(g, 2, rank, width, ms, rows)
    plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(rows, 2), ints([(0, 1, -1)[r % 3] if r % 50 == 2 else r // 100 for r in range(rows)]))
    x = torch.randn(rows, width, device="cuda", generator=g).half()
    ys = [torch.randn(rows, m, device="cuda", generator=g).half() for m in ms]
    want = K.spqr_adapters(bank, plan, x, ys)
    far = torch.empty((rows - 1) * stride + 2048, dtype=torch.float16, device="cuda")
    place = lambda at, m: torch.as_strided(far, (rows, m), (stride, 1), at)  # noqa: E731
    places = [place(0, width), place(512, ms[0]), place(1024, ms[1])]
    for to, t in zip(places, [x] + ys):
        to.copy_(t)
    got = K.spqr_adapters(bank, plan, places[0], places[1:], places[1:])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(places[0], x)


def test_banks_that_share_scratch_and_steps_of_fewer_rows():
    """Banks called one after the other on one scratch, for steps of any size up to theirs, give what each gives on its own."""
    g = torch.Generator(device="cuda").manual_seed(5)
    shapes = [(64, 512, [512, 128]), (16, 512, [900]), (130, 900, [512])]
    alone = [some_bank(g, 3, *s, rows=700) for s in shapes]
    room = torch.empty(max(b.workspace.numel() for b in alone), dtype=torch.uint8, device="cuda")
    g.manual_seed(5)
    shared = [some_bank(g, 3, *s, rows=700, workspace=room) for s in shapes]
    for rows in (1, 17, 64, 700, 129, 2):
        plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(rows, 3), ints([(r * 7 // 5) % 4 - 1 for r in range(rows)]))
        xs = [torch.randn(rows, s[1], device="cuda", generator=g).half() for s in shapes]
        want = [K.spqr_adapters(b, plan, x) for b, x in zip(alone, xs)]
        room.fill_(255)                                     # (NaN)
        got = [K.spqr_adapters(b, plan, x) for b, x in zip(shared, xs)]
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))
    with pytest.raises(P.SpQRError):                        # more rows than there is scratch for
        plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(5000, 3), ints([0] * 5000))
        K.spqr_adapters(alone[0], plan, torch.zeros(5000, 512, dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("dtype,y", [("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("m", [33, 63, 223, 300, 1751])
@pytest.mark.parametrize("rows", [5, 100, 700])
def test_the_ends_of_rows_stay_in_their_rows(rows, m, dtype, y):
    """Outputs whose rows lie side by side in a wider tensor, at odd places: the elements between them stay, long ranks and short ones."""
    for rank in (8, 64, 72, 200):
        g = torch.Generator(device="cuda").manual_seed(rank + m)
        bank = some_bank(g, 2, rank, 300, [m], rows, dtype=TYPES[dtype])
        plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(rows, 2), ints([r % 3 - 1 for r in range(rows)]))
        x = torch.randn(rows, 300, device="cuda", generator=g).to(TYPES[dtype])
        base = torch.randn(rows, m, device="cuda", generator=g).to(TYPES[y])
        want, = K.spqr_adapters(bank, plan, x, [base])
        wide = torch.full((rows, m + 7), 3.0, dtype=TYPES[y], device="cuda")
        into = wide[:, 3:3 + m]
        into.copy_(base)
        K.spqr_adapters(bank, plan, x, [into], [into])
        assert torch.equal(into, want) and bool((wide[:, :3] == 3.0).all()) and bool((wide[:, 3 + m:] == 3.0).all())
