"""Attention of chains and trees of new tokens over a paged cache on the GPU, against the formula in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


def i32(a):
    import torch
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).to("cuda:0").contiguous()


def i64(a):
    import torch
    return torch.as_tensor(np.asarray(a), dtype=torch.int64).to("cuda:0").contiguous()


class Problem:
    """Requests over a cache of shuffled pages.  sees[r][i]: the new tokens that row i of r sees."""

    def __init__(self, cached, fresh, heads, kv, D, page, dtype, kind="chain", seed=0, layers=1, spread=1.0, spare=0):
        import torch
        self.rng = rng = np.random.default_rng([seed, heads, D, page])
        g = torch.Generator(device="cuda:0").manual_seed(seed + 17)
        self.cached, self.fresh, self.heads, self.kv, self.D, self.page = list(cached), list(fresh), heads, kv, D, page
        self.dtype, self.kind = getattr(torch, dtype), kind
        self.q_start = [0] + np.cumsum(fresh).tolist()
        T = self.q_start[-1]
        held = [-(-(c + f) // page) for c, f in zip(cached, fresh)]
        width = max(1, max(held))
        self.pages = sum(held) + 3
        ids = rng.permutation(self.pages)
        self.table = np.full((len(cached), width), -1)
        at = 0
        for r, h in enumerate(held):
            self.table[r, :h] = ids[at:at + h]
            at += h
        shape = (layers, self.pages, kv, page, D)
        self.k, self.v = (torch.randn(shape, device="cuda:0", generator=g).to(self.dtype) for _ in range(2))
        self.q = (spread * torch.randn(T + spare, heads, D, device="cuda:0", generator=g)).to(self.dtype)
        self.words = 0 if kind == "chain" else max(1, -(-max(fresh) // 64))
        self.sees = []
        for n in fresh:
            rows = []
            for i in range(n):
                if kind == "chain":
                    rows.append(set(range(i + 1)))
                elif kind == "tree":
                    p = int(rng.integers(max(-1, i // 2 - 2), i)) if i else -1
                    rows.append((rows[p] if p >= 0 else set()) | {i})
                elif kind == "any":                       # any set, the empty one among them
                    rows.append({j for j in range(n) if rng.random() < (0.0, 0.1, 0.6)[i % 3]})
                else:
                    rows.append(set())
            self.sees.append(rows)

    def masks(self):
        rows = [[sum(1 << (j - 64 * w) for j in s if 64 * w <= j < 64 * w + 64) for w in range(self.words)] for r in self.sees for s in r]
        return i64(np.array(rows, dtype=np.uint64).reshape(-1, self.words).view(np.int64))

    def step(self, S, **more):
        import torch
        T = self.q.shape[0]
        if self.words:
            m = self.masks()
            more["mask"] = torch.cat([m, torch.full((T - m.shape[0], self.words), -1, dtype=torch.int64, device="cuda:0")])
        return S.SpQRStep(self.k, self.v, self.heads, cached=i32(self.cached), table=i32(self.table), q_start=i32(self.q_start), tokens=T,
                          **{"max_fresh": max(self.fresh), **more})

    def visible(self, r):
        """Keys that each row of r sees, the ones on pages that are not there taken out."""
        keys = self.cached[r] + self.fresh[r]
        there = np.array([j // self.page < self.table.shape[1] and 0 <= self.table[r, j // self.page] < self.pages for j in range(keys)], dtype=bool)
        rows = np.zeros((self.fresh[r], keys), dtype=bool)
        rows[:, :self.cached[r]] = True
        for i, s in enumerate(self.sees[r]):
            rows[i, [self.cached[r] + j for j in s]] = True
        return rows & there[None, :] if keys else rows

    def check(self, out, layer=0, scale=None):
        """|out - exact| within what the kernel's roundings can do.  u: half a unit of the type.  Scores are binary32 sums of D
        exact products: off by at most D 2^-24 sum |q k| scale; exp and its argument (scaled by log2 e) 2^-22 of the
        score's size and 2^-21 of the result; p is rounded to the type (u, and a half of binary16's smallest step below its
        normal range); sums of n terms in binary32, in parts and rescaled: sqrt(n) 2^-22 covers their random walk."""
        import torch
        scale = scale or 1.0 / math.sqrt(self.D)
        u, least = (2.0 ** -11, 2.0 ** -25) if self.dtype == torch.float16 else (2.0 ** -8, 0.0)
        group = self.heads // self.kv
        worst = 0.0
        for r in range(len(self.cached)):
            f, c = self.fresh[r], self.cached[r]
            if f == 0:
                continue
            keys = c + f
            vis = torch.from_numpy(self.visible(r)).cuda()
            ids = torch.from_numpy(np.clip(self.table[r, [min(j // self.page, self.table.shape[1] - 1) for j in range(keys)]], 0, self.pages - 1)).cuda()
            row = torch.arange(keys, device="cuda:0") % self.page
            # [keys, kv, D]; what nobody sees is zero from here on
            K, V = (x[layer][ids, :, row].double() for x in (self.k, self.v))
            for i in range(self.kv):
                q = self.q[self.q_start[r]:self.q_start[r + 1], i * group:(i + 1) * group].double()        # [f, group, D]
                for row_i in range(f):
                    on = vis[row_i]
                    got = out[self.q_start[r] + row_i, i * group:(i + 1) * group].double()
                    if not bool(on.any()):
                        assert not bool(got.any()), "a row that sees nothing"
                        continue
                    k, v = K[on, i], V[on, i]
                    s = q[row_i] @ k.T * scale
                    p = torch.softmax(s, 1)
                    want = p @ v
                    size = (q[row_i].abs() @ k.abs().T * scale).amax(1, keepdim=True)
                    off = self.D * 2.0 ** -24 * size + 2.0 ** -22 * s.abs().amax(1, keepdim=True) + 2.0 ** -21
                    mass = p @ v.abs()
                    bound = (u + 2 * off + math.sqrt(keys) * 2.0 ** -22) * mass + (u + 2.0 ** -22) * want.abs() + least * (
                        v.abs().sum(0, keepdim=True) / torch.exp(s - s.amax(1, keepdim=True)).sum(1, keepdim=True) + 1)
                    ratio = ((got - want).abs() / bound)
                    assert bool((ratio <= 1).all()), f"request {r} row {row_i} kv head {i}: {float(ratio.max())} of the bound"
                    worst = max(worst, float(ratio.max()))
        return worst


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,page,kind", [
    ([0], [1], 1, 1, 64, 16, "chain"),                          # one key
    ([5], [1], 4, 4, 128, 16, "chain"),
    ([1024], [1], 8, 8, 128, 16, "chain"),
    ([31, 32, 33, 0, 63, 15, 16, 17], [1] * 8, 2, 2, 128, 16, "chain"),
    ([300, 0, 1, 129], [3, 17, 1, 33], 6, 2, 96, 32, "chain"),
    ([700, 20], [16, 9], 4, 4, 128, 16, "tree"),
    ([255, 256, 0], [5, 64, 64], 16, 2, 128, 64, "tree"),
    ([77], [65], 3, 1, 64, 128, "tree"),
    ([130, 3], [256, 200], 2, 1, 128, 16, "tree"),
    ([40], [130], 8, 1, 256, 32, "tree"),
    ([100, 9], [7, 2], 71, 1, 64, 16, "tree"),
    ([0, 10, 0], [64, 3, 1], 4, 2, 128, 16, "any"),             # rows that see nothing, with and without a prefix
    ([0, 0], [5, 1], 2, 2, 256, 256, "none"),
    ([2000], [2], 40, 8, 96, 256, "chain"),
    ([50, 7, 90], [0, 4, 0], 4, 2, 128, 16, "chain"),           # requests without new tokens
])
def test_against_the_formula(S, dtype, cached, fresh, heads, kv, D, page, kind):
    p = Problem(cached, fresh, heads, kv, D, page, dtype, kind)
    p.check(S.spqr_tree_attention(p.step(S), p.q))


@pytest.mark.parametrize("dtype,heads,kv,D,cached,fresh", [("float16", 4, 4, 128, 9000, 2), ("bfloat16", 16, 2, 64, 20011, 9), ("float16", 2, 1, 256, 5000, 33),
                                                           ("bfloat16", 8, 1, 96, 33333, 1)])
def test_long_prefixes(S, dtype, heads, kv, D, cached, fresh):
    p = Problem([cached, 3, cached // 3], [fresh, 1, fresh], heads, kv, D, 64, dtype, "tree" if fresh > 2 else "chain")
    p.check(S.spqr_tree_attention(p.step(S), p.q))


@pytest.mark.parametrize("R", [65, 300, 1024])
def test_many_requests(S, R):
    rng = np.random.default_rng(R)
    p = Problem(rng.integers(0, 90, R), rng.integers(0, 4, R), 2, 1, 64, 16, "float16", "tree")
    p.check(S.spqr_tree_attention(p.step(S), p.q))


@pytest.mark.parametrize("hint", [0, 1, 256])
def test_the_hint_changes_no_result_beyond_rounding(S, hint):
    p = Problem([500, 0, 130], [40, 3, 17], 8, 2, 128, 16, "float16", "tree")
    p.check(S.spqr_tree_attention(p.step(S, max_fresh=hint), p.q))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kind,fresh,D", [("tree", [20, 5, 1], 128), ("any", [7, 40, 2], 64), ("chain", [1, 3, 12], 128), ("any", [9, 30, 3], 256), ("tree", [70, 3, 1], 96)])
def test_what_nobody_sees_does_not_count(S, dtype, bad, kind, fresh, D):
    """Stale rows behind the last key, on free pages, and new tokens of other branches hold NaN and infinities."""
    import torch
    p = Problem([37, 0, 64], fresh, 4, 2, D, 16, dtype, kind)
    want = S.spqr_tree_attention(p.step(S), p.q)
    seen = torch.zeros(p.k.shape[:4], dtype=torch.bool)
    for r in range(3):
        for j in np.nonzero(p.visible(r).any(0))[0]:
            seen[0, p.table[r, j // 16], :, j % 16] = True
    for c in (p.k, p.v):
        c[~seen.cuda()] = bad
    step = p.step(S)
    out = S.spqr_tree_attention(step, p.q)
    p.check(out)
    assert torch.equal(out, want)
    # a sibling's row, seen by some rows only: the others stay as they were
    for r in range(3):
        vis = p.visible(r)
        for j in range(p.cached[r], p.cached[r] + fresh[r]):
            some = vis[:, j]
            if some.any() and not some.all():
                at = (0, p.table[r, j // 16], slice(None), j % 16)
                old = p.k[at].clone(), p.v[at].clone()
                p.v[at], p.k[at] = bad, 0.0
                got = S.spqr_tree_attention(step, p.q)[p.q_start[r]:p.q_start[r + 1]]
                rows = torch.from_numpy(~some).cuda()
                assert torch.equal(got[rows], want[p.q_start[r]:p.q_start[r + 1]][rows])
                seeing = got[~rows]
                assert bool(torch.isnan(seeing).all()) if math.isnan(bad) else bool((seeing == bad).all())
                p.k[at], p.v[at] = bad, old[1]
                got = S.spqr_tree_attention(step, p.q)[p.q_start[r]:p.q_start[r + 1]]
                assert torch.equal(got[rows], want[p.q_start[r]:p.q_start[r + 1]][rows])
                p.k[at] = old[0]
                break


def test_seen_values_that_are_not_finite_come_through(S):
    """A NaN in a cached value reaches its element of every row, an infinity too; large finite ones stay finite."""
    import torch
    for D in (64, 128):
        p = Problem([200], [4], 4, 2, D, 16, "float16", "tree")
        row = (0, p.table[0, 3], 1, 7)
        p.v[row][5], p.v[row][9] = math.nan, -math.inf
        p.v[0, p.table[0, 5], 1, 2, 11] = 65504.0
        out = S.spqr_tree_attention(p.step(S), p.q)
        assert bool(torch.isnan(out[:, 2:, 5]).all()) and bool((out[:, 2:, 9] == -math.inf).all())
        rest = [d for d in range(D) if d not in (5, 9)]
        assert bool(torch.isfinite(out[:, 2:, rest]).all()) and bool(torch.isfinite(out[:, :2]).all())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_scores_of_any_size(S, dtype):
    """Scores of hundreds either way, a maximum that comes late, keys that are all the same."""
    import torch
    p = Problem([900, 33], [6, 30], 4, 2, 128, 16, dtype, "tree", spread=40.0)
    p.check(S.spqr_tree_attention(p.step(S), p.q))
    order = torch.arange(900, dtype=torch.float64) / 900
    for j in range(900):                       # scores that grow along the prefix
        p.k[0, p.table[0, j // 16], :, j % 16] = (p.q[0, 0].double().cpu() * order[j] * 0.05).to(p.dtype).cuda()
    p.check(S.spqr_tree_attention(p.step(S), p.q))
    p.k[:] = p.k[0, 0, 0, 0]
    p.check(S.spqr_tree_attention(p.step(S), p.q))
    p.q.zero_()
    p.check(S.spqr_tree_attention(p.step(S, scale=-3.0), p.q), scale=-3.0)


@pytest.mark.parametrize("page", [16, 64])
def test_pages_that_are_not_there(S, page):
    p = Problem([400, 200, 90], [5, 17, 3], 4, 2, 128, page, "float16", "tree")
    p.table[0, 1], p.table[0, -1], p.table[1, 0], p.table[2, :] = -1, p.pages, 2 ** 31 - 1, -2 ** 31
    p.check(S.spqr_tree_attention(p.step(S), p.q))


def test_strides_layers_scale_and_unused_rows(S):
    import torch
    p = Problem([100, 40], [3, 2], 4, 2, 128, 16, "float16", "tree", layers=3, spare=4)
    T = p.q.shape[0]
    wide = torch.zeros(T, 5, 4, 128, dtype=torch.float16, device="cuda:0")
    wide[:, 2] = p.q
    out = torch.full((T, 1024), -7.0, dtype=torch.float16, device="cuda:0")
    step = p.step(S, scale=0.3)
    S.spqr_tree_attention(step, wide[:, 2], layer=2, out=out[:, 256:768])
    p.check(out[:, 256:768].view(T, 4, 128), layer=2, scale=0.3)
    assert bool((out[5:] == -7).all()) and bool((out[:, :256] == -7).all()) and bool((out[:, 768:] == -7).all())
    flat = S.spqr_tree_attention(step, p.q.view(T, -1), layer=2)
    assert torch.equal(flat[:5], out[:5, 256:768])
    for bad in (dict(q=p.q[:4]), dict(q=p.q.bfloat16()), dict(q=p.q.transpose(0, 1)), dict(q=p.q, out=out.float()), dict(q=p.q, out=out)):
        with pytest.raises(ValueError):
            S.spqr_tree_attention(step, **bad)


def test_lengths_that_make_no_sense_stay_in_the_arrays(S):
    """Lengths beyond the table and rows beyond the step: the call ends, nothing outside `out` is written."""
    import torch
    p = Problem([60, 60], [4, 4], 4, 2, 128, 16, "float16", "tree")
    guard = torch.full((40, 4, 128), -7.0, dtype=torch.float16, device="cuda:0")
    for cached, q_start in (([2 ** 31 - 1, 60], [0, 4, 8]), ([-2 ** 31, -5], [0, 4, 8]), ([60, 60], [0, 900, 2 ** 31 - 1]), ([60, 60], [-9, 4, 2]),
                            ([60, 60], [2 ** 31 - 1, -2 ** 31, 8]), ([60, 60], [7, 3, 1])):
        step = p.step(S)
        step.cached.copy_(i32(cached))
        step.q_start.copy_(i32(q_start))
        S.spqr_tree_attention(step, p.q, out=guard[16:24])
        torch.cuda.synchronize()
        assert bool((guard[:16] == -7).all()) and bool((guard[24:] == -7).all())


def test_offsets_beyond_32_bits(S):
    """Pages whose first element lies behind 2^31 and 2^32 elements of the cache (9 GB for k and for v)."""
    import torch
    page, kv, D = 256, 8, 128
    pages = (2 ** 32 + 2 ** 28) // (page * kv * D)
    p = Problem([1000], [3], 16, kv, D, page, "float16", "tree")
    big = [torch.empty(1, pages, kv, page, D, dtype=torch.float16, device="cuda:0") for _ in range(2)]
    ids = [pages - 1, 2 ** 31 // (page * kv * D) + 1, 0, 2 ** 32 // (page * kv * D) + 1]
    for old, new in zip((p.k, p.v), big):
        for at, id_ in enumerate(ids):
            new[0, id_] = old[0, p.table[0, at]]
    p.k, p.v = big
    p.table[0, :4], p.pages = ids, pages
    p.check(S.spqr_tree_attention(p.step(S), p.q))
    # ... and stores and moves to them
    step = p.step(S, slot=i32([(pages - 1) * page + 5, 3, (pages - 2) * page + 255]), position=i32([0, 1, 2]))
    x = torch.randn(3, kv, D, device="cuda:0", dtype=torch.float16)
    S.spqr_cache_store(step, p.q, x, 2 * x)
    for t, s in enumerate(step.slot.tolist()):
        assert torch.equal(p.k[0, s // page, :, s % page], x[t]) and torch.equal(p.v[0, s // page, :, s % page], 2 * x[t])


def roomy(p, S, **more):
    """A step over the same cache and tables in a pool of 70 MB and more, with a table as wide: what many rows over long prefixes
    take."""
    import torch
    pages = max(p.pages, -(-(70 << 20) // (4 * len(p.cached) * p.kv * p.D * p.page)))
    k, v = (torch.full((1, pages) + tuple(p.k.shape[2:]), math.nan, dtype=p.dtype, device="cuda:0") for _ in range(2))
    k[:, :p.pages], v[:, :p.pages] = p.k, p.v
    wide = np.full((len(p.cached), pages), -1)
    wide[:, :p.table.shape[1]] = p.table
    p.k, p.v, p.pages, p.table = k, v, pages, wide
    return p.step(S, **more)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("cached,fresh,heads,kv,D,kind", [
    ([700, 0, 129], [20, 40, 1], 8, 2, 128, "tree"),             # rows that end inside a wavefront's, chunks with idle wavefronts
    ([333], [256], 4, 2, 128, "tree"), ([90, 2000], [33, 2], 16, 2, 64, "any"), ([1000, 31], [30, 65], 12, 4, 96, "chain"),
    ([500, 7], [70, 18], 8, 2, 256, "tree"), ([3000], [100], 8, 1, 256, "any"), ([0, 64], [64, 70], 71, 1, 64, "tree")])
def test_many_rows_over_long_prefixes(S, dtype, cached, fresh, heads, kv, D, kind):
    p = Problem(cached, fresh, heads, kv, D, 16, dtype, kind)
    p.check(S.spqr_tree_attention(roomy(p, S), p.q))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("rows", [(15, 1), (16, 1), (3, 7), (31, 1), (32, 1), (11, 3), (8, 8), (64, 1), (13, 5)])
def test_every_number_of_rows_a_chunk_can_have(S, dtype, D, rows):
    """1 .. 16, 17 .. 32, 33 .. 64 and 65 rows of a key head, over prefixes that one launch takes and that are cut."""
    fresh, group = rows
    for cached in ([100, 3], [1500, 64]):
        p = Problem(cached, [fresh, 1], 2 * group, 2, D, 32, dtype, "tree", seed=fresh)
        p.check(S.spqr_tree_attention(p.step(S), p.q))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_pages_missing_and_values_masked_under_many_rows(S, D):
    """NaN in a sibling's value and missing pages, with rows of their own a wavefront."""
    import torch
    p = Problem([200, 90], [70, 40], 4, 2, D, 16, "float16", "tree")
    p.table[0, 2], p.table[1, 1] = -1, 10 ** 6
    vis = p.visible(0)
    j = next(k for k in range(201, 270) if vis[:, k].any() and not vis[:, k].all())
    want = S.spqr_tree_attention(roomy(p, S), p.q)
    p.check(want)
    p.v[0, p.table[0, j // 16], :, j % 16] = math.nan
    got = S.spqr_tree_attention(p.step(S), p.q)
    sees = torch.from_numpy(vis[:, j]).cuda()
    assert torch.equal(got[:70][~sees], want[:70][~sees]) and torch.equal(got[70:], want[70:])
    assert bool(torch.isnan(got[:70][sees]).all())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("D,group,fresh,page", [(64, 71, 3, 16), (96, 16, 5, 32), (128, 8, 40, 64), (256, 8, 9, 128)])
def test_tiles_shared_by_many_rows(S, dtype, D, group, fresh, page):
    """Many full tiles in a row, in a workgroup's part and over several: as they are, with a page missing in their middle, and with
    scores that grow along the prefix."""
    import torch
    p = Problem([6000, 777], [fresh, 1], 2 * group, 2, D, page, dtype, "tree", seed=D)
    step = roomy(p, S)
    p.check(S.spqr_tree_attention(step, p.q))
    p.table[0, 2000 // page] = -1
    step.table.copy_(i32(p.table))
    p.check(S.spqr_tree_attention(step, p.q))
    order = torch.arange(6000, dtype=torch.float64) / 6000
    for j in range(0, 6000, 3):
        if p.table[0, j // page] >= 0:
            p.k[0, p.table[0, j // page], 0, j % page] = (p.q[0, 0].double().cpu() * order[j] * 0.4).to(p.dtype).cuda()
    p.check(S.spqr_tree_attention(step, p.q))


def test_values_that_are_not_finite_come_through_shared_tiles(S):
    """A NaN and an infinity in cached values reach their elements of every row and no other element."""
    import torch
    for D in (64, 128, 256):
        p = Problem([900], [40], 8, 2, D, 16, "bfloat16", "tree")
        step = roomy(p, S)
        row = (0, p.table[0, 3], 1, 7)
        p.v[row][5], p.v[row][D - 2] = math.nan, -math.inf
        out = S.spqr_tree_attention(step, p.q)
        assert bool(torch.isnan(out[:, 4:, 5]).all()) and bool((out[:, 4:, D - 2] == -math.inf).all())
        rest = [d for d in range(D) if d not in (5, D - 2)]
        assert bool(torch.isfinite(out[:, 4:, rest]).all()) and bool(torch.isfinite(out[:, :4]).all())


@pytest.mark.parametrize("D", [64, 256])
def test_many_requests_of_many_rows(S, D):
    """As many requests as there can be, their list in LDS beside the tiles."""
    rng = np.random.default_rng(D)
    p = Problem(rng.integers(0, 90, 1024), rng.integers(0, 2, 1024), 80, 1, D, 16, "float16", "chain")
    p.check(S.spqr_tree_attention(roomy(p, S), p.q))


def test_many_rows_in_one_launch(S):
    """Short tables of many requests: nothing is cut, chunks of many rows."""
    rng = np.random.default_rng(3)
    p = Problem(rng.integers(0, 600, 110), rng.integers(0, 15, 110), 5, 1, 256, 16, "bfloat16", "tree")
    p.table = np.concatenate([p.table, np.full((110, 40 - p.table.shape[1]), -1)], axis=1)
    p.check(S.spqr_tree_attention(p.step(S, max_fresh=14), p.q))


def test_same_bits_every_time_on_any_stream_and_from_a_graph(S):
    import torch
    p = Problem([900, 20, 333], [16, 1, 9], 16, 4, 128, 16, "bfloat16", "tree")
    step = p.step(S)
    want = S.spqr_tree_attention(step, p.q)
    for _ in range(5):
        assert torch.equal(S.spqr_tree_attention(step, p.q), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(p.q)
    S.spqr_tree_attention(step, p.q, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    q = p.q.clone()
    out.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.spqr_tree_attention(step, q, out=out)
    for turn in range(4):
        q.copy_(p.q * (1.0 + turn))
        step.cached.copy_(i32([900 - 100 * turn, 20 + turn, 333 - turn]))
        eager = S.spqr_tree_attention(step, q)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
