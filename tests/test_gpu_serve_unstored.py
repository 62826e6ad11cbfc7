"""New tokens that are not stored (no page for them, no row of the rotary table, no slot) and what later steps make of it: the
lengths behind a step cover stored tokens only, so that nobody attends to rows that nobody wrote."""
import math

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
PAGE, D = 16, 64


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


def i32(a):
    import torch
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).to("cuda:0").contiguous()


class Sequences:
    """Two sequences, one key head of two query heads, over four pages of NaN; what was stored is kept on the host beside it."""

    def __init__(self, S, words, rotary=None, width=4, pages=4):
        import torch
        self.S, self.g = S, torch.Generator(device="cuda:0").manual_seed(11)
        self.k, self.v = (torch.full((1, pages, 1, PAGE, D), math.nan, dtype=torch.float16, device="cuda:0") for _ in range(2))
        self.words = words
        self.parent = i32([-1] * 64) if words else None
        self.step = S.SpQRStep(self.k, self.v, 2, requests=2, tokens=64, max_pages=width, mask_words=words, parent=self.parent, rotary=rotary)
        self.stored = [[], []]               # (k, v) of each token that counts, 64 bits

    def plan(self, fresh, parents=None):
        step = self.step
        step.fresh.copy_(i32(fresh))
        if self.words:
            flat = [p for n, ps in zip(fresh, parents or [None] * 2) for p in (ps or range(-1, n - 1))]
            step.parent[:len(flat)] = i32(flat)
        self.S.spqr_cache_plan(step)
        self.start = [0, fresh[0]]

    def store(self):
        """q as the attention takes it."""
        import torch
        q, k, v = (torch.randn(64, h, D, generator=self.g, device="cuda:0").half() for h in (2, 1, 1))
        return self.S.spqr_cache_store(self.step, q, k, v)

    def row(self, token):
        """(k, v) that the cache holds in the token's slot, as written; None without a slot."""
        slot = int(self.step.slot[token])
        return None if slot < 0 else tuple(c[0, slot // PAGE, 0, slot % PAGE].double().cpu() for c in (self.k, self.v))

    def check(self, q, out, r, i, news):
        """Row i of r against the formula over what is stored and its new tokens `news`.  The bound: probabilities rounded to
        f16 (2^-11, 2^-25 below the normal range), the result rounded once; scores in binary32, off by less than 2^-13."""
        import torch
        keys = self.stored[r] + [self.rows[r][j] for j in news]
        K, V = (torch.stack([x[n] for x in keys]) for n in (0, 1))
        p = torch.softmax(q[self.start[r] + i].double().cpu() @ K.T / 8.0, 1)
        got = out[self.start[r] + i].double().cpu()
        bound = (2.0 ** -11 + 2.0 ** -12) * (p @ V.abs()) + 2.0 ** -11 * (p @ V).abs() + 2.0 ** -25 * (V.abs().sum(0) + 1)
        assert bool(torch.isfinite(got).all())
        assert bool(((got - p @ V).abs() <= bound).all())

    def keep(self, last, paths):
        got = self.S.spqr_cache_keep(self.step, None if last is None else i32(last)).tolist()
        for r, path in enumerate(paths):
            self.stored[r] += [self.rows[r][j] for j in path]
        assert got == [len(x) for x in self.stored]
        self.step.advance()

    def turn(self, fresh, last, paths, parents=None):
        """A step whose accepted and stored tokens are `paths`, each of which sees those before it."""
        self.plan(fresh, parents)
        q = self.store()
        self.rows = [[self.row(self.start[r] + j) for j in range(n)] for r, n in enumerate(fresh)]       # before anything moves
        out = self.S.spqr_tree_attention(self.step, q)
        for r, path in enumerate(paths):
            for n, i in enumerate(path):
                self.check(q, out, r, i, path[:n + 1])
        self.keep(last, paths)


@pytest.mark.parametrize("form", ["masks", "masks-all", "no-masks", "no-masks-all", "tree"])
def test_a_ring_that_runs_dry(S, form):
    """Tokens behind the last page do not count in any form of the call; when a page comes back, with another sequence's rows or
    NaN in it, it is filled before it is seen."""
    s = Sequences(S, 0 if form.startswith("no-masks") else 1)
    s.turn([45, 10], None, [list(range(45)), list(range(10))])
    assert s.step.ends.tolist()[:2] == [4, 4]
    if form == "tree":           # keys 45 ..: 0, its children 1 and 2; 3 under 1, 4 under 2, 5 under 4; from 3 on there is no page
        parents = [[-1, 0, 0, 1, 2, 4], [-1]]
        last, paths, fresh = [5, 0], [[0, 2], [0]], [6, 1]
    else:
        parents, fresh = None, [6, 1]
        last, paths = None if form.endswith("all") else [5, 0], [[0, 1, 2], [0]]
    s.turn(fresh, last, paths, parents)
    kept = 47 if form == "tree" else 48
    assert s.step.cached.tolist() == [kept, 11]
    # the second sequence ends; its page holds its rows, the rest of it NaN
    gone = int(s.step.table[1, 0])
    s.step.cached[1] = 0
    s.stored[1] = []
    s.plan([0, 0])
    s.keep(None, [[], []])
    s.k[0, gone, 0, 12:], s.v[0, gone, 0, 12:] = math.nan, math.nan
    s.turn([3, 0], None, [[0, 1, 2], []])
    assert int(s.step.table[0, 3]) == gone and s.step.cached.tolist() == [kept + 3, 0]


def test_the_same_from_a_table_that_is_too_narrow(S):
    """Keys behind the table's last column have no page; the length stays at what the table holds."""
    s = Sequences(S, 1, width=2)
    s.turn([30, 3], None, [list(range(30)), list(range(3))])
    s.turn([5, 1], [4, 0], [[0, 1], [0]])
    s.turn([4, 1], None, [[], [0]])
    assert s.step.cached.tolist() == [32, 5]


@pytest.mark.parametrize("words,every", [(1, False), (1, True), (0, False), (0, True)])
def test_positions_behind_the_rotary_table(S, words, every):
    import torch
    angle = torch.arange(20, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    rotary = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
    s = Sequences(S, words, rotary=rotary)
    s.turn([18, 4], None, [list(range(18)), list(range(4))])
    s.turn([4, 2], None if every else [3, 1], [[0, 1], [0, 1]])
    assert s.step.cached.tolist() == [20, 6]
    s.turn([3, 1], None, [[], [0]])


def test_a_branch_that_is_too_deep_and_one_that_is_not(S):
    import torch
    rotary = torch.cat([torch.ones(20, D // 2), torch.zeros(20, D // 2)], 1).cuda()
    for last, path in (([3, 0], [0, 2]), ([4, 0], [0, 4])):
        s = Sequences(S, 1, rotary=rotary)
        s.turn([18, 1], None, [list(range(18)), [0]])
        s.turn([5, 1], last, [path, [0]], parents=[[-1, 0, 0, 2, 0], [-1]])
        assert s.step.cached.tolist() == [20, 2]


@pytest.mark.parametrize("words", [0, 1])
def test_slots_and_positions_that_a_caller_takes_away(S, words):
    for what in ("slot", "position"):
        s = Sequences(S, words)
        s.plan([6, 3])
        getattr(s.step, what)[3] = -1
        s.store()
        got = S.spqr_cache_keep(s.step, i32([5, 2]))
        assert got.tolist() == [3, 3]
        assert S.spqr_cache_keep(s.step).tolist() == [3, 3]
        assert S.spqr_cache_keep(s.step, i32([2, -1])).tolist() == [3, 0]
        setattr(s.step.desc, what, None)                     # not looked at
        assert S.spqr_cache_keep(s.step, i32([5, 2])).tolist() == [6, 3]


def test_addresses_that_are_not_aligned_are_refused(S):
    from paper_2306_03078_amd import SpQRError
    for what in ("slot", "position"):
        s = Sequences(S, 1)
        setattr(s.step.desc, what, getattr(s.step, what).data_ptr() + 2)
        with pytest.raises(SpQRError):
            S.spqr_cache_keep(s.step)
