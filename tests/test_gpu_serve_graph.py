"""A whole decode step in one HIP graph, replayed with other lengths, trees and values, against the same calls made one by one."""
import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
R, TOKENS, LAYERS, HEADS, KV, PAGE, D, PAGES, WIDTH = 3, 24, 2, 4, 2, 16, 64, 40, 12


@pytest.fixture(scope="module")
def S():
    import paper_2306_03078_amd.serve_binding as S
    S._lib()
    return S


class Decode:
    """A step's arrays and the calls on them; the lengths go from cached_out back to cached by a copy, so that addresses stay."""

    def __init__(self, S):
        import torch
        self.S = S
        g = torch.Generator(device="cuda:0").manual_seed(4)
        self.k, self.v = (torch.randn(LAYERS, PAGES, KV, PAGE, D, device="cuda:0", generator=g).half() for _ in range(2))
        angle = torch.arange(WIDTH * PAGE, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        self.step = S.SpQRStep(self.k, self.v, HEADS, requests=R, tokens=TOKENS, max_pages=WIDTH, mask_words=1, max_fresh=8,
                               parent=torch.full((TOKENS,), -1, dtype=torch.int32, device="cuda:0"),
                               rotary=torch.cat([angle.cos(), angle.sin()], 1).float().cuda())
        self.rows = torch.zeros(TOKENS, (HEADS + 2 * KV) * D, device="cuda:0")
        self.last = torch.zeros(R, dtype=torch.int32, device="cuda:0")
        self.q, self.out = (torch.zeros(TOKENS, HEADS, D, dtype=torch.float16, device="cuda:0") for _ in range(2))

    def calls(self):
        step, x = self.step, self.rows
        self.S.spqr_cache_plan(step)
        for layer in range(LAYERS):
            self.S.spqr_cache_store(step, x[:, :HEADS * D], x[:, HEADS * D:(HEADS + KV) * D], x[:, (HEADS + KV) * D:], layer=layer, out=self.q)
            self.S.spqr_tree_attention(step, self.q, layer=layer, out=self.out)
        self.S.spqr_cache_keep(step, self.last)
        step.cached.copy_(step.cached_out)
        step.held.copy_(step.held_out)
        step.ends.copy_(step.ends_out)

    def inputs(self, turn):
        import torch
        rng = np.random.default_rng([turn, 9])
        fresh = rng.integers(0, 9, R)
        parents = [int(rng.integers(-1, i)) if i else -1 for n in fresh for i in range(n)]
        self.step.fresh.copy_(torch.tensor(fresh, dtype=torch.int32))
        self.step.parent.copy_(torch.tensor(parents + [-1] * (TOKENS - len(parents)), dtype=torch.int32))
        self.last.copy_(torch.tensor([int(rng.integers(-1, n + 1)) for n in fresh], dtype=torch.int32))
        self.rows.copy_(torch.from_numpy(rng.standard_normal(self.rows.shape).astype(np.float32)))
        last, at, paths = self.last.tolist(), 0, []
        for n, leaf in zip(fresh, last):         # lengths of the accepted paths, by the parents
            here, at, length = parents[at:at + n], at + n, 0
            while 0 <= leaf < n:
                leaf, length = here[leaf], length + 1
            paths.append(length)
        if turn % 4 == 3:        # all sequences end, their pages go back
            self.step.cached.zero_()
            self.step.fresh.zero_()
            return None
        return paths

    def state(self):
        s = self.step
        used = int(s.q_start[R])
        return [s.cached, s.held, s.ends, s.q_start, s.position, s.slot, s.mask, s.table, s.pool, self.k, self.v, self.q, self.out[:used]]


def test_a_step_from_a_graph(S):
    import torch
    one, other = Decode(S), Decode(S)
    one.inputs(0)
    other.inputs(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.calls()
    lengths = [0] * R
    for turn in range(12):
        paths = [d.inputs(turn) for d in (one, other)][0]
        lengths = [0] * R if paths is None else [a + b for a, b in zip(lengths, paths)]
        one.calls()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(one.state(), other.state()):
            assert torch.equal(a, b)
        assert one.step.cached.tolist() == lengths
