"""A block of a decoder's step with its norms, adapters and log probabilities as they are used one after another: against 64 bits, and out of
a graph that is replayed with other requests, tokens and adapters."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd as P  # noqa: E402
import paper_2306_03078_amd.block_binding as K  # noqa: E402
import spqr_synth as synth  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
HIDDEN, FFN, VOCAB, ROWS, SLOTS = 256, 512, 1000, 24, 3


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Block:
    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(0)
        self.fs = [synth.make_matrix(m, n, w_bits=3, beta1=16, beta2=16, group_axis=1, outlier_rate=0.01, outlier_structure="uniform", seed=(3, i))
                   for i, (m, n) in enumerate(((FFN, HIDDEN), (FFN, HIDDEN), (HIDDEN, FFN)))]
        self.matrices = [P.SpQRMatrix.from_logical(f) for f in self.fs]
        self.dense = [P.spqr_dequant_dense(m, P.SPQR_OUT_DENSE_F32 | P.SPQR_OUT_WITH_OUTLIERS).double() for m in self.matrices]
        self.A = [torch.randn(SLOTS, 8, HIDDEN, device="cuda", generator=g).mul_(HIDDEN ** -0.5).half() for _ in range(2)]
        self.B = [torch.randn(SLOTS, FFN, 8, device="cuda", generator=g).half() for _ in range(2)]
        self.rank, self.scale = ints([8, 3, 8]), torch.tensor([1.0, 0.5, 2.0], device="cuda")
        self.bank = K.SpQRAdapters(self.A, self.B, rank=self.rank, scale=self.scale, rows=ROWS)
        self.plan = K.SpQRAdapterPlan(ROWS, SLOTS)
        self.w = 1 + 0.1 * torch.randn(HIDDEN, device="cuda", generator=g)
        self.before, self.after = K.SpQRResidualNorm(HIDDEN, x_weight=self.w), K.SpQRResidualNorm(HIDDEN, norm_y="rms", norm_x="rms", scale=0.5, out_dtype="float32")
        self.each, self.gated = K.SpQRResidualNorm(FFN, norm_y="rms", norm_x=None, out_dtype="float32"), K.SpQRResidualNorm(FFN, norm_y="rms", norm_x=None, act="silu")
        self.head = torch.randn(VOCAB, HIDDEN, device="cuda", generator=g) / 4
        self.scores = K.SpQRScores(ROWS, VOCAB, given=2, top=5)
        self.scratch = torch.empty(max(256, P.spqr_workspace_bytes(self.matrices[:2], ROWS), P.spqr_workspace_bytes(self.matrices[2], ROWS)), dtype=torch.uint8, device="cuda")

    def run(self, x, adapter, q_start, tokens):
        K.spqr_adapter_plan(self.plan, adapter, q_start)
        _, h = K.spqr_residual_norm(self.before, x)
        gate, up = P.spqr_gemm_fused_ws(self.matrices[:2], h, self.scratch)
        K.spqr_adapters(self.bank, self.plan, h, [gate, up], outs=[gate, up])
        _, f = K.spqr_residual_norm(self.gated, y=up, gate=K.spqr_residual_norm(self.each, y=gate)[1])
        y = P.spqr_gemm_smallbatch_ws(self.matrices[2], f, self.scratch)
        s, out = K.spqr_residual_norm(self.after, x, y)
        K.spqr_token_logprobs(self.scores, out @ self.head.T, tokens)
        return [s, self.scores.logprob, self.scores.entropy, self.scores.top_token, self.scores.top_logprob]

    def plain(self, x, adapter, q_start, tokens):
        rms = lambda v: v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
        x = x.double()
        h = rms(x) * self.w.double()
        both = []
        for p in range(2):
            v = h @ self.dense[p].T
            for r, a in enumerate(adapter.tolist()):
                if 0 <= a < SLOTS:
                    k, at = int(self.rank[a]), slice(int(q_start[r]), int(q_start[r + 1]))
                    v[at] += float(self.scale[a]) * h[at] @ self.A[p][a, :k].double().T @ self.B[p][a, :, :k].double().T
            both.append(rms(v))
        s = x + 0.5 * rms((both[0] * torch.sigmoid(both[0]) * both[1]) @ self.dense[2].T)
        logp = torch.log_softmax(rms(s) @ self.head.double().T, 1)
        return s, logp.gather(1, tokens.long()), -(logp.exp() * logp).sum(1), logp


def inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(ROWS, HIDDEN, device="cuda", generator=g) * 3
    tokens = torch.randint(0, VOCAB, (ROWS, 2), dtype=torch.int32, device="cuda", generator=g)
    lengths = [(1, 7, 0, 16), (16, 1, 1, 2), (5, 5, 5, 5)][seed % 3]
    q = [0]
    for n in lengths:
        q.append(q[-1] + n)
    return x, ints([(seed + r) % 4 - 1 for r in range(4)]), ints(q), tokens


def test_a_block_against_64_bits():
    """h, f and the products' inputs are binary16 (2^-11 of each element, of random signs: a share of 2^-11 of a product's size, some times over in a
    chain of three products, norms that bring it back to size 1, logits of size 4): 40 * 2^-11 of the values' size."""
    block = Block()
    for seed in range(3):
        x, adapter, q, tokens = inputs(seed)
        s, logprob, entropy, top, top_logprob = block.run(x, adapter, q, tokens)
        used = int(q[-1])
        want_s, want, want_entropy, logp = block.plain(x, adapter, q, tokens)
        tol = 40 * 2.0 ** -11
        assert (s - want_s)[:used].abs().max() <= tol * want_s.abs().max()
        assert (logprob - want)[:used].abs().max() <= tol * 4 and (entropy - want_entropy)[:used].abs().max() <= tol * 4
        found = logp.gather(1, top.long())
        assert (top_logprob - found)[:used].abs().max() <= tol * 4
        assert (found[:, 0] >= logp.amax(1) - 2 * tol * 4)[:used].all()


def test_a_block_out_of_a_graph():
    block = Block()
    x, adapter, q, tokens = inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.run(x, adapter, q, tokens)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = block.run(x, adapter, q, tokens)
    torch.cuda.synchronize()
    other = Block()                                      # eager work of other handles between the replays
    for seed in (0, 1, 2, 1, 0):
        for to, new in zip((x, adapter, q, tokens), inputs(seed)):
            to.copy_(new)
        want = [v.clone() for v in other.run(x, adapter, q, tokens)]
        for v in outs:
            v.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        used = int(q[-1])
        for a, b in zip(outs, want):
            if a.dtype == torch.int32:
                continue                                 # (near ties may change places with the last bits of the products)
            assert math.isfinite(float(a[:used].abs().max())) and (a - b)[:used].abs().max() <= 1e-3 * max(1.0, float(b[:used].abs().max()))
