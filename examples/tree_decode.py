"""Several sequences decoded with a small decoder whose matrices are in SpQR form, token by token and with trees of drafted tokens
that one pass verifies; both give the same tokens.

A step of either kind is, on one stream and without a copy to the host before its logits:

    spqr_cache_plan                        pages, slots, positions, masks of the new tokens
    spqr_adapter_plan                      the step's rows by their sequences' adapters
    per layer: spqr_gemm_fused             q, k, v
               spqr_adapters               ... and what a sequence's adapter adds to them
               spqr_cache_store            rotary embedding, keys and values to the cache
               spqr_tree_attention
               spqr_gemm_smallbatch, ...   o, gate and up, down
               spqr_residual_norm          norms, gates and sums between them
    spqr_token_logprobs                    the choice behind every new token, and how probable it is
    spqr_cache_keep                        the accepted path's rows move together, the lengths grow

Weights are random; every second sequence has one of two adapters.  The drafter guesses from the sequences that token-by-token decoding gave (right with a given probability a
token, wrong siblings beside it): it stands for a small model.

    python examples/tree_decode.py
"""
from __future__ import annotations

import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_03078_amd as P  # noqa: E402
import paper_2306_03078_amd.block_binding as K  # noqa: E402
import paper_2306_03078_amd.serve_binding as S  # noqa: E402
import spqr_synth as synth  # noqa: E402


class Decoder:
    """Embedding, layers of attention and gated feed-forward with SpQR matrices, head."""

    def __init__(self, layers=3, hidden=512, heads=8, kv_heads=4, ffn=1024, vocab=640, positions=512, seed=0):
        self.layers, self.hidden, self.heads, self.kv_heads, self.D = layers, hidden, heads, kv_heads, hidden // heads
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        self.embedding = torch.randn(vocab, hidden, device="cuda:0", generator=g)
        self.head = torch.randn(vocab, hidden, device="cuda:0", generator=g)

        def matrix(m, n, *key):
            return P.SpQRMatrix.from_logical(synth.make_matrix(m, n, w_bits=3, beta1=16, beta2=16, group_axis=1, outlier_rate=0.01,
                                                               outlier_structure="uniform", seed=(seed,) + key))
        kv = kv_heads * self.D
        self.blocks = [dict(qkv=[matrix(hidden, hidden, i, 0), matrix(kv, hidden, i, 1), matrix(kv, hidden, i, 2)], o=matrix(hidden, hidden, i, 3),
                            gate_up=[matrix(ffn, hidden, i, 4), matrix(ffn, hidden, i, 5)], down=matrix(hidden, ffn, i, 6)) for i in range(layers)]
        # two adapters of 16 ranks (the second of 5) beside q, k and v of each layer
        down = lambda: torch.randn(2, 16, hidden, device="cuda:0", generator=g).mul_(hidden ** -0.5).half()  # noqa: E731
        up = lambda m: torch.randn(2, m, 16, device="cuda:0", generator=g).half()  # noqa: E731
        self.ranks = torch.tensor([16, 5], dtype=torch.int32, device="cuda:0")
        self.adapters = [([down() for _ in range(3)], [up(m) for m in (hidden, kv, kv)]) for _ in range(layers)]
        # x; x + norm(y), both before the next block; norm(y); silu(g) * norm(y); and what the head takes
        norm = K.SpQRResidualNorm
        self.before, self.join = norm(hidden), norm(hidden, norm_y="rms")
        self.q_norm, self.k_norm, self.gate_norm = (norm(n, norm_y="rms", norm_x=None, out_dtype="float32") for n in (hidden, kv, ffn))
        self.gated, self.last = norm(ffn, norm_y="rms", norm_x=None, act="silu"), norm(hidden, norm_y="rms", out_dtype="float32")
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, self.D, 2, dtype=torch.float64) / self.D)
        self.rotary = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()

    def step(self, requests, tokens, length, max_fresh, page=16):
        """A step of up to `tokens` rows for `requests` sequences of up to `length` tokens, and the cache for them."""
        width = -(-length // page)
        k, v = (torch.zeros(self.layers, requests * width, self.kv_heads, page, self.D, dtype=torch.float16, device="cuda:0") for _ in range(2))
        return S.SpQRStep(k, v, self.heads, requests=requests, tokens=tokens, max_pages=width, mask_words=-(-max_fresh // 64), max_fresh=max_fresh,
                          rotary=self.rotary, parent=torch.full((tokens,), -1, dtype=torch.int32, device="cuda:0"))

    def banks(self, rows):
        """The layers' adapters for steps of up to `rows` rows; one scratch for all."""
        banks = []
        for A, B in self.adapters:
            banks.append(K.SpQRAdapters(A, B, rank=self.ranks, rows=rows, workspace=banks[0].workspace if banks else None))
        return banks

    def logits(self, step, tokens, banks, plan):
        """The planned step's rows: tokens [rows] -> [rows, vocab].  (Rows that belong to no sequence give anything.)"""
        norm = K.spqr_residual_norm
        x = self.embedding[tokens]
        _, h = norm(self.before, x)
        for i, block in enumerate(self.blocks):
            q, k, v = P.spqr_gemm_fused(block["qkv"], h)
            K.spqr_adapters(banks[i], plan, h, [q, k, v], outs=[q, k, v])
            q = S.spqr_cache_store(step, norm(self.q_norm, y=q)[1], norm(self.k_norm, y=k)[1], v / self.hidden ** 0.5, layer=i)
            a = S.spqr_tree_attention(step, q, layer=i, out=torch.zeros_like(q))
            x, h = norm(self.join, x, P.spqr_gemm_smallbatch(block["o"], a.view(len(tokens), -1)))
            gate, up = P.spqr_gemm_fused(block["gate_up"], h)
            _, h = norm(self.gated, y=up, gate=norm(self.gate_norm, y=gate)[1])
            x, h = norm(self.join if i + 1 < self.layers else self.last, x, P.spqr_gemm_smallbatch(block["down"], h))
        return h @ self.head.T


class Session:
    """Sequences over one cache.  Each call gives, per sequence, the new tokens' ids and their parents."""

    def __init__(self, model, requests, tokens, length, max_fresh):
        self.model, self.step = model, model.step(requests, tokens, length, max_fresh)
        self.banks, self.plan = model.banks(tokens), K.SpQRAdapterPlan(tokens, 2)
        self.adapter = torch.tensor([r // 2 % 2 if r % 2 == 0 else -1 for r in range(requests)], dtype=torch.int32, device="cuda:0")
        self.scores = K.SpQRScores(tokens, model.embedding.shape[0], given=0, top=1)

    def verify(self, ids, parents):
        """Greedy choice behind every new token, as lists per sequence; the step stays open until keep()."""
        step, flat = self.step, sum(ids, [])
        tree = sum(parents, [])
        pad = step.tokens - len(flat)
        step.fresh.copy_(torch.tensor([len(x) for x in ids], dtype=torch.int32))
        step.parent.copy_(torch.tensor(tree + [-1] * pad, dtype=torch.int32))
        S.spqr_cache_plan(step)
        K.spqr_adapter_plan(self.plan, self.adapter, step.q_start)
        self.best = self.model.logits(step, torch.tensor(flat + [0] * pad, device="cuda:0"), self.banks, self.plan)
        choice = K.spqr_token_logprobs(self.scores, self.best).top_token[:, 0].tolist()
        if int(step.ends_out[2]):
            raise RuntimeError(f"the cache lacks {int(step.ends_out[2])} pages")
        starts = np.cumsum([0] + [len(x) for x in ids])
        return [choice[starts[r]:starts[r + 1]] for r in range(len(ids))]

    def keep(self, last=None):
        S.spqr_cache_keep(self.step, None if last is None else torch.tensor(last, dtype=torch.int32, device="cuda:0"))
        self.step.advance()


def chain(n):
    return list(range(-1, n - 1))


def token_by_token(model, prompts, count, capacity):
    """`count` tokens behind each prompt, and how far each choice's logit is from the second best."""
    s = Session(model, len(prompts), capacity, max(map(len, prompts)) + count + 64, max(map(len, prompts)))
    got = [[c[-1]] for c in s.verify(prompts, [chain(len(p)) for p in prompts])]
    s.keep()
    ahead = [[math.inf] for _ in got]
    for _ in range(count - 1):
        choices = s.verify([[x[-1]] for x in got], [[-1]] * len(got))
        two = s.best[:len(got)].topk(2, 1).values
        for x, a, c, d in zip(got, ahead, choices, (two[:, 0] - two[:, 1]).tolist()):
            x.append(c[0])
            a.append(d)
        s.keep()
    return got, ahead


def draft(rng, root, continuation, depth, width, vocab, right):
    """A tree under `root`: at each depth one guess and width - 1 siblings, the next depth under one of them."""
    ids, parents, at = [root], [-1], 0
    for d in range(min(depth, len(continuation))):
        guess = [int(rng.integers(0, vocab)) for _ in range(width)]
        place = int(rng.integers(0, width))
        if rng.random() < right:
            guess[place] = continuation[d]
        parents += [at] * width
        at = len(ids) + place
        ids += guess
    return ids, parents


def with_trees(model, prompts, known, count, capacity, depth=4, width=3, right=0.8, seed=0):
    """The same tokens by verifying trees; also the number of passes.  `known`: what the drafter guesses from."""
    rng = np.random.default_rng(seed)
    vocab = model.embedding.shape[0]
    s = Session(model, len(prompts), capacity, max(map(len, prompts)) + count + 64, max(max(map(len, prompts)), 1 + depth * width))
    got = [[c[-1]] for c in s.verify(prompts, [chain(len(p)) for p in prompts])]
    s.keep()
    passes = 0
    while min(map(len, got)) < count:
        trees = [draft(rng, x[-1], k[len(x):], depth, width, vocab, right) for x, k in zip(got, known)]
        choices = s.verify([t[0] for t in trees], [t[1] for t in trees])
        last = []
        for x, (ids, parents), choice in zip(got, trees, choices):
            at = 0
            while True:                      # down the tree as long as a child is what the model chose
                x.append(choice[at])
                below = [i for i in range(at + 1, len(ids)) if parents[i] == at and ids[i] == choice[at]]
                if not below or len(x) >= count:
                    break
                at = below[0]
            last.append(at)
        s.keep(last)
        passes += 1
    return [x[:count] for x in got], passes


def main(count=40, requests=3, seed=0):
    model = Decoder(seed=seed)
    rng = np.random.default_rng([seed, 1])
    prompts = [rng.integers(0, 640, n).tolist() for n in rng.integers(3, 14, requests)]
    capacity = 16 * requests
    plain, ahead = token_by_token(model, prompts, count, capacity)
    trees, passes = with_trees(model, prompts, plain, count, capacity)
    same = sum(x == y for x, y in zip(plain, trees))
    print(f"{requests} sequences, {count} tokens each: {count - 1} passes token by token, {passes} with trees; "
          f"{same} of {requests} give the same tokens (the closest second choice: {min(map(min, ahead)):.3f} behind)")
    return plain, trees, ahead, passes


if __name__ == "__main__":
    main()
