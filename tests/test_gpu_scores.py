"""Log probabilities, entropy and most probable tokens of rows of logits, against 64 bits.

Tolerance.  The sum of e^(z - max) has at most vocab / 256 terms in a row and some 40 partial sums; an exponential is off by 2^-23 and by the
roundings of its argument, 2 * 2^-24 of its size d.  With D1, D2 the means of |d|, d^2 over the softmax: the logarithm of the sum is off by
(vocab / 256 + 100 + 2 D1) 2^-24, the mean of d by (vocab / 256 + 100) 2^-24 D1 + 4 * 2^-24 D2 more; then half a step of binary32."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


def same(got, want, bound):
    assert got.shape == want.shape
    inf = want < -3.4028236e38           # rounds to -infinity: 1.9 times the lowest binary32 number is -6.5e38
    assert torch.equal(got == -math.inf, inf)
    off = (got.double() - want).abs()[~inf]
    allowed = (bound.expand_as(want) + U * want.abs())[~inf] + 1e-37
    bad = ~(off <= allowed)
    assert not bad.any(), (int(bad.sum()), float((off / allowed).max()))


def check(logits, tokens, top, scale=1.0, scores=None):
    rows, vocab = logits.shape
    given = 0 if tokens is None else tokens.shape[1]
    s = scores or K.SpQRScores(rows, vocab, given=given, top=top)
    for t in (s.logprob, s.entropy, s.top_token, s.top_logprob):
        t.fill_(12345)
    K.spqr_token_logprobs(s, logits, tokens, scale=scale)
    z = logits.double() * float(torch.tensor(scale, dtype=torch.float32))
    empty = (z == -math.inf).all(1, keepdim=True)
    d = torch.where(empty, -math.inf, z - z.amax(1, keepdim=True))
    e = d.exp()
    total = torch.where(empty, 1.0, e.sum(1, keepdim=True))
    lse, p = total.log(), e / total
    d1 = torch.where(p > 0, p * d.abs(), 0.0).sum(1, keepdim=True)
    d2 = torch.where(p > 0, p * d * d, 0.0).sum(1, keepdim=True)
    terms = vocab / 256 + 100
    logp = d - lse
    entropy = torch.where(p > 0, -p * logp, 0.0).sum(1)
    same(s.entropy[:rows], entropy, ((terms + 2 * d1) * U + terms * U * d1 + 4 * U * d2)[:, 0])
    bound = (terms + 2 * d1) * U
    if given:
        inside = (tokens >= 0) & (tokens < vocab)
        want = torch.where(inside, logp.gather(1, tokens.long().clamp(0, vocab - 1)), 0.0)
        same(s.logprob[:rows], want, bound)
    if top:
        # by value, then by id: a stable sort
        order = torch.sort(logits.double(), dim=1, descending=True, stable=True)
        k = min(top, vocab)
        ids = torch.where(order.values[:, :k] > -math.inf, order.indices[:, :k], -1)
        ids = torch.nn.functional.pad(ids, (0, top - k), value=-1)
        assert torch.equal(s.top_token[:rows].long(), ids)
        want = torch.where(ids >= 0, logp.gather(1, ids.clamp(min=0)), -math.inf)
        same(s.top_logprob[:rows], want, bound)
    return s


def draw(rows, vocab, dtype="f32", seed=0, size=3.0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = (torch.randn(rows, vocab + pad, generator=g, device="cuda") * size).to(TYPES[dtype])[:, :vocab]
    return logits, lambda given: torch.randint(0, vocab, (rows, given), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 64, 65, 500, 511, 512, 513, 2047, 2048, 4099, 8191, 8192, 8193, 16385, 32000, 50000, 65537, 128000, 256001])
def test_vocabularies(vocab, dtype):
    logits, tokens = draw(3, vocab, dtype, seed=vocab)
    check(logits, tokens(2), 10)
    check(logits[:1], tokens(1)[:1], 64, scale=0.7)


@pytest.mark.parametrize("rows", [1, 2, 3, 8, 17, 100, 256, 300, 1000, 3000])
def test_rows(rows):
    for vocab, dtype in ((1000, "f32"), (9001, "bf16"), (33000, "f16")):
        logits, tokens = draw(rows, vocab, dtype, seed=rows)
        check(logits, tokens(1), 5)


@pytest.mark.parametrize("rows,vocab", [(1024, 20001), (1025, 20001), (1100, 8193), (1030, 49152), (1030, 49153)])
def test_many_rows_of_middling_length(rows, vocab):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    logits = (torch.randn(rows, vocab, device="cuda", generator=g) * 3).half()
    check(logits, torch.randint(0, vocab, (rows, 2), dtype=torch.int32, device="cuda", generator=g), 7)


@pytest.mark.parametrize("top", [0, 1, 2, 5, 16, 31, 32, 33, 63, 64])
def test_alternatives(top):
    for rows, vocab in ((1, 32000), (5, 70000), (40, 3001), (3, 40)):
        logits, tokens = draw(rows, vocab, "f32", seed=top)
        check(logits, tokens(3), top)
        logits, tokens = draw(rows, vocab, "bf16", seed=top, size=0.5)       # many equal ones
        check(logits, None, top)


@pytest.mark.parametrize("given", [0, 1, 2, 64])
def test_given_tokens(given):
    logits, tokens = draw(6, 5000, seed=given)
    t = tokens(given) if given else None
    check(logits, t, 3)
    if given:
        t[0, 0], t[3, given - 1], t[5, 0] = -1, 5000, -2 ** 31
        s = check(logits, t, 0)
        assert s.logprob[0, 0] == 0 and s.logprob[3, given - 1] == 0


@pytest.mark.parametrize("pad", [1, 7, 8, 64])
def test_rows_of_wider_tensors_at_any_address(pad):
    for dtype in ("f32", "f16", "bf16"):
        logits, tokens = draw(9, 1003, dtype, seed=pad, pad=pad)
        check(logits, tokens(1), 7)
        wide, tokens = draw(3, 65000, dtype, seed=pad, pad=pad + 1)
        check(wide[:, 1:64001], tokens(1) % 64000, 7)


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 0.5, 1.0, 1.7, 30.0, 1e6])
def test_scales(scale):
    for rows in (2, 300):
        logits, tokens = draw(rows, 20000, "f32", seed=3)
        check(logits, tokens(2), 12, scale=scale)


@pytest.mark.parametrize("rows,vocab", [(1, 100000), (20, 3000), (300, 3000), (2, 600)])
def test_masks(rows, vocab):
    g = torch.Generator(device="cuda").manual_seed(rows)
    for dtype in ("f32", "f16", "bf16"):
        lowest = torch.finfo(TYPES[dtype]).min
        for kind in ("half", "seven", "one", "none", "lowest", "lowest-all", "range", "tail"):
            logits, tokens = draw(rows, vocab, dtype, seed=rows)
            if kind == "half":
                logits[torch.rand(rows, vocab, generator=g, device="cuda") < 0.5] = -math.inf
            elif kind in ("seven", "one"):
                keep = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
                keep.scatter_(1, tokens(7 if kind == "seven" else 1).long(), True)
                logits[~keep] = -math.inf
            elif kind == "none":
                logits[:] = -math.inf
            elif kind == "lowest":
                logits[torch.rand(rows, vocab, generator=g, device="cuda") < 0.9] = lowest
            elif kind == "lowest-all":
                logits[:] = lowest
            elif kind == "range":
                logits[:, 100:] = -math.inf
            else:
                logits[:, :-5] = -math.inf
            for top in (0, 5, 40):
                check(logits, tokens(3), top, scale=1.0 if kind != "lowest" else 1.9)


def test_equal_logits_and_zeros_of_both_signs():
    for rows, vocab in ((1, 50000), (3, 1000), (300, 2500), (2, 200000)):
        for value in (0.0, -7.25, 3.0):
            logits = torch.full((rows, vocab), value, device="cuda")
            check(logits, None, 40)
            logits[:, vocab // 2:] = value + 1
            check(logits.half(), None, 64)
        zeros = torch.zeros(rows, vocab, device="cuda")
        zeros[:, ::3] = -0.0
        check(zeros, None, 20)
        steps = (torch.arange(vocab, device="cuda") % 97).float().expand(rows, vocab).contiguous()
        check(steps, None, 64)
        check(torch.arange(vocab, device="cuda").float().expand(rows, vocab).contiguous() / vocab, None, 64)
        check(-torch.arange(vocab, device="cuda").float().expand(rows, vocab).contiguous() / vocab, None, 64)


def test_large_logits():
    logits, tokens = draw(4, 30000, "f32", seed=5, size=1e4)
    check(logits, tokens(4), 9)
    logits[1] += 1e30
    logits[2] *= 1e30
    check(logits, tokens(4), 9)
    logits[3] = -3e38
    logits[3, 77] = 3e38
    check(logits, tokens(4), 9)


@pytest.mark.parametrize("rows,vocab", [(1, 90000), (5, 700), (300, 2000)])
def test_nan_and_infinity_stay_in_their_row(rows, vocab):
    logits, tokens = draw(rows + 2, vocab, "f32", seed=rows)
    t = tokens(1)
    s = K.SpQRScores(rows + 2, vocab, given=1, top=5)
    want = [v.clone() for v in (lambda o: (o.logprob, o.entropy, o.top_token, o.top_logprob))(K.spqr_token_logprobs(s, logits, t))]
    bad = logits.clone()
    bad[0, vocab // 2], bad[rows + 1, vocab - 1] = math.nan, math.inf
    K.spqr_token_logprobs(s, bad, t)
    for r in (0, rows + 1):
        assert s.logprob[r].isnan().all() and s.entropy[r].isnan() and s.top_logprob[r].isnan().all()
    assert s.top_token[rows + 1, 0] == vocab - 1
    without = bad[0].clone()
    without[vocab // 2] = -math.inf
    assert torch.equal(s.top_token[0].long(), without.topk(5).indices)
    for a, b in zip((s.logprob, s.entropy, s.top_token, s.top_logprob), want):
        assert torch.equal(a[1:rows + 1], b[1:rows + 1])


def test_fewer_rows_than_the_handle_has_room_for():
    s = K.SpQRScores(50, 4000, given=1, top=3)
    for rows in (50, 1, 7, 33):
        logits, tokens = draw(rows, 4000, seed=rows)
        check(logits, tokens(1), 3, scores=s)
        assert (s.entropy[rows:] == 12345).all() and (s.top_token[rows:] == 12345).all() and (s.logprob[rows:] == 12345).all()
    before = s.entropy.clone()
    K.spqr_token_logprobs(s, torch.zeros(0, 4000, device="cuda"), torch.zeros(0, 1, dtype=torch.int32, device="cuda"))
    assert torch.equal(s.entropy, before)


def test_offsets_beyond_32_bits():
    """Rows whose distance times their number passes 2^31 elements (bf16, 4.3 GB)."""
    wide = torch.zeros(9, 1 << 28, dtype=torch.bfloat16, device="cuda")
    logits = wide[:, 5:5 + 1000]
    logits.copy_(torch.randn(9, 1000, device="cuda") * 3)
    check(logits, torch.arange(9, dtype=torch.int32, device="cuda")[:, None].contiguous(), 4)


def test_another_stream_and_a_captured_call():
    for rows, vocab in ((2, 60000), (64, 3000)):
        logits, tokens = draw(rows, vocab, "f16", seed=1)
        other, _ = draw(rows, vocab, "f16", seed=2)
        t = tokens(1)
        s, s2 = K.SpQRScores(rows, vocab, top=7), K.SpQRScores(rows, vocab, top=7)
        every = lambda o: [v.clone() for v in (o.logprob, o.entropy, o.top_token, o.top_logprob)]  # noqa: E731
        want, want2 = every(K.spqr_token_logprobs(s, logits, t)), every(K.spqr_token_logprobs(s, other, t))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            K.spqr_token_logprobs(s, logits, t)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(every(s), want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            K.spqr_token_logprobs(s, logits, t)
        for turn in range(3):
            s.logprob.zero_()
            graph.replay()
            K.spqr_token_logprobs(s2, other, t)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(every(s), want)) and all(torch.equal(a, b) for a, b in zip(every(s2), want2))
        logits.copy_(other)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(every(s), want2))


def test_refusals_of_the_binding():
    s = K.SpQRScores(4, 100, given=2, top=3)
    logits, t = torch.zeros(4, 100, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for args in ((logits, None), (logits, t[:3]), (logits, t.long()), (logits[:, :99], t), (logits.double(), t), (logits.cpu(), t), (logits[0], t),
                 (torch.zeros(5, 100, device="cuda"), t), (logits.t().contiguous().t(), t)):
        with pytest.raises(ValueError):
            K.spqr_token_logprobs(s, *args)
    with pytest.raises(ValueError):
        K.spqr_token_logprobs(K.SpQRScores(4, 100, given=0), logits, t)
