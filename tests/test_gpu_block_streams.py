"""Calls with stream= beside a busy current stream: handles made there, results of the call's own memory, weights loaded on a stream and let go."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
ROWS, WIDTH, M, VOCAB = 70, 512, 256, 40000


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def busy():
    """Some milliseconds of work on the current stream, in memory that is free again when this returns."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(8):
        a = a @ a * 1e-4
    return [torch.full((ROWS, n), 7.0, device="cuda", dtype=t) * 2 for n in (WIDTH, M, VOCAB // 64) for t in (torch.float16, torch.float32)]


def operators(stream, norm, x, y, A, B, adapter, logits, tokens):
    """One call of each on `stream` (None: the current one), the handles with scratch made just before."""
    busy()
    plan = K.SpQRAdapterPlan(ROWS, 3)
    bank = K.SpQRAdapters([A], [B], rows=ROWS)
    scores = K.SpQRScores(ROWS, VOCAB, given=1, top=5)
    busy()
    K.spqr_adapter_plan(plan, adapter, stream=stream)
    total, out = K.spqr_residual_norm(norm, x, y, stream=stream)
    made, = K.spqr_adapters(bank, plan, out, stream=stream)
    base = torch.ones(ROWS, M, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    again, = K.spqr_adapters(bank, plan, out, [base], stream=stream)
    K.spqr_token_logprobs(scores, logits, tokens, stream=stream)
    kept = busy()                                        # memory that is given out on the current stream meanwhile is other memory
    torch.cuda.synchronize()
    assert all((t == 14).all() for t in kept)
    return [t.clone() for t in (plan.count, plan.tile, plan.row, total, out, made, again, scores.logprob, scores.entropy, scores.top_token, scores.top_logprob)]


def test_every_operator_on_a_stream_of_the_call():
    g = torch.Generator(device="cuda").manual_seed(0)
    x, y = (torch.randn(ROWS, WIDTH, device="cuda", generator=g) for _ in range(2))
    A = (torch.randn(3, 16, WIDTH, device="cuda", generator=g) / 20).half()
    B = torch.randn(3, M, 16, device="cuda", generator=g).half()
    logits = torch.randn(ROWS, VOCAB, device="cuda", generator=g)
    args = (K.SpQRResidualNorm(WIDTH, norm_y="rms"), x, y, A, B, ints([r % 4 - 1 for r in range(ROWS)]), logits, ints([[r] for r in range(ROWS)]))
    want = operators(None, *args)
    torch.cuda.synchronize()
    for side in (torch.cuda.Stream(), torch.cuda.Stream()):
        for got in (operators(side, *args), operators(side, *args)):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_loaded_on_a_stream():
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda n: ((torch.randn(n, 16, WIDTH, device="cuda", generator=g) / 20).half(), torch.randn(n, M, 16, device="cuda", generator=g).half())  # noqa: E731
    A, B = make(2)
    plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(ROWS, 2), ints([r % 2 for r in range(ROWS)]))
    x = torch.randn(ROWS, WIDTH, device="cuda", generator=g).half()
    bank = K.SpQRAdapters([A], [B], rows=ROWS)
    before = K.spqr_adapters(bank, plan, x)[0].clone()
    A2, B2 = make(1)
    other = K.SpQRAdapters([torch.cat([A[:1], A2])], [torch.cat([B[:1], B2])], rows=ROWS)
    want = K.spqr_adapters(other, plan, x)[0].clone()
    assert not torch.equal(before, want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    bank.load(1, [A2], [B2], stream=side)
    del A2, B2
    for _ in range(3):                                   # (their memory is not these tensors')
        torch.full((1, 16, WIDTH), 9.0, dtype=torch.float16, device="cuda")
        torch.full((1, M, 16), 9.0, dtype=torch.float16, device="cuda")
    got = K.spqr_adapters(bank, plan, x, stream=side)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_stream_of_the_call_in_a_capture():
    norm = K.SpQRResidualNorm(WIDTH, norm_y="rms")
    x, y = torch.randn(ROWS, WIDTH, device="cuda"), torch.randn(ROWS, WIDTH, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        K.spqr_residual_norm(norm, x, y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = K.spqr_residual_norm(norm, x, y, stream=side)
    torch.cuda.synchronize()
    for _ in range(3):
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        want = K.spqr_residual_norm(norm, x, y)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_current_stream_is_the_one_it_was():
    """After calls with stream=, ones that are refused too, on the default stream and inside another stream's context."""
    norm = K.SpQRResidualNorm(WIDTH)
    x, side, other = torch.randn(ROWS, WIDTH, device="cuda"), torch.cuda.Stream(), torch.cuda.Stream()
    want = K.spqr_residual_norm(norm, x, x)
    torch.cuda.synchronize()
    for context in (torch.cuda.default_stream(), other):
        with torch.cuda.stream(context):
            got = K.spqr_residual_norm(norm, x, x, stream=side)
            assert torch.cuda.current_stream() == context
            with pytest.raises(ValueError):
                K.spqr_residual_norm(norm, x, x[:3], stream=side)
            assert torch.cuda.current_stream() == context
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
