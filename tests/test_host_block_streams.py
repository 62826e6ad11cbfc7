"""Calls with stream=: the tensors that they make come from that stream's memory, and the launch goes there.  No GPU: the library's call is replaced
by one that notes what it was given, torch's allocations and streams by ones that note the current stream."""
import pytest
import torch

import paper_2306_03078_amd.binding as B
import paper_2306_03078_amd.block_binding as K
import paper_2306_03078_amd.serve_binding as S

T, N, M = 3, 64, 32


class Tensor:
    """What the binding asks of a tensor; `of`: the stream that was current when it was made."""

    def __init__(self, shape, dtype=torch.float32, of=None):
        self.shape, self.dtype, self.of, self.device = torch.Size(shape), dtype, of, torch.device("cuda", 0)
        self.recorded = []

    def stride(self):
        return (self.shape[-1], 1)[2 - len(self.shape):]

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.recorded.append(stream)


class Stream:
    def __init__(self, address, device_index=0):
        self.cuda_stream, self.device_index = address, device_index


HOME = Stream(1)


@pytest.fixture
def world(monkeypatch):
    """(addresses of the streams that launches went to, a function that says what stream is current)"""
    K._lib()
    got, current = [], [HOME]

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.old, current[0] = current[0], self.stream

        def __exit__(self, *_):
            current[0] = self.old

    def call(entry, desc, *args):
        got.append(args[-1])
        return 0

    class One:
        def new_empty(self, shape):
            return Tensor(shape, torch.float16, current[0])

    monkeypatch.setattr(B, "_call", call)
    monkeypatch.setattr(S, "_raw_stream", lambda index: current[0].cuda_stream)
    monkeypatch.setattr(S, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_on", On)
    monkeypatch.setattr(K, "_empty", lambda shape, dtype, device: Tensor(shape, dtype, current[0]))
    monkeypatch.setattr(K, "_empty_like", lambda t: Tensor(t.shape, t.dtype, current[0]))
    return got, (lambda: current[0]), One()


def handle(cls, desc, **more):
    h = cls.__new__(cls)
    h.__dict__.update(desc=desc, device=torch.device("cuda", 0), _index=0, **more)
    return h


def handles(one):
    plan = handle(K.SpQRAdapterPlan, K.spqr_adapter_plan_t(), rows=T, slots=2, _at=0)
    return (handle(K.SpQRResidualNorm, K.spqr_residual_norm_t(), width=N, out_dtype=torch.float16, _out_type=1, _one=one), plan,
            handle(K.SpQRAdapters, K.spqr_adapters_t(), m=[M], max_rank=[4], width=N, slots=2, dtype=torch.float16),
            handle(K.SpQRScores, K.spqr_token_logprobs_t(), rows=T, vocab=N, given=1, top=0))


@pytest.mark.parametrize("stream", [None, Stream(5)])
def test_what_a_call_makes_is_the_streams(world, stream):
    got, now, one = world
    norm, plan, bank, scores = handles(one)
    x, half, ints = Tensor((T, N)), Tensor((T, N), torch.float16), Tensor((T,), torch.int32)
    made = list(K.spqr_residual_norm(norm, x, x, stream=stream))
    made += K.spqr_adapters(bank, plan, half, stream=stream) + K.spqr_adapters(bank, plan, half, [Tensor((T, M))], stream=stream)
    K.spqr_adapter_plan(plan, ints, stream=stream)
    K.spqr_token_logprobs(scores, x, ints, stream=stream)
    here = stream or HOME
    assert [t.of for t in made] == [here] * 4 and got == [here.cuda_stream] * 5 and now() is HOME


def test_tensors_that_are_given_are_used(world):
    got, now, one = world
    norm, plan, bank, _ = handles(one)
    x, half, sum_, out, y = Tensor((T, N)), Tensor((T, N), torch.float16), Tensor((T, N)), Tensor((T, N), torch.float16), Tensor((T, M))
    assert K.spqr_residual_norm(norm, x, x, sum=sum_, out=out, stream=Stream(5)) == (sum_, out)
    assert K.spqr_adapters(bank, plan, half, [y], [y], stream=Stream(5)) == [y]
    assert got == [5, 5] and now() is HOME


def test_a_stream_of_another_device_is_refused(world):
    got, now, one = world
    norm, plan, bank, scores = handles(one)
    x, half, ints = Tensor((T, N)), Tensor((T, N), torch.float16), Tensor((T,), torch.int32)
    away = Stream(5, 1)
    for call in (lambda: K.spqr_residual_norm(norm, x, x, stream=away), lambda: K.spqr_adapters(bank, plan, half, stream=away),
                 lambda: K.spqr_adapter_plan(plan, ints, stream=away), lambda: K.spqr_token_logprobs(scores, x, ints, stream=away)):
        with pytest.raises(ValueError):
            call()
    assert got == [] and now() is HOME


def test_weights_that_are_loaded_on_a_stream_stay_until_it_has_read_them(world, monkeypatch):
    """A, B and rank may go after load(): their memory is not given away before the stream has passed."""
    got, _, one = world
    bank = handles(one)[2]

    class Lib:
        def spqr_adapters_pack(self, *args):
            got.append(args[-1])
            return 0

    class Device:
        def __init__(self, index):
            pass

        __enter__ = __exit__ = lambda self, *_: None

    monkeypatch.setattr(K, "_lib", Lib)
    monkeypatch.setattr(torch.cuda, "device", Device)
    for stream in (Stream(5), None):
        A, B_, rank = Tensor((1, 4, N), torch.float16), Tensor((1, M, 4), torch.float16), Tensor((1,), torch.int32)
        bank.load(1, [A], [B_], rank, stream=stream)
        assert all(t.recorded == ([] if stream is None else [stream]) for t in (A, B_, rank))
    assert got == [5, HOME.cuda_stream]
    with pytest.raises(ValueError):
        bank.load(1, [A], [B_], rank, stream=Stream(5, 1))
