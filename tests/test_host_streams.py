"""Calls with stream= of the products, the quantiser and the cache: results and scratch that they make come from that stream's memory.  No GPU: the
library's calls are replaced by ones that note the stream, torch's allocations and streams by ones that note the current stream."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

import paper_2306_03078_amd.binding as B
import paper_2306_03078_amd.encode_binding as E
import paper_2306_03078_amd.serve_binding as S
from test_host_serve_devices import HEADS, KV, Row, step_on

HOME, SIDE = SimpleNamespace(cuda_stream=1, synchronize=lambda: None), SimpleNamespace(cuda_stream=5, synchronize=lambda: None)


@pytest.fixture
def world(monkeypatch):
    """(streams of launches, streams that were current when memory was asked for, the current one)"""
    launched, asked, current = [], [], [HOME]
    B.load_library()
    S._lib()

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.old, current[0] = current[0], self.stream

        def __exit__(self, *_):
            current[0] = self.old

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *_: 256
            return lambda *args: launched.append(args[-1]) or 0

    def noting(f):
        def g(*args, **more):
            asked.append(current[0])
            return f(*args, **more)
        return g

    monkeypatch.setattr(B, "_call", lambda entry, desc, *args: launched.append(args[-1]) or 0)
    for m in (B, E):
        monkeypatch.setattr(m, "load_library", Lib)
    monkeypatch.setattr(E, "_on", On)
    monkeypatch.setattr(E, "_lib", Lib)
    address = lambda stream: (current[0] if stream is None else stream).cuda_stream  # noqa: E731
    monkeypatch.setattr(B, "_stream_ptr", address)
    monkeypatch.setattr(E, "_stream_ptr", address)
    monkeypatch.setattr(S, "_raw_stream", lambda index: current[0].cuda_stream)
    monkeypatch.setattr(S, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_on", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: current[0])
    monkeypatch.setattr(torch, "empty", noting(torch.empty))
    monkeypatch.setattr(torch, "empty_like", noting(lambda t, **_: t))
    return launched, asked, current


def calls():
    A = SimpleNamespace(m=32, n=64, beta1=16, beta2=16, group_axis=1, desc=B.spqr_matrix_t(), device=torch.device("cpu"))
    x, X = torch.zeros(64, dtype=torch.float16), torch.zeros(3, 64, dtype=torch.float16)
    H, W, perm = torch.zeros(64, 64, dtype=torch.float64), torch.zeros(32, 64, dtype=torch.float64), torch.zeros(64, dtype=torch.int32)
    y, Y = torch.zeros(32), torch.zeros(3, 32)
    step, q, kv = step_on(0), Row(HEADS, 0), Row(KV, 0)
    without = [lambda s: B.spqr_gemv(A, x, stream=s), lambda s: B.spqr_gemm_smallbatch(A, X, stream=s), lambda s: B.spqr_gemv_fused([A, A], x, stream=s),
               lambda s: B.spqr_gemm_fused([A, A], X, stream=s), lambda s: B.spqr_gemm_smallbatch_ws(A, X, None, stream=s),
               lambda s: B.spqr_gemm_fused_ws([A], X, None, stream=s), lambda s: B.spqr_gemv_grouped([A], [x], stream=s),
               lambda s: B.spqr_dequant_dense(A, B.SPQR_OUT_DENSE_F32, stream=s), lambda s: S.spqr_cache_store(step, q, kv, kv, stream=s),
               lambda s: S.spqr_tree_attention(step, q, stream=s), lambda s: E.spqr_hessian(H, stream=s), lambda s: E.spqr_inverse_cholesky(H, 1.0, stream=s),
               lambda s: E.spqr_act_order(H, stream=s), lambda s: E.spqr_permute_columns(W, perm, stream=s), lambda s: E.spqr_permute_symmetric(H, perm, stream=s),
               lambda s: E.spqr_quantize_device(W, H, 3, 16, 16, 1.0, stream=s)]
    given = [lambda s: B.spqr_gemv(A, x, out=y, stream=s), lambda s: B.spqr_gemm_smallbatch(A, X, out=Y, stream=s), lambda s: B.spqr_gemv_fused([A], x, outs=[y], stream=s),
             lambda s: B.spqr_gemm_fused([A], X, outs=[Y], stream=s), lambda s: S.spqr_cache_store(step, q, kv, kv, out=q, stream=s),
             lambda s: S.spqr_tree_attention(step, q, out=q, stream=s)]
    return without, given


@pytest.mark.parametrize("stream", [None, SIDE])
@pytest.mark.parametrize("which", range(16))
def test_what_a_call_makes_is_the_streams(world, which, stream):
    launched, asked, current = world
    call = calls()[0][which]
    call(stream)
    here = stream or HOME
    assert asked and all(s is here for s in asked) and launched and set(launched) == {here.cuda_stream} and current == [HOME]


@pytest.mark.parametrize("which", range(6))
def test_what_it_is_given_needs_no_memory(world, which):
    launched, asked, _ = world
    calls()[1][which](SIDE)
    assert asked == [] and launched == [5]
