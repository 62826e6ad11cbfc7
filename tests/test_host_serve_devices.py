"""Where the tensors of a decode step's calls are: addresses of other memory than the step's device's never reach a kernel, and launches
go to the step's device.  No GPU: the library's call is replaced by one that notes what it was given."""
import ctypes as C

import pytest
import torch

import paper_2306_03078_amd.binding as B
import paper_2306_03078_amd.serve_binding as S

T, HEADS, KV, D = 3, 4, 2, 64


class Row:
    """What the binding asks of a tensor."""

    def __init__(self, heads, device, dtype=torch.float16, shape=None, strides=None):
        self.shape, self.dtype, self.index = torch.Size(shape or (T, heads, D)), dtype, device
        self.strides = strides or (heads * D, D, 1)
        self.device = torch.device("cuda", device) if device >= 0 else torch.device("cpu")
        self.is_cuda = device >= 0

    def stride(self):
        return self.strides

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def calls(monkeypatch):
    """What reached the library: (the device that was current, the entry's arguments)."""
    S._lib()
    got, current = [], [0]

    class Device:
        def __init__(self, index):
            self.index = getattr(index, "index", index)

        def __enter__(self):
            self.old, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.old

    def call(entry, desc, *args):
        got.append((current[0], args))
        return 0

    monkeypatch.setattr(B, "_call", call)
    monkeypatch.setattr(S, "_raw_stream", lambda index: ("stream of", index))
    monkeypatch.setattr(S, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    return got, current


def step_on(index):
    s = S.SpQRStep.__new__(S.SpQRStep)
    rows = S.spqr_rows_t()
    s.__dict__.update(desc=S.spqr_step_t(), dtype=torch.float16, requests=2, tokens=T, heads=HEADS, kv_heads=KV, head_dim=D,
                      device=torch.device("cuda", index), _index=index, _rows=rows, _rows_at=C.addressof(rows), _q_of=Row(HEADS, index),
                      _q_like=((T, HEADS, D), (HEADS * D, D, 1), index), _kv_like=((T, KV, D), (KV * D, D, 1), index), cached_out=None)
    return s


@pytest.mark.parametrize("where", [-1, 1])
def test_tensors_of_other_memory_are_refused(calls, where):
    step, q, kv, out = step_on(0), Row(HEADS, 0), Row(KV, 0), Row(HEADS, 0)
    away, kv_away = Row(HEADS, where), Row(KV, where)
    for bad in (dict(q=away, k=kv, v=kv), dict(q=q, k=kv_away, v=kv), dict(q=q, k=kv, v=kv_away), dict(q=q, k=kv, v=kv, out=away)):
        with pytest.raises(ValueError):
            S.spqr_cache_store(step, **{"out": out, **bad})
    for bad in (dict(q=away, out=out), dict(q=q, out=away)):
        with pytest.raises(ValueError):
            S.spqr_tree_attention(step, **bad)
    with pytest.raises(ValueError):
        S.spqr_cache_keep(step, Row(1, where, dtype=torch.int32, shape=(2,), strides=(1,)))
    assert calls[0] == []


def test_real_host_tensors_are_refused(calls):
    step = step_on(0)
    q, kv = torch.zeros(T, HEADS, D, dtype=torch.float16), torch.zeros(T, KV, D, dtype=torch.float16)
    with pytest.raises(ValueError):
        S.spqr_cache_store(step, q, kv, kv, out=Row(HEADS, 0))
    with pytest.raises(ValueError):
        S.spqr_tree_attention(step, q, out=Row(HEADS, 0))
    with pytest.raises(ValueError):
        S.spqr_cache_keep(step, torch.zeros(2, dtype=torch.int32))
    assert calls[0] == []


@pytest.mark.parametrize("current", [0, 1])
def test_launches_go_to_the_steps_device(calls, current):
    got, now = calls
    for index in (0, 1):
        now[0] = current
        step, q, kv, out = step_on(index), Row(HEADS, index), Row(KV, index), Row(HEADS, index)
        del got[:]
        S.spqr_cache_plan(step)
        S.spqr_cache_store(step, q, kv, kv, out=out)
        S.spqr_tree_attention(step, q, out=out)
        S.spqr_cache_keep(step)
        assert [device for device, _ in got] == [index] * 4
        assert [args[-1] for _, args in got] == [("stream of", index)] * 4
        assert now[0] == current


def test_a_step_in_host_memory_is_refused():
    with pytest.raises(ValueError):
        S.SpQRStep(None, None, page=16, pages=4, requests=1, tokens=1, max_pages=1, device="cpu")
