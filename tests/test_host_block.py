"""The entry points beside a step's products and attention: what they refuse, without a GPU (refusals come before any HIP call)."""
import ctypes as C
import math
import os
import re

import pytest

import paper_2306_03078_amd as P
import paper_2306_03078_amd.block_binding as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, PARAM, SIZE, ALIGN, DTYPE, WORKSPACE = 0, -1, -2, -3, -4, -5, -10, -11
SOME = 1 << 20                   # an aligned address that nothing reads
F32, F16, BF16 = 0, 1, 2


def filled(d, values, change):
    for name, v in {**values, **change}.items():
        if isinstance(v, (list, tuple)):
            for i, x in enumerate(v):
                getattr(d, name)[i] = x
        else:
            setattr(d, name, v)
    return d


def norm(**change):
    at = {n: SOME + 4096 * i for i, n in enumerate(("x", "y", "gate", "sum", "out", "y_weight", "y_bias", "x_weight", "x_bias"))}
    d = filled(K.spqr_residual_norm_t(), dict(rows=3, width=100, x_dtype=F32, y_dtype=F32, gate_dtype=F32, out_dtype=F16, weight_dtype=F32, norm_y=1, norm_x=2,
                                              act=1, eps=1e-6, skip=1.0, scale=1.0, x_stride=100, y_stride=100, gate_stride=0, sum_stride=100, out_stride=100,
                                              **at), change)
    return K._lib().spqr_residual_norm(C.byref(d), None)


def plan_of(**change):
    at = {n: SOME + 4096 * i for i, n in enumerate(("adapter", "q_start", "count", "tile", "row"))}
    return filled(K.spqr_adapter_plan_t(), dict(rows=130, slots=5, requests=4, max_tiles=8, **at), change)


def plan(**change):
    return K._lib().spqr_adapter_plan(C.byref(plan_of(**change)), None)


def bank(**change):
    at = {n: [SOME + 4096 * (2 * i + p) for p in range(2)] for i, n in enumerate(("bank", "scale", "y", "out"))}
    return filled(K.spqr_adapters_t(), dict(count=2, width=64, slots=5, dtype=F16, y_dtype=F32, m=[96, 32], max_rank=[16, 8], y_stride=[96, 32],
                                            out_stride=[96, 32], x=SOME, x_stride=64, workspace=SOME, workspace_bytes=1 << 40, **at), change)


def adapt(p=None, **change):
    p = plan_of() if p is None else p
    return K._lib().spqr_adapters(C.byref(bank(**change)), C.byref(p), None)


def scores_of(**change):
    at = {n: SOME + 4096 * i for i, n in enumerate(("logits", "tokens", "logprob", "entropy", "top_token", "top_logprob", "workspace"))}
    return filled(K.spqr_token_logprobs_t(), dict(rows=3, vocab=1000, dtype=F16, given=2, top=5, scale=1.0, stride=1000, workspace_bytes=1 << 40, **at), change)


def score(**change):
    return K._lib().spqr_token_logprobs(C.byref(scores_of(**change)), None)


def test_every_declared_symbol_is_exported_and_the_descriptors_have_the_headers_fields():
    text = open(os.path.join(ROOT, "include", "spqr_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(spqr_[a-z_0-9]+)\s*\(", text))
    assert names == {"spqr_residual_norm", "spqr_adapter_tiles", "spqr_adapter_plan", "spqr_adapters_bank_bytes", "spqr_adapters_pack", "spqr_adapters_workspace_bytes", "spqr_adapters",
                     "spqr_token_logprobs_workspace_bytes", "spqr_token_logprobs"}
    for n in names:
        assert hasattr(C.CDLL(P.library_path()), n)
    for cls in (K.spqr_residual_norm_t, K.spqr_adapter_plan_t, K.spqr_adapters_t, K.spqr_token_logprobs_t):
        body = re.search(r"typedef struct %s \{(.*?)\}" % cls.__name__, text, flags=re.S).group(1)
        fields = [w for line in body.split(";") for w in re.findall(r"(\w+)\s*(?:\[\w+\])?\s*(?:,|$)", line.strip().replace("*", " "))]
        assert fields == [n for n, _ in cls._fields_]
    for name in ("SPQR_MAX_WIDTH", "SPQR_ADAPTER_TILE", "SPQR_MAX_SLOTS", "SPQR_MAX_RANK", "SPQR_MAX_TOP", "SPQR_MAX_GIVEN"):
        assert int(re.search(r"#define %s\s+(\d+)" % name, text).group(1)) == getattr(K, name)
    assert "SPQR_MAX_ROWS     (1 << 20)" in text and K.SPQR_MAX_ROWS == 1 << 20


def test_missing_descriptors():
    lib = K._lib()
    assert lib.spqr_residual_norm(None, None) == NULL and lib.spqr_adapter_plan(None, None) == NULL
    assert lib.spqr_adapters(None, C.byref(plan_of()), None) == NULL and lib.spqr_adapters(C.byref(bank()), None, None) == NULL
    assert lib.spqr_token_logprobs(None, None) == NULL and lib.spqr_token_logprobs_workspace_bytes(None) == NULL
    assert lib.spqr_adapters_workspace_bytes(None, 1) == NULL


@pytest.mark.parametrize("field,value,status", [
    ("rows", -1, SHAPE), ("width", 0, SHAPE), ("width", 65537, SHAPE), ("norm_y", 3, PARAM), ("norm_y", -1, PARAM), ("norm_x", 3, PARAM), ("act", 4, PARAM),
    ("act", -1, PARAM), ("eps", 0.0, PARAM), ("eps", -1e-6, PARAM), ("eps", math.inf, PARAM), ("eps", math.nan, PARAM), ("weight_offset", math.nan, PARAM),
    ("skip", math.inf, PARAM), ("scale", math.nan, PARAM), ("x_dtype", 3, DTYPE), ("y_dtype", -1, DTYPE), ("gate_dtype", 7, DTYPE), ("out_dtype", 3, DTYPE),
    ("weight_dtype", 3, DTYPE), ("x_stride", 99, SHAPE), ("y_stride", 0, SHAPE), ("sum_stride", 1, SHAPE), ("out_stride", -100, SHAPE), ("gate_stride", 99, SHAPE),
    ("x_stride", 1 << 62, SHAPE), ("x", SOME + 2, ALIGN), ("y", SOME + 2, ALIGN), ("gate", SOME + 1, ALIGN), ("sum", SOME + 2, ALIGN), ("out", SOME + 1, ALIGN),
    ("y_weight", SOME + 2, ALIGN), ("x_bias", SOME + 2, ALIGN)])
def test_norm_refuses(field, value, status):
    assert norm(**{field: value}) == status


def test_norm_refuses_nothing_to_read_or_write():
    assert norm(x=None, y=None) == NULL and norm(sum=None, out=None) == NULL
    assert norm(rows=0, x=None, y=None, out=None, sum=None) == OK


@pytest.mark.parametrize("field,value,status", [
    ("rows", -1, SHAPE), ("rows", (1 << 20) + 1, SHAPE), ("slots", 0, SHAPE), ("slots", 4097, SHAPE), ("requests", -1, SHAPE), ("requests", 1025, SHAPE),
    ("q_start", None, SHAPE), ("max_tiles", 7, SIZE), ("adapter", None, NULL), ("count", None, NULL), ("tile", None, NULL), ("row", None, NULL),
    ("adapter", SOME + 2, ALIGN), ("q_start", SOME + 1, ALIGN), ("count", SOME + 2, ALIGN), ("tile", SOME + 2, ALIGN), ("row", SOME + 3, ALIGN)])
def test_plan_refuses(field, value, status):
    assert plan(**{field: value}) == status


def test_a_plan_of_no_rows():
    assert plan(rows=0, max_tiles=0, count=None, tile=None, row=None, adapter=None) == OK


def test_tiles_are_enough_for_any_rows():
    lib = K._lib()
    for rows, slots, most in ((0, 1, 0), (1, 9, 1), (64, 1, 3), (130, 5, 8), (1 << 20, 4096, (1 << 14) + 4097)):
        assert lib.spqr_adapter_tiles(rows, slots) == most
    for counts in ([64, 1], [65, 64, 63, 1], [1] * 7, [129]):
        assert sum(-(-c // 64) for c in counts) <= lib.spqr_adapter_tiles(sum(counts), max(1, len(counts) - 1))
    assert lib.spqr_adapter_tiles(-1, 1) == SHAPE and lib.spqr_adapter_tiles(1, 0) == SHAPE


@pytest.mark.parametrize("field,value,status", [
    ("count", 0, PARAM), ("count", 9, PARAM), ("width", 0, SHAPE), ("width", 65537, SHAPE), ("slots", 4, PARAM), ("dtype", F32, DTYPE), ("dtype", 3, DTYPE),
    ("y_dtype", 3, DTYPE), ("m", [96, 0], SHAPE), ("m", [65537], SHAPE), ("max_rank", [16, 0], PARAM), ("max_rank", [257], PARAM), ("x_stride", 63, SHAPE),
    ("y_stride", [96, 31], SHAPE), ("out_stride", [95], SHAPE), ("out_stride", [1 << 62], SHAPE), ("bank", [None], NULL), ("bank", [SOME, None], NULL),
    ("out", [None], NULL), ("x", None, NULL), ("workspace", None, NULL), ("x", SOME + 1, ALIGN), ("bank", [SOME + 128], ALIGN), ("scale", [SOME + 2], ALIGN), ("y", [SOME + 2], ALIGN), ("out", [SOME, SOME + 2], ALIGN), ("workspace", SOME + 128, ALIGN),
    ("workspace_bytes", 0, WORKSPACE), ("workspace_bytes", -1, WORKSPACE)])
def test_adapters_refuse(field, value, status):
    assert adapt(**{field: value}) == status


def pack(p=0, first=0, slots=5, A=SOME, B=SOME, rank=SOME, **change):
    return K._lib().spqr_adapters_pack(C.byref(bank(**change)), p, first, slots, A, B, rank, None)


def test_pack_refuses():
    assert pack(p=-1) == PARAM and pack(p=2) == PARAM and pack(first=-1) == PARAM and pack(first=1) == PARAM and pack(slots=-1) == PARAM and pack(slots=6) == PARAM
    assert pack(first=5, slots=0, A=None) == OK and pack(dtype=F32) == DTYPE and pack(max_rank=[0]) == PARAM and pack(width=0) == SHAPE
    assert pack(A=None) == NULL and pack(B=None) == NULL and pack(bank=[None]) == NULL
    assert pack(A=SOME + 1) == ALIGN and pack(B=SOME + 1) == ALIGN and pack(rank=SOME + 2) == ALIGN and pack(bank=[SOME + 128]) == ALIGN


def test_bank_bytes():
    """Ranks rounded up to 16 (A) and 32 (B, above 16), widths to 128, m to 64."""
    lib = K._lib()
    for width, m, rank, elements in ((64, 96, 16, 16 * 128 + 128 * 16), (129, 64, 17, 32 * 256 + 64 * 32), (1, 1, 1, 16 * 128 + 64 * 16),
                                     (8192, 8192, 64, 2 * 64 * 8192), (128, 64, 40, 48 * 128 + 64 * 64)):
        assert lib.spqr_adapters_bank_bytes(C.byref(bank(width=width, m=[m, 32], max_rank=[rank, 8])), 0) == 256 + 5 * 2 * elements
    assert lib.spqr_adapters_bank_bytes(C.byref(bank()), 2) == PARAM and lib.spqr_adapters_bank_bytes(None, 0) == NULL
    assert lib.spqr_adapters_bank_bytes(C.byref(bank(slots=4097)), 0) == SHAPE


def test_adapters_refuse_a_plan_that_is_none():
    assert adapt(plan_of(max_tiles=7)) == SIZE and adapt(plan_of(tile=None)) == NULL and adapt(plan_of(row=SOME + 2)) == ALIGN
    assert adapt(plan_of(rows=0), x=None, workspace=None) == OK


def test_the_adapters_workspace_goes_by_the_sizes():
    lib = K._lib()
    got = [lib.spqr_adapters_workspace_bytes(C.byref(bank(x=None, workspace=None, bank=[None] * 2)), n) for n in (0, 1, 16, 200, 5000)]
    assert all(b % 256 == 0 for b in got) and got[0] == 0 and 0 < got[1] and got == sorted(got)
    assert adapt(workspace_bytes=lib.spqr_adapters_workspace_bytes(C.byref(bank()), 130) - 1) == WORKSPACE
    assert lib.spqr_adapters_workspace_bytes(C.byref(bank()), -1) == SHAPE and lib.spqr_adapters_workspace_bytes(C.byref(bank()), (1 << 20) + 1) == SHAPE


@pytest.mark.parametrize("field,value,status", [
    ("rows", -1, SHAPE), ("vocab", 0, SHAPE), ("vocab", 1 << 24, SHAPE), ("given", -1, PARAM), ("given", 65, PARAM), ("top", -1, PARAM), ("top", 65, PARAM),
    ("dtype", 3, DTYPE), ("scale", 0.0, PARAM), ("scale", -1.0, PARAM), ("scale", math.inf, PARAM), ("scale", math.nan, PARAM), ("scale", 3.4e38, PARAM),
    ("stride", 999, SHAPE), ("stride", 1 << 62, SHAPE), ("logits", None, NULL), ("tokens", None, NULL), ("logprob", None, NULL), ("top_token", None, NULL),
    ("top_logprob", None, NULL), ("logits", SOME + 1, ALIGN), ("tokens", SOME + 2, ALIGN), ("logprob", SOME + 2, ALIGN), ("entropy", SOME + 1, ALIGN),
    ("top_token", SOME + 2, ALIGN), ("top_logprob", SOME + 2, ALIGN)])
def test_scores_refuse(field, value, status):
    assert score(**{field: value}) == status


def test_scores_of_nothing():
    assert score(given=0, top=0, entropy=None) == NULL
    assert score(rows=0, logits=None) == OK


def test_scores_refuse_a_workspace_that_is_none():
    """Rows that are cut into parts need one; no fewer bytes for more rows."""
    lib = K._lib()
    bytes_of = lambda **change: lib.spqr_token_logprobs_workspace_bytes(C.byref(scores_of(**change)))  # noqa: E731
    assert bytes_of() == 0 and bytes_of(rows=100000) == 0
    got = [bytes_of(rows=n, vocab=100000, top=64) for n in (0, 1, 2, 7, 100, 512, 513, 5000)]
    assert got == sorted(got) and got[0] == 0 and got[1] > 0 and all(b % 256 == 0 for b in got)
    for rows in (1, 3, 40):
        wide = dict(rows=rows, vocab=100000, stride=100000)
        assert score(workspace=None, **wide) == NULL and score(workspace=SOME + 128, **wide) == ALIGN and score(workspace_bytes=0, **wide) == WORKSPACE


def test_handles_refuse_what_is_not_on_the_card():
    import torch
    with pytest.raises(ValueError):
        K.SpQRResidualNorm(64, x_weight=torch.ones(64))
    with pytest.raises(ValueError):
        K.SpQRResidualNorm(64, device="cpu")
    with pytest.raises(ValueError):
        K.SpQRAdapters([torch.zeros(2, 4, 64, dtype=torch.float16)], [torch.zeros(2, 32, 4, dtype=torch.float16)], rows=1)
    with pytest.raises(ValueError):
        K.SpQRAdapters([], [], rows=1)
    with pytest.raises(P.SpQRError):
        K.SpQRAdapterPlan(4, 0, device="cpu")
    with pytest.raises(ValueError):
        K.SpQRAdapterPlan(4, 1, device="cpu")
    with pytest.raises(ValueError):
        K.SpQRScores(4, 100, device="cpu")
