"""The entry points around a decode step's attention: what they refuse, without a GPU (refusals come before any HIP call)."""
import ctypes as C
import math
import os
import re

import pytest

import paper_2306_03078_amd as P
import paper_2306_03078_amd.serve_binding as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, PARAM, ALIGN, DTYPE, WORKSPACE = -1, -2, -3, -5, -10, -11
SOME = 1 << 20                   # an aligned address that nothing reads


def descriptor(**change):
    d = S.spqr_step_t()
    values = dict(requests=2, tokens=5, max_fresh=4, max_pages=3, mask_words=1, dtype=P.SPQR_F16, heads=8, kv_heads=2, head_dim=128, page=16,
                  pages=9, layers=2, rotary_dim=128, rotary_positions=64, rotary_pairs=0, scale=0.1, workspace_bytes=1 << 40)
    for i, (name, kind) in enumerate(S.spqr_step_t._fields_):
        if kind is C.c_void_p:
            values[name] = SOME + 4096 * i
    values.update(change)
    for name, v in values.items():
        setattr(d, name, v)
    return d


def rows(**change):
    r = S.spqr_rows_t(q=SOME, k=SOME + 256, v=SOME + 512, q_stride=1024, k_stride=256, v_stride=256, x_dtype=P.SPQR_F32)
    for name, v in change.items():
        setattr(r, name, v)
    return r


def plan(d):
    return S._lib().spqr_cache_plan(C.byref(d), None)


def store(d, r, layer=0, out=SOME):
    return S._lib().spqr_cache_store(C.byref(d), layer, C.addressof(r) if r is not None else None, out, None)


def attend(d, layer=0, q=SOME, q_stride=1024, out=SOME, out_stride=1024):
    return S._lib().spqr_tree_attention(C.byref(d), layer, q, q_stride, out, out_stride, None)


def keep(d, last=SOME):
    return S._lib().spqr_cache_keep(C.byref(d), last, None)


def test_every_declared_symbol_is_exported_and_the_descriptor_has_the_headers_fields():
    text = open(os.path.join(ROOT, "include", "spqr_serve.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(spqr_[a-z_0-9]+)\s*\(", text))
    assert names == {"spqr_cache_plan", "spqr_cache_store", "spqr_tree_attention", "spqr_tree_attention_workspace_bytes", "spqr_cache_keep"}
    for n in names:
        assert hasattr(C.CDLL(P.library_path()), n)
    for struct, cls in (("spqr_step_t", S.spqr_step_t), ("spqr_rows_t", S.spqr_rows_t)):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct, text, flags=re.S).group(1)
        fields = [w for line in body.split(";") for w in re.findall(r"(\w+)\s*(?:,|$)", line.strip().replace("*", " "))]
        assert fields == [n for n, _ in cls._fields_]


SIZES = [("requests", 0, SHAPE), ("requests", 1025, SHAPE), ("tokens", 0, SHAPE), ("max_pages", 0, SHAPE), ("mask_words", -1, PARAM),
         ("mask_words", 5, PARAM), ("max_fresh", 257, PARAM), ("max_fresh", -1, PARAM), ("page", 8, PARAM), ("page", 48, PARAM), ("page", 512, PARAM),
         ("pages", 0, SHAPE), ("pages", 1 << 27, SHAPE)]


@pytest.mark.parametrize("field,value,status", SIZES)
def test_sizes_that_every_call_refuses(field, value, status):
    d = descriptor(**{field: value})
    assert plan(d) == status and store(d, rows()) == status and attend(d) == status and keep(d) == status
    assert S._lib().spqr_tree_attention_workspace_bytes(C.byref(d)) == status


@pytest.mark.parametrize("field,value,status", [
    ("dtype", P.SPQR_F32, DTYPE), ("dtype", 3, DTYPE), ("head_dim", 80, PARAM), ("head_dim", 0, PARAM), ("heads", 0, SHAPE), ("heads", 7, SHAPE),
    ("kv_heads", 0, SHAPE), ("layers", 0, SHAPE), ("k", None, NULL), ("v", None, NULL), ("k", SOME + 8, ALIGN), ("v", SOME + 2, ALIGN)])
def test_caches_that_the_calls_on_them_refuse(field, value, status):
    d = descriptor(**{field: value})
    assert store(d, rows()) == status and attend(d) == status and keep(d) == status


def test_a_missing_descriptor():
    lib = S._lib()
    assert lib.spqr_cache_plan(None, None) == NULL and lib.spqr_cache_keep(None, None, None) == NULL
    assert lib.spqr_cache_store(None, 0, None, None, None) == NULL and lib.spqr_tree_attention(None, 0, None, 0, None, 0, None) == NULL
    assert lib.spqr_tree_attention_workspace_bytes(None) == NULL


def test_plan_refuses():
    for name in ("cached", "fresh", "held", "table", "pool", "ends", "q_start", "position", "slot", "held_out", "ends_out", "mask"):
        assert plan(descriptor(**{name: None})) == NULL, name
        assert plan(descriptor(**{name: SOME + 2})) == ALIGN, name
    for name in ("ends", "ends_out", "mask"):
        assert plan(descriptor(**{name: SOME + 4})) == ALIGN, name
    assert plan(descriptor(parent=SOME + 1)) == ALIGN
    d = descriptor()
    assert plan(descriptor(held=d.held_out)) == PARAM and plan(descriptor(ends_out=d.ends)) == PARAM


def test_store_refuses():
    d = descriptor()
    assert store(d, None) == NULL and store(d, rows(), out=None) == NULL and store(d, rows(), out=SOME + 8) == ALIGN
    assert store(d, rows(), layer=2) == PARAM and store(d, rows(), layer=-1) == PARAM
    for name in ("q", "k", "v"):
        assert store(d, rows(**{name: None})) == NULL and store(d, rows(**{name: SOME + 2})) == ALIGN
        assert store(d, rows(**{name: SOME + 1, "x_dtype": S.SPQR_BF16})) == ALIGN
        assert store(d, rows(**{name + "_stride": 255})) == SHAPE
    assert store(d, rows(x_dtype=3)) == DTYPE and store(d, rows(x_dtype=-1)) == DTYPE
    for name in ("position", "slot", "rotary"):
        assert store(descriptor(**{name: None}), rows()) == NULL and store(descriptor(**{name: SOME + 2}), rows()) == ALIGN
    for dim in (-2, 63, 130):
        assert store(descriptor(rotary_dim=dim), rows()) == PARAM
    assert store(descriptor(rotary_positions=0), rows()) == SHAPE


def test_attention_refuses():
    d = descriptor()
    assert attend(d, layer=2) == PARAM and attend(d, layer=-1) == PARAM
    assert attend(d, q=None) == NULL and attend(d, out=None) == NULL
    assert attend(d, q=SOME + 8) == ALIGN and attend(d, out=SOME + 2) == ALIGN
    assert attend(d, q_stride=1023) == SHAPE and attend(d, out_stride=8) == SHAPE
    assert attend(d, q_stride=1028) == ALIGN and attend(d, out_stride=1028) == ALIGN
    for name in ("cached", "table", "q_start", "mask"):
        assert attend(descriptor(**{name: None})) == NULL and attend(descriptor(**{name: SOME + 2})) == ALIGN
    for scale in (math.inf, -math.inf, math.nan):
        assert attend(descriptor(scale=scale)) == PARAM


def test_attention_refuses_a_workspace_that_is_none():
    need = S._lib().spqr_tree_attention_workspace_bytes(C.byref(descriptor()))
    assert need > 0
    assert attend(descriptor(workspace=None)) == NULL and attend(descriptor(workspace=SOME + 128)) == ALIGN
    for size in (0, -1, need - 1):
        assert attend(descriptor(workspace_bytes=size)) == WORKSPACE
    assert attend(descriptor(heads=2048, kv_heads=1)) == SHAPE


@pytest.mark.parametrize("head_dim", [64, 96, 128, 256])
def test_the_workspace_goes_by_the_sizes_and_not_by_pointers(head_dim):
    """As many rows of partial results, twice a workgroup, as a chunk has."""
    lib = S._lib()
    got = set()
    for max_fresh in (1, 5, 9, 16, 17, 40, 256, 0):
        for max_pages in (1, 9, 1 << 20):
            d = descriptor(head_dim=head_dim, max_fresh=max_fresh, max_pages=max_pages, pages=1 << 20)
            n = lib.spqr_tree_attention_workspace_bytes(C.byref(d))
            e = descriptor(head_dim=head_dim, max_fresh=max_fresh, max_pages=max_pages, pages=1 << 20, k=SOME, v=SOME, cached=None, table=None, mask=None, workspace=None)
            assert n == lib.spqr_tree_attention_workspace_bytes(C.byref(e))
            got.add(n)
    assert 3 <= len(got) <= 5 and min(got) > 0 and max(got) <= 140 << 20


def test_keep_refuses():
    for name in ("cached", "table", "q_start", "cached_out", "mask"):
        assert keep(descriptor(**{name: None})) == NULL and keep(descriptor(**{name: SOME + 2})) == ALIGN
    assert keep(descriptor(), last=SOME + 1) == ALIGN
    d = descriptor()
    assert keep(descriptor(cached=d.cached_out)) == PARAM
    assert keep(descriptor(layers=1 << 20, pages=1, page=16)) == SHAPE       # more columns than a launch has workgroups


def test_the_step_refuses_arrays_that_do_not_fit_on_the_cpu():
    import torch
    kc = torch.zeros(1, 4, 2, 16, 64, dtype=torch.float16)
    for bad in (dict(k_cache=kc, v_cache=None), dict(k_cache=kc, v_cache=kc), dict(k_cache=kc[..., :32], v_cache=kc[..., :32]),
                dict(k_cache=None, v_cache=None)):
        with pytest.raises(ValueError):
            S.SpQRStep(requests=1, tokens=1, max_pages=1, **bad)
    with pytest.raises(TypeError):
        S.SpQRStep(None, None, page=16, pages=4, requests=1, tokens=1, max_pages=1, lengths=kc)
