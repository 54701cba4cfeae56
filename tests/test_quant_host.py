"""Refusals of the calls on an 8-bit cache, before anything is launched (no
GPU), and the plain reference that the GPU tests use."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest
import torch

import quantref as R
from paper_2606_00024_amd import _lib, api

PTR = 4096      # never read: every call here is refused, or has nothing to do


def _shape(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=64, page_size=64,
             num_pages=40, max_pages_per_seq=16, max_blocks_per_list=0, list_per_head=1,
             k_stride_page=2 * 64 * 128, k_stride_head=64 * 128, k_stride_token=128,
             v_stride_page=2 * 64 * 128, v_stride_head=64 * 128, v_stride_token=128)
    d.update(kw)
    return _lib.DecodeShape(**d)


def _opts(**kw):
    d = dict(softmax_scale=1 / math.sqrt(128), tau=1e-3, phi=1e-4, patience=5)
    d.update(kw)
    return _lib.DecodeOpts(**d)


def _spec(**kw):
    d = dict(format=_lib.QUANT_E4M3, scale_tokens=32, k_scale_stride_page=4, k_scale_stride_head=2,
             v_scale_stride_page=4, v_scale_stride_head=2)
    d.update(kw)
    return _lib.QuantCacheSpec(**d)


def _rows(**kw):
    d = dict(rows_dtype=_lib.ROWS_BF16, rows=4, k_stride_row=256, k_stride_head=128,
             v_stride_row=256, v_stride_head=128)
    d.update(kw)
    return _lib.QuantRows(**d)


def _decode(shape, opts, spec, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, page_table=PTR, seq_lens=PTR, block_list=0,
             block_list_len=0, out=PTR, lse=PTR, stop_block=PTR, workspace=PTR, workspace_bytes=1 << 30,
             stream=0)
    a.update(kw)
    return _lib.decode_attention_quant(shape, opts, spec, *a.values())


def _append(shape, spec, rows, **kw):
    a = dict(k_rows=PTR, v_rows=PTR, row_offsets=0, positions=0, page_table=PTR, k=PTR, v=PTR,
             k_scale=PTR, v_scale=PTR, stream=0)
    a.update(kw)
    return _lib.quant_append(shape, spec, rows, *a.values())


def _read(shape, spec, rows, **kw):
    a = dict(k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, row_offsets=0, positions=0, page_table=PTR,
             k_rows=PTR, v_rows=PTR, stream=0)
    a.update(kw)
    return _lib.quant_read(shape, spec, rows, *a.values())


BAD_SHAPES = [
    (dict(head_dim=64), _lib.ERR_UNSUPPORTED),
    (dict(page_size=8), _lib.ERR_UNSUPPORTED),
    (dict(page_size=96), _lib.ERR_UNSUPPORTED),
    (dict(batch=-1), _lib.ERR_INVALID_ARG),
    (dict(num_kv_heads=0), _lib.ERR_INVALID_ARG),
    (dict(num_pages=0), _lib.ERR_INVALID_ARG),
    (dict(max_pages_per_seq=0), _lib.ERR_INVALID_ARG),
    (dict(k_stride_page=-16), _lib.ERR_INVALID_ARG),
    (dict(k_stride_token=136), _lib.ERR_UNSUPPORTED),
    (dict(v_stride_head=8), _lib.ERR_UNSUPPORTED),
    (dict(v_stride_page=24), _lib.ERR_UNSUPPORTED),
    (dict(k_stride_token=1 << 24), _lib.ERR_UNSUPPORTED),
]
BAD_SPECS = [
    (dict(format=2), _lib.ERR_INVALID_ARG),
    (dict(format=-1), _lib.ERR_INVALID_ARG),
    (dict(scale_tokens=0), _lib.ERR_INVALID_ARG),
    (dict(scale_tokens=-16), _lib.ERR_INVALID_ARG),
    (dict(scale_tokens=8), _lib.ERR_UNSUPPORTED),
    (dict(scale_tokens=48), _lib.ERR_UNSUPPORTED),
    (dict(scale_tokens=128), _lib.ERR_UNSUPPORTED),      # longer than a page
    (dict(k_scale_stride_page=-1), _lib.ERR_INVALID_ARG),
    (dict(v_scale_stride_head=-1), _lib.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_SHAPES)
def test_shapes(kw, status):
    assert _decode(_shape(**kw), _opts(), _spec()) == status
    assert _append(_shape(**kw), _spec(), _rows()) == status
    assert _read(_shape(**kw), _spec(), _rows()) == status


@pytest.mark.parametrize("kw,status", BAD_SPECS)
def test_specs(kw, status):
    assert _decode(_shape(), _opts(), _spec(**kw)) == status
    assert _append(_shape(), _spec(**kw), _rows()) == status
    assert _read(_shape(), _spec(**kw), _rows()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), _lib.ERR_INVALID_ARG),
    (dict(rows=3), _lib.ERR_INVALID_ARG),                # no offsets, two sequences
    (dict(rows_dtype=3), _lib.ERR_INVALID_ARG),
    (dict(rows_dtype=-1), _lib.ERR_INVALID_ARG),
    (dict(k_stride_row=-8), _lib.ERR_INVALID_ARG),
    (dict(v_stride_head=-8), _lib.ERR_INVALID_ARG),
    (dict(k_stride_row=260), _lib.ERR_UNSUPPORTED),
    (dict(v_stride_head=4), _lib.ERR_UNSUPPORTED),
    (dict(rows_dtype=_lib.ROWS_F32, v_stride_head=2), _lib.ERR_UNSUPPORTED),
    (dict(rows=1 << 24), _lib.ERR_UNSUPPORTED),
    (dict(k_stride_row=1 << 27), _lib.ERR_UNSUPPORTED),
])
def test_rows(kw, status):
    assert _append(_shape(), _spec(), _rows(**kw)) == status
    assert _read(_shape(), _spec(), _rows(**kw)) == status


@pytest.mark.parametrize("name", ["k_rows", "v_rows", "page_table", "k", "v", "k_scale", "v_scale"])
def test_null_and_misaligned_arrays(name):
    assert _append(_shape(), _spec(), _rows(), **{name: 0}) == _lib.ERR_INVALID_ARG
    assert _read(_shape(), _spec(), _rows(), **{name: 0}) == _lib.ERR_INVALID_ARG
    if name in ("k_rows", "v_rows", "k", "v"):
        assert _append(_shape(), _spec(), _rows(), **{name: PTR + 8}) == _lib.ERR_UNSUPPORTED
        assert _read(_shape(), _spec(), _rows(), **{name: PTR + 8}) == _lib.ERR_UNSUPPORTED
    elif name != "page_table":
        assert _append(_shape(), _spec(), _rows(), **{name: PTR + 2}) == _lib.ERR_INVALID_ARG
        assert _read(_shape(), _spec(), _rows(), **{name: PTR + 2}) == _lib.ERR_INVALID_ARG


def test_runs_of_more_than_256_slots_are_read_but_not_written():
    shape = _shape(page_size=512, k_stride_head=512 * 128, v_stride_head=512 * 128)
    assert _append(shape, _spec(scale_tokens=512), _rows()) == _lib.ERR_UNSUPPORTED
    assert _read(shape, _spec(scale_tokens=512), _rows(rows=0)) == _lib.OK


def test_nothing_to_do():
    assert _append(_shape(), _spec(), _rows(rows=0), k_rows=0, v_rows=0) == _lib.OK
    assert _read(_shape(), _spec(), _rows(rows=0), k_rows=0, v_rows=0) == _lib.OK
    assert _append(_shape(batch=0), _spec(), _rows()) == _lib.OK
    assert _decode(_shape(batch=0), _opts(), _spec()) == _lib.OK


@pytest.mark.parametrize("kw,status", [
    (dict(k_scale=0), _lib.ERR_INVALID_ARG),
    (dict(v_scale=0), _lib.ERR_INVALID_ARG),
    (dict(v_scale=PTR + 2), _lib.ERR_INVALID_ARG),
    (dict(q=0), _lib.ERR_INVALID_ARG),
    (dict(k=PTR + 8), _lib.ERR_UNSUPPORTED),
    (dict(workspace=0), _lib.ERR_WORKSPACE_TOO_SMALL),
    (dict(workspace_bytes=64), _lib.ERR_WORKSPACE_TOO_SMALL),
    (dict(workspace=PTR + 4), _lib.ERR_INVALID_ARG),
    (dict(block_list=PTR), _lib.ERR_INVALID_ARG),
])
def test_decode_arguments(kw, status):
    assert _decode(_shape(), _opts(), _spec(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(tau=float("nan")), _lib.ERR_INVALID_ARG),
    (dict(patience=0), _lib.ERR_INVALID_ARG),
])
def test_decode_options(kw, status):
    assert _decode(_shape(), _opts(**kw), _spec()) == status
    assert _decode(_shape(num_q_heads=6), _opts(), _spec()) == _lib.ERR_UNSUPPORTED   # g = 3


def test_null_structs():
    lib = _lib.load()
    assert lib.art_quant_append(None, None, None, *[PTR] * 9, None) == _lib.ERR_INVALID_ARG
    assert lib.art_quant_read(ctypes.byref(_shape()), ctypes.byref(_spec()), None, *[PTR] * 9, None) == _lib.ERR_INVALID_ARG
    assert lib.art_decode_attention_quant(ctypes.byref(_shape()), None, ctypes.byref(_spec()), *[PTR] * 13,
                                          1 << 30, None) == _lib.ERR_INVALID_ARG


# ---- the binding, on CPU tensors ---------------------------------------------------

def test_new_cache():
    c = api.new_quant_cache(5, 3, 128, device="cpu")
    assert c.k.shape == (5, 3, 128, 128) and c.k.dtype == torch.float8_e4m3fn
    assert c.k_scale.shape == (5, 3, 2) and c.scale_tokens == 64
    c = api.new_quant_cache(5, 3, 16, dtype=torch.int8, device="cpu")
    assert c.scale_tokens == 16 and c.v.dtype == torch.int8
    assert api.new_quant_cache(5, 3, 128, scale_tokens=16, device="cpu").k_scale.shape == (5, 3, 8)
    with pytest.raises(ValueError):
        api.new_quant_cache(5, 3, 128, scale_tokens=48, device="cpu")
    with pytest.raises(ValueError):
        api.new_quant_cache(5, 3, 128, dtype=torch.uint8, device="cpu")


def test_binding_refuses_cpu_tensors():
    c = api.new_quant_cache(5, 2, 64, device="cpu")
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    table = torch.zeros((2, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensor"):
        api.quant_append(c, x, x, table, None)
    with pytest.raises(ValueError, match="GPU tensor"):
        api.quant_read(c, table, None, rows=4)
    with pytest.raises(ValueError, match="GPU tensor"):
        api.decode_attention_quant(torch.zeros((2, 8, 128), dtype=torch.bfloat16), c, table,
                                   torch.zeros(2, dtype=torch.int32), block_size=64, tau=0, phi=0,
                                   patience=1)
    with pytest.raises(ValueError, match="rows is needed"):
        api.quant_read(c, table, None)


# ---- the plain reference --------------------------------------------------------

@pytest.mark.parametrize("form", R.FORMATS)
def test_reference_encode_is_the_nearest_code(form):
    """By search over all codes; ties to the code whose last bit is zero."""
    rng = np.random.default_rng(1)
    vals = R.table(form)
    codes = [c for c in range(256) if not math.isnan(vals[c]) and abs(vals[c]) <= R.TOP[form] and c != 128]
    x = np.concatenate([rng.standard_normal(500) * np.exp2(rng.integers(-12, 8, 500)),
                        [vals[c] for c in codes],
                        [(vals[a] + vals[b]) / 2 for a, b in zip(codes, codes[1:])]])
    for v, got in zip(x, R.encode(x, form)):
        best = min(abs(vals[c] - v) for c in codes)
        near = [c for c in codes if abs(vals[c] - v) == best]
        assert any(vals[c] == vals[got] for c in near), (v, got)
        if len({vals[c] for c in near}) > 1:
            assert got % 2 == 0


@pytest.mark.parametrize("form", R.FORMATS)
def test_reference_scale(form):
    top = R.TOP[form]
    assert R.need(top, form) == 1.0 and R.need(np.nextafter(top, 1e9), form) == 2.0
    assert R.need(top / 2, form) == 0.5 and R.need(0.0, form) == 2.0 ** -120
    assert R.need(3.3e38, form) * top >= 3.3e38
