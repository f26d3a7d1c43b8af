"""The paged cache without a GPU: page sizes, workspaces, refusals, and the
oracle's number formats.  Every call here is refused before it looks at a
device (pointers are never dereferenced)."""
from __future__ import annotations

import math
import os

import numpy as np
import pytest

from oracle import bf16_bits_to_f64
from oracle import cache as oc
from paper_2609_33184_amd import build_lib
from paper_2609_33184_amd import specstream as ss

PAGES, TABLE, K, V, ROWS, END, WS = (0x7F0000000000 + i * (1 << 24) for i in range(7))


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ss.lib_path()):
        build_lib.build(verbose=False)
    return ss.load()


def _desc(**kw):
    a = dict(num_requests=4, num_kv_heads=2, format=ss.SS_CACHE_MXFP8, page_tokens=32, num_pages=64, table_stride=16,
             num_q_heads=8, max_rows=2)
    a.update(kw)
    return ss.make_cache_desc(**a)


@pytest.mark.parametrize("fmt", (oc.BF16, oc.MXFP8, oc.MXFP4))
@pytest.mark.parametrize("page", (16, 256))
@pytest.mark.parametrize("hkv", (1, 5))
def test_page_bytes(fmt, page, hkv):
    assert ss.ss_cache_page_bytes(_desc(format=fmt, page_tokens=page, num_kv_heads=hkv, num_q_heads=hkv)) == oc.page_bytes(fmt, hkv, page)


BAD = [
    (dict(num_requests=0), "num_requests", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(num_requests=4097), "num_requests", ss.SS_ERR_UNSUPPORTED),
    (dict(num_kv_heads=0), "num_kv_heads", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(num_kv_heads=65536), "num_kv_heads", ss.SS_ERR_UNSUPPORTED),
    (dict(head_dim=64), "head_dim", ss.SS_ERR_UNSUPPORTED),
    (dict(format=3), "format", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(format=-1), "format", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(page_tokens=8), "page_tokens", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(page_tokens=48), "page_tokens", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(page_tokens=512), "page_tokens", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(num_pages=0), "num_pages", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(table_stride=0), "table_stride", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(table_stride=(1 << 25) + 1), "table_stride", ss.SS_ERR_UNSUPPORTED),
    (dict(table_stride=1 << 25, num_requests=64), "table_stride", ss.SS_ERR_UNSUPPORTED),
    (dict(page_stride=2 * 32 * 2 * 132 - 16), "page_stride", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(page_stride=2 * 32 * 2 * 132 + 8), "page_stride", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(page_stride=-16), "page_stride", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(max_rows=0), "max_rows", ss.SS_ERR_INVALID_ARGUMENT),
]
BAD_ATTEND = [
    (dict(num_q_heads=0), "num_q_heads", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(num_q_heads=9), "num_q_heads", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(max_rows=9), "max_rows", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(max_rows=8, num_q_heads=18), "rows per KV head", ss.SS_ERR_UNSUPPORTED),
    (dict(softmax_scale=0.0), "softmax_scale", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(softmax_scale=float("nan")), "softmax_scale", ss.SS_ERR_INVALID_ARGUMENT),
    (dict(causal=2), "causal", ss.SS_ERR_INVALID_ARGUMENT),
]


def _refused(status, word, fn, *a, **kw):
    with pytest.raises(ss.SpecStreamError) as e:
        fn(*a, **kw)
    assert e.value.status == status and word in str(e.value), e.value


def _write(d, pages=PAGES, table=TABLE, k=K, v=V, num_rows=8, end=END, **kw):
    ss.ss_cache_write(d, pages, table, k, v, num_rows, end, **kw)


def _read(d, pages=PAGES, table=TABLE, k=K, v=V, num_rows=8, end=END, **kw):
    ss.ss_cache_read(d, pages, table, k, v, num_rows, end, **kw)


def _attend(d, pages=PAGES, table=TABLE, q=K, num_rows=8, end=END, out=V, workspace=WS, workspace_bytes=1 << 30, **kw):
    ss.ss_cache_attend(d, pages, table, q, num_rows, end, out, workspace=workspace, workspace_bytes=workspace_bytes, **kw)


@pytest.mark.parametrize("kw,word,status", BAD, ids=lambda x: str(x)[:40])
def test_descriptors_that_every_call_refuses(kw, word, status):
    d = _desc(**kw)
    assert ss.ss_cache_page_bytes(d) == 0 and word in ss.ss_last_error()
    assert ss.ss_cache_attend_workspace_bytes(d) == 0 and word in ss.ss_last_error()
    for call in (_write, _read, _attend):
        _refused(status, word, call, d)


@pytest.mark.parametrize("kw,word,status", BAD_ATTEND, ids=lambda x: str(x)[:40])
def test_descriptors_that_the_attention_refuses(kw, word, status):
    d = _desc(**kw)
    assert ss.ss_cache_page_bytes(d) > 0
    assert ss.ss_cache_attend_workspace_bytes(d) == 0 and word in ss.ss_last_error()
    _refused(status, word, _attend, d)


@pytest.mark.parametrize("call", (_write, _read, _attend))
def test_shared_arguments(call):
    d, bad = _desc(), ss.SS_ERR_INVALID_ARGUMENT
    for kw in (dict(pages=0), dict(pages=PAGES + 8), dict(table=0), dict(table=TABLE + 2), dict(end=0), dict(end=END + 1),
               dict(row_start=ROWS + 2, num_rows=3), dict(num_rows=0), dict(num_rows=-1), dict(num_rows=7)):
        _refused(bad, "", call, d, **kw)


def test_rows_arguments():
    d, bad = _desc(), ss.SS_ERR_INVALID_ARGUMENT
    for call in (_write, _read):
        for kw in (dict(k=0), dict(v=0), dict(k=K + 8), dict(v=V + 2)):
            _refused(bad, "k and v", call, d, **kw)
    for stride in (-256, 248, 260):
        _refused(bad, "row_stride", _write, d, row_stride=stride)
    for layout in (-1, 3):
        _refused(bad, "kv_layout", _read, d, kv_layout=layout)
    _refused(bad, "head_dim", _read, d, kv_layout=ss.SS_KV_HEAD_MAJOR_KV)


def test_attend_arguments():
    d, bad = _desc(), ss.SS_ERR_INVALID_ARGUMENT
    need = ss.ss_cache_attend_workspace_bytes(d)
    assert need > 0 and need % 256 == 0
    for kw in (dict(q=0), dict(q=K + 8), dict(out=0), dict(out=V + 4), dict(lse=V + 2), dict(q_row_stride=1016), dict(q_row_stride=1028),
               dict(prev_out=V), dict(prev_lse=V), dict(prev_out=V + 8, prev_lse=V), dict(prev_out=V, prev_lse=V + 1)):
        _refused(bad, "", _attend, d, **kw)
    for kw in (dict(workspace=0), dict(workspace=WS + 64), dict(workspace_bytes=need - 1)):
        _refused(ss.SS_ERR_WORKSPACE, "workspace", _attend, d, **kw)


def test_null_descriptor():
    assert ss.load().ss_cache_page_bytes(None) == 0
    assert ss.load().ss_cache_attend_workspace_bytes(None) == 0
    assert ss.load().ss_cache_write(None, PAGES, TABLE, K, V, 0, 8, None, END, None) == ss.SS_ERR_INVALID_ARGUMENT


# ---- the oracle's formats -------------------------------------------------------------------------
def test_code_values():
    v8, v4 = oc.code_values(oc.MXFP8), oc.code_values(oc.MXFP4)
    assert list(v4[:8]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6] and list(v4[8:]) == [-x for x in v4[:8]]
    assert v8[0x7E] == 448 and v8[0x01] == 2.0 ** -9 and v8[0x08] == 2.0 ** -6 and v8[0xB8] == -1 and math.isnan(v8[0x7F])


def _bits(x):
    w = np.asarray(x, np.float32).view(np.uint32)
    return (w >> 16).astype(np.uint16)


@pytest.mark.parametrize("fmt,top,half", ((oc.MXFP8, 448.0, 2.0 ** -4), (oc.MXFP4, 6.0, 0.25)))
def test_encode_is_nearest_and_its_exponent_smallest(fmt, top, half):
    """half: half a step of the format, relative to the value (e2m1's coarsest: 2 to 3)."""
    rng = np.random.default_rng(3)
    x = bf16_bits_to_f64(_bits(rng.standard_normal((64, 128)) * np.exp2(rng.integers(-40, 40, (64, 1)))))
    bits = _bits(x)
    code, scale = oc.encode(bits, fmt)
    got = oc.decode(code, scale, fmt)
    peak = np.abs(x).reshape(64, 4, 32).max(-1)
    f = np.exp2(scale.astype(np.float64) - 127)
    assert (peak <= top * f).all() and (peak > top * f / 2).all()
    smallest = (2.0 ** -6 if fmt == oc.MXFP8 else 1.0) * np.repeat(f, 32, -1)     # normal number: below it steps are even
    assert (np.abs(got - x) <= half * np.maximum(np.abs(x), smallest)).all()


def test_encode_border_values():
    x = np.zeros((6, 128), np.float32)
    x[0, 0], x[0, 1] = 448.0, -0.0
    x[1, 0] = 450.0                       # above F: the next exponent
    x[2, 0], x[2, 32] = np.inf, 1.0       # one block of the row is no number
    x[3, 64] = np.nan
    x[4, :] = 2.0 ** -126
    code, scale = oc.encode(_bits(x), oc.MXFP8)
    assert scale[0, 0] == 127 and code[0, 0] == 0x7E and code[0, 1] == 0x80 and scale[0, 1] == 16
    assert scale[1, 0] == 128 and code[1, 0] == 0x76
    assert scale[2, 0] == 255 and (code[2, :32] == 0).all() and scale[2, 1] == 127 - 8
    assert list(scale[3]) == [16, 16, 255, 16] and np.isnan(oc.decode(code, scale, oc.MXFP8)[3, 64:96]).all()
    assert (scale[4] == 16).all() and (code[4] == 0).all() and scale[5, 0] == 16
