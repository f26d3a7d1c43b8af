"""The harness's page bookkeeping, on CPU tensors: no call of the library looks at a device here."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2609_33184_amd import build_lib
from paper_2609_33184_amd import harness as H
from paper_2609_33184_amd import specstream as ss


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ss.lib_path()):
        build_lib.build(verbose=False)
    return ss.load()


def _state(p):
    return list(p.tokens), [list(x) for x in p.owned], list(p.free), p.table.tolist(), p.end.tolist()


def test_pages_come_and_go():
    p = H.PagedCache(3, 8, 2, 100, ss.SS_CACHE_MXFP8, 16, num_pages=9, device="cpu")
    p.grow([16, 17, 0])
    assert p.tokens == [16, 17, 0] and p.end.tolist() == [16, 17, 0] and [len(x) for x in p.owned] == [1, 2, 0]
    for b in range(3):
        assert p.table[b, :len(p.owned[b])].tolist() == p.owned[b]
    p.grow([1, 15, 1])
    assert [len(x) for x in p.owned] == [2, 2, 1] and len(p.free) == 4
    pages = [x for o in p.owned for x in o] + p.free
    assert sorted(pages) == list(range(9))
    p.release([1, 16, 0])
    assert p.tokens == [16, 16, 1] and [len(x) for x in p.owned] == [1, 1, 1] and len(p.free) == 6


def test_a_full_cache_refuses_and_stays_as_it_was():
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, num_pages=5, device="cpu")
    p.grow([40, 16])
    before = _state(p)
    for rows in ([1, 33], [30, 0], [0, 49]):      # too many pages; too long for the table
        with pytest.raises(MemoryError):
            p.grow(rows)
        assert _state(p) == before
    with pytest.raises(ss.SpecStreamError):
        H.PagedCache(2, 9, 2, 64, ss.SS_CACHE_BF16, 16, device="cpu")


def test_counts_are_checked_before_anything_moves():
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, device="cpu")
    p.grow([20, 5])
    before = _state(p)
    for call, rows in ((p.grow, [1]), (p.grow, [1, -1]), (p.grow, [1, 1, 1]), (p.release, [21, 0]), (p.release, [1, -1]),
                       (p.release, [3])):
        with pytest.raises(ValueError):
            call(rows)
        assert _state(p) == before
    p.release([20, 5])
    assert p.tokens == [0, 0] and len(p.free) == 8


def test_rows_whose_memory_the_calls_cannot_describe_are_refused():
    """Every refusal comes before the library is called, so the CPU tensors reach no kernel."""
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, max_rows=4, device="cpu")
    p.grow([4, 4])
    k = torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    fused = torch.zeros(8, 4, 128, dtype=torch.bfloat16)
    assert p._row_stride(k, 2) == 256 and p._row_stride(fused[:, 2:], 2) == 512
    assert p._row_stride(k[:1].expand(1, 2, 128), 2) == 0 and p._row_stride(k[:0], 2) == 0
    for bad in (k.float(), k[:1].expand(8, 2, 128), k.transpose(0, 1), torch.zeros(2, 8, 128, dtype=torch.bfloat16).transpose(0, 1),
                k.reshape(8, 256), torch.zeros(8, 2, 256, dtype=torch.bfloat16)[..., ::2], k[:, :1].expand(8, 2, 128)):
        with pytest.raises(ValueError):
            p.write(bad, k, 0)
        with pytest.raises(ValueError):
            p.write(k, bad, 0)
    for v in (k[:7], fused[:, :2]):                # fewer rows than k; another row stride
        with pytest.raises(ValueError):
            p.write(k, v, 0)
    q, out, lse = torch.zeros(8, 8, 128, dtype=torch.bfloat16), torch.zeros(8, 8, 128), torch.zeros(8, 8)
    for args in ((q.float(), out, lse), (q[:1].expand(8, 8, 128), out, lse), (q, out[:7], lse), (q, out.half(), lse),
                 (q, out.transpose(0, 1), lse), (q, out, lse[:, :4]), (q, out, lse.double())):
        with pytest.raises(ValueError):
            p.attend(*args, 0)
    for prev in ((out[:7], lse), (out, lse[:7]), (out.half(), lse), (out, lse.t())):
        with pytest.raises(ValueError):
            p.attend(q, out, None, 0, prev=prev)
