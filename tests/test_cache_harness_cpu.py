"""The harness's page bookkeeping, on CPU tensors: no call of the library looks at a device here."""
from __future__ import annotations

import os

import pytest

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
