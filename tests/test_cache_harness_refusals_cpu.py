"""What PagedCache refuses before the library is called: on CPU tensors, so nothing here reaches a kernel."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2609_33184_amd import build_lib
from paper_2609_33184_amd import harness as H
from paper_2609_33184_amd import specstream as ss

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ss.lib_path()):
        build_lib.build(verbose=False)
    return ss.load()


@pytest.fixture
def reached(monkeypatch):
    """The library's calls that were made, none of which runs."""
    calls = []
    for name in ("ss_cache_write", "ss_cache_read", "ss_cache_attend"):
        monkeypatch.setattr(ss, name, lambda *a, _name=name, **kw: calls.append((_name, a)))
    return calls


def _cache(**kw):
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, **{"max_rows": 4, "device": "cpu", **kw})
    p.grow([20, 20])
    return p


def _rows(t=8):
    return torch.zeros(t, 2, 128, dtype=BF), torch.zeros(t, 8, 128, dtype=BF), torch.zeros(t, 8, 128), torch.zeros(t, 8)


BAD_STARTS = {
    "int64": torch.tensor([0, 4, 8]),
    "int16": torch.tensor([0, 4, 8], dtype=torch.int16),
    "short": torch.tensor([0, 4], dtype=torch.int32),
    "long": torch.tensor([0, 4, 8, 8], dtype=torch.int32),
    "two dimensions": torch.tensor([[0, 4, 8]], dtype=torch.int32),
    "strided": torch.tensor([0, 0, 4, 0, 8, 0], dtype=torch.int32)[::2],
    "elsewhere": torch.empty(3, dtype=torch.int32, device="meta"),
    "a list": [0, 4, 8],
}


@pytest.mark.parametrize("kind", sorted(BAD_STARTS))
def test_row_starts(kind, reached):
    p, (k, q, out, lse), bad = _cache(), _rows(), BAD_STARTS[kind]
    for call in (lambda: p.write(k, k, 0, bad), lambda: p.read(k, k, 8, 0, bad), lambda: p.attend(q, out, lse, 0, bad)):
        with pytest.raises(ValueError, match="row_start"):
            call()
    assert reached == []


def test_ends_of_a_read(reached):
    p, (k, _, _, _) = _cache(), _rows()
    start = torch.tensor([0, 4, 8], dtype=torch.int32)
    for bad in (torch.tensor([4, 4]), torch.tensor([4], dtype=torch.int32), torch.tensor([4, 0, 4, 0], dtype=torch.int32)[::2],
                torch.empty(2, dtype=torch.int32, device="meta"), [4, 4]):
        with pytest.raises(ValueError, match="end"):
            p.read(k, k, 8, 0, start, end=bad)
    assert reached == []
