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
    monkeypatch.setattr(H.PagedCache, "_on_current_device", lambda self: None, raising=False)
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


T, H_, HKV = ss.SS_KV_TOKEN_MAJOR, ss.SS_KV_HEAD_MAJOR, ss.SS_KV_HEAD_MAJOR_KV


def test_chunks_that_a_read_accepts(reached):
    """8 rows of 2 KV heads: a chunk of its shape, a longer staging buffer, and the interleaved layout's views."""
    p, start = _cache(), torch.tensor([0, 4, 8], dtype=torch.int32)
    flat = torch.zeros(2, 5000, dtype=BF)
    both = torch.zeros(2, 8, 2, 128, dtype=BF)
    for k, v, layout in ((torch.zeros(8, 2, 128, dtype=BF), torch.zeros(8, 2, 128, dtype=BF), T),
                         (torch.zeros(2, 8, 128, dtype=BF), torch.zeros(2, 8, 128, dtype=BF), H_), (flat[0], flat[1], T),
                         (both, both[:, :, 1], HKV), (both[:, :, 0], both[:, :, 1], HKV), (both.view(-1), both.view(-1)[128:], HKV)):
        p.read(k, v, 8, 0, start, layout)
    assert [c[1][3:5] for c in reached[-3:]] == [(both.data_ptr(), both.data_ptr() + 256)] * 3 and len(reached) == 6


def test_chunks_that_a_read_refuses(reached):
    p, start = _cache(), torch.tensor([0, 4, 8], dtype=torch.int32)
    k = torch.zeros(8, 2, 128, dtype=BF)
    both, one = torch.zeros(2, 8, 2, 128, dtype=BF), torch.zeros(1, 8, 2, 128, dtype=BF)
    bad = [(x, layout) for layout in (T, H_) for x in (
        k.float(), k.half(), k[:7], k[:0], torch.zeros(8, 2, 256, dtype=BF)[..., ::2], torch.zeros(8, 4, 128, dtype=BF)[:, :2], k[:1].expand(8, 2, 128),
        torch.zeros(2, 8, 128, dtype=BF).transpose(0, 1), torch.empty(8, 2, 128, dtype=BF, device="meta"), None, k.data_ptr())]
    pairs = [(x, k, layout) for x, layout in bad] + [(k, x, layout) for x, layout in bad]
    pairs += [(both, both[:, :, 0], HKV), (both[:, :, 1], both[:, :, 0], HKV), (k, k, HKV), (both, both.clone()[:, :, 1], HKV),
              (both[:, :7], both[:, :7, 1], HKV), (both[:, :7, 0], both[:, :7, 1], HKV), (one, one[:, :, 1], HKV), (both.float(), both.float()[:, :, 1], HKV),
              (torch.zeros(8, 2, 2, 128, dtype=BF).transpose(0, 1), both[:, :, 1], HKV), (both[..., ::2], both[:, :, 1], HKV),
              (both, None, HKV)]
    for a, b, layout in pairs:
        with pytest.raises(ValueError):
            p.read(a, b, 8, 0, start, layout)
    for rows in (9, 1 << 40):                           # more rows than the chunk holds
        with pytest.raises(ValueError):
            p.read(k, k.clone(), rows, 0, start)
    assert reached == []


def test_rows_on_another_device(reached):
    p, (k, q, out, lse) = _cache(), _rows()
    there = lambda x: torch.empty_like(x, device="meta")
    for call in (lambda: p.write(there(k), k, 0), lambda: p.write(k, there(k), 0), lambda: p.attend(there(q), out, lse, 0),
                 lambda: p.attend(q, there(out), lse, 0), lambda: p.attend(q, out, there(lse), 0),
                 lambda: p.attend(q, out, lse, 0, prev=(there(out), lse)), lambda: p.attend(q, out, lse, 0, prev=(out, there(lse)))):
        with pytest.raises(ValueError, match="meta"):
            call()
    assert reached == []
    p.write(k, k, 0)
    p.attend(q, out, None, 0, prev=(out, lse))
    assert [c[0] for c in reached] == ["ss_cache_write", "ss_cache_attend"]


def test_devices_without_the_cache(monkeypatch):
    """A cache on the CPU counts pages and runs nothing; one of another GPU than the current runs nothing either."""
    calls = []
    for name in ("ss_cache_write", "ss_cache_read", "ss_cache_attend"):
        monkeypatch.setattr(ss, name, lambda *a, **kw: calls.append(a))
    p, (k, q, out, lse) = _cache(), _rows()
    every = (lambda: p.write(k, k, 0), lambda: p.read(k, k.clone(), 8, 0), lambda: p.attend(q, out, lse, 0))
    for call in every:
        with pytest.raises(ValueError, match="CPU"):
            call()

    class Pages:
        device = torch.device("cuda", 1)

    p.pages = Pages()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current"):
        p._on_current_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    p._on_current_device()
    assert calls == []


def test_counts_are_whole_numbers():
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, device="cpu")
    p.grow([20, 5])
    state = lambda: (list(p.tokens), [list(x) for x in p.owned], list(p.free), p.table.tolist(), p.end.tolist())
    before = state()
    for call in (p.grow, p.release):
        for rows in ([0, 1.5], [13.0, 1], [1, "1"], [1, None], torch.tensor([1.0, 1.0])):
            with pytest.raises(TypeError):
                call(rows)
            assert state() == before
    for rows in (torch.tensor([13, 1]), (torch.tensor(13).numpy(), True)):
        p.grow(rows)
        assert p.tokens == [33, 6] and p.end.tolist() == [33, 6] and all(type(n) is int for n in p.tokens)
        p.release(rows)
        assert p.tokens == [20, 5] and p.end.tolist() == [20, 5] and [len(x) for x in p.owned] == [2, 1]


def test_released_pages_leave_the_table():
    """What a request no longer owns it does not reach, whoever gets the page next."""
    p = H.PagedCache(3, 8, 2, 100, ss.SS_CACHE_BF16, 16, num_pages=12, device="cpu")
    p.grow([60, 17, 33])
    for release, grow in (([30, 0, 1], [0, 40, 0]), ([0, 57, 0], [10, 0, 30]), ([40, 0, 62], [0, 0, 0])):
        p.release(release)
        p.grow(grow)
        for b, owned in enumerate(p.owned):
            assert p.table[b].tolist() == owned + [-1] * (p.table.shape[1] - len(owned))


def test_a_change_that_fails_changes_nothing(monkeypatch):
    """Memory that runs out, pinned or on the device, leaves the host's counts as they were."""
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, device="cpu")
    p.grow([20, 5])
    state = lambda: (list(p.tokens), [list(x) for x in p.owned], list(p.free), p.table.tolist(), p.end.tolist())
    before = state()

    def full(*a, **kw):
        raise RuntimeError("out of memory")

    with monkeypatch.context() as m:
        m.setattr(torch, "tensor", full)
        for call, rows in ((p.grow, [30, 1]), (p.release, [20, 1])):
            with pytest.raises(RuntimeError):
                call(rows)
            assert state() == before
    p.grow([30, 1])
    assert p.tokens == [50, 6] and p.table[0].tolist() == p.owned[0] and len(p.owned[0]) == 4
