"""PagedCache on the GPU: its table and ends follow the host's without making it wait."""
from __future__ import annotations

import pytest
import torch

from paper_2609_33184_amd import harness as H
from paper_2609_33184_amd import specstream as ss

pytestmark = pytest.mark.gpu


def _busy(stream=None, products=60):
    """About 36 ms of work on a stream; its event, and what it uses."""
    a = torch.ones(8192, 8192, dtype=torch.bfloat16, device="cuda")
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
        for _ in range(products):
            torch.mm(a, a, out=b)
        done.record()
    return done, a, b


def _as_the_host_has_it(p):
    torch.cuda.synchronize()
    table = p.table.tolist()
    assert p.end.tolist() == p.tokens
    for b, owned in enumerate(p.owned):
        assert table[b][:len(owned)] == owned
    assert sorted([x for o in p.owned for x in o] + p.free) == list(range(p.desc.num_pages))


def test_growing_does_not_wait_for_the_gpu():
    p = H.PagedCache(16, 8, 2, 2000, ss.SS_CACHE_MXFP8, 16)
    p.grow([1] * 16)
    p.release([1] * 16)
    _as_the_host_has_it(p)
    work = _busy()
    for i in range(40):
        p.grow([(i * b) % 23 for b in range(16)])
        p.release([(i * b) % 23 // 2 for b in range(16)])
    assert not work[0].query()
    _as_the_host_has_it(p)


def test_counts_do_not_change_in_a_graph():
    """A replay would count the same tokens again without their pages."""
    p = H.PagedCache(2, 8, 2, 100, ss.SS_CACHE_MXFP8, 16)
    p.grow([20, 3])
    x = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x += 1
        for call in (p.grow, p.release):
            with pytest.raises(RuntimeError, match="captured"):
                call([1, 1])
    g.replay()
    assert p.tokens == [20, 3]
    _as_the_host_has_it(p)


def _filled(max_rows=2, num_pages=None):
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = lambda t, heads: torch.randn(t, heads, 128, generator=g, device="cuda").to(torch.bfloat16)
    p = H.PagedCache(3, 8, 2, 4000, ss.SS_CACHE_MXFP8, 16, max_rows=max_rows, num_pages=num_pages)
    p.grow([3000, 40, 900])
    start = torch.tensor([0, 3000, 3040, 3940], dtype=torch.int32, device="cuda")
    p.write(rows(3940, 2), rows(3940, 2), torch.cuda.current_stream().cuda_stream, start)
    return p, rows


def test_changes_come_after_the_calls_before_them():
    """An attention and a read that still wait on another stream see the table and the ends as they were, and the
    released pages keep what they hold until both are done."""
    p, rows = _filled(num_pages=300)
    home, side = torch.cuda.current_stream(), torch.cuda.Stream()
    q, out, lse = rows(6, 8), torch.empty(6, 8, 128, device="cuda"), torch.empty(6, 8, device="cuda")
    k, v = torch.empty(2, 60, 2, 128, dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 20, 40, 60], dtype=torch.int32, device="cuda")
    p.attend(q, out, lse, home.cuda_stream)
    p.read(k, v, 60, home.cuda_stream, some)
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, lse, k, v)]
    for x in (out, lse, k, v):
        x.fill_(7.0)
    new = rows(2000, 2)
    start = torch.tensor([0, 0, 2000, 2000], dtype=torch.int32, device="cuda")
    work = _busy(side)
    p.attend(q, out, lse, side.cuda_stream)
    p.read(k, v, 60, side.cuda_stream, some)
    p.release([2900, 0, 850])
    p.grow([0, 2000, 0])                               # takes the released pages
    p.write(new, new, home.cuda_stream, start)
    assert not work[0].query()
    torch.cuda.synchronize()
    for got, x in zip((out, lse, k, v), want):
        assert torch.equal(got, x)
    _as_the_host_has_it(p)


def test_calls_come_after_the_changes_before_them():
    p, rows = _filled()
    side = torch.cuda.Stream()
    start = torch.tensor([0, 5, 5, 70], dtype=torch.int32, device="cuda")
    new = rows(70, 2)
    torch.cuda.synchronize()
    work = _busy()
    p.grow([5, 0, 65])
    p.write(new, new, side.cuda_stream, start)
    assert not work[0].query()
    torch.cuda.synchronize()
    k, v = torch.empty(2, 70, 2, 128, dtype=torch.bfloat16, device="cuda")
    p.read(k, v, 70, torch.cuda.current_stream().cuda_stream, start)
    torch.cuda.synchronize()
    assert torch.equal(k, v) and (k - new).abs().max() <= 2.0 ** -4 * new.abs().max()        # half a step of e4m3


def test_attentions_on_several_streams():
    """They share the cache's workspace and give the results of each by itself; so do a graph's."""
    p, rows = _filled()
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    qs = [rows(6, 8) for _ in range(6)]
    out, want = torch.empty(6, 6, 8, 128, device="cuda"), torch.empty(6, 6, 8, 128, device="cuda")
    for q, o in zip(qs, want):
        p.attend(q, o, None, streams[0].cuda_stream)
    torch.cuda.synchronize()
    for i in range(30):
        out.fill_(7.0)
        torch.cuda.synchronize()
        for j, (q, o) in enumerate(zip(qs, out)):
            p.attend(q, o, None, streams[(i + j * (1 + i % 2)) % 3].cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for q, o in zip(qs, out):
            p.attend(q, o, None, torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        p.attend(qs[0], out[0], None, streams[0].cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
