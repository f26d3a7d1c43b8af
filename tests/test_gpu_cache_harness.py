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
