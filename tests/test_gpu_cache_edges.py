"""Trees of many rows over the paged cache where some rows see a value that is no number and others do not: at a window's
edges, among its first tokens, beside pages that are none and slots that nobody wrote (tolerances: see test_gpu_cache)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import tree as ot
from test_gpu_cache import FORMATS, IDS, Cache, _ints, _normal
from test_gpu_cache_tree import TreeRows, _trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((4, 10), (4, 24), (8, 64)))
@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_window_edges(fmt, hq, n, value):
    rng = np.random.default_rng(n)
    end0, window, sinks = 230 + n, 50, 3
    words = _trees(rng, (n, 20))
    sees = [ot.tree_sees(words[0][i], i, n, end0, window, sinks) for i in range(n)]
    low = [min(t for t in s if t >= sinks) for s in sees]
    for t in sorted({0, sinks - 1, sinks, 100, min(low) - 1, min(low), max(low), max(low) - 1, end0 - n - 1, end0 - n, end0 - 1}):
        end = [end0, 50]
        for which in (0, 1):
            kv = [_normal(5, sum(end), 1, 128), _normal(6, sum(end), 1, 128)]
            kv[which][t, 0, 77] = value
            c = Cache(fmt, 1, 32, end)
            c.fill_tokens(end, 5, *kv)
            r = TreeRows(c, hq, words, end, window=window, sinks=sinks).run()
            torch.cuda.synchronize()
            want, _ = r.want()
            got = r.out.cpu().numpy()
            for i in range(n):
                if t in sees[i]:
                    if which:
                        assert not np.isfinite(got[i, :, 77]).any()
                        assert np.isfinite(got[i, :, :64]).all() and np.isfinite(got[i, :, 96:]).all()
                else:
                    assert np.abs(got[i] - want[i]).max() <= r._bound(), (t, which, i)
            assert np.abs(got[n:] - want[n:]).max() <= r._bound()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("fill", (0xFF, 0x7F))
@pytest.mark.parametrize("window", (0, 90))
def test_pages_that_are_none_among_no_numbers(fmt, page, fill, window):
    """Slots that nobody wrote, and the page that stands in for one that is none, hold what is no number."""
    rng = np.random.default_rng(page)
    end = [200, 270, 77, 140]
    c = Cache(fmt, 2, page, end, fill=fill)
    c.fill_tokens(end, 5)
    zero = int(np.argwhere(c.table == 0)[0][0]) if (c.table == 0).any() else -1
    for b in range(4):
        if b != zero:
            c.table[b, (b + 1) % (end[b] // page)] = (-1, c.num_pages, -7, 1 << 30)[b]
    held = oc.parts(c.pages, fmt, page)
    if zero < 0:
        for part in held:
            part[0] = fill
        c.dev.copy_(torch.from_numpy(c.pages))
    c.dtable = _ints(c.table)
    TreeRows(c, 8, _trees(rng, (40, 64, 30, 20)), end, window=window, sinks=20 if window else 0).run().check()
