"""Trees and windows over the paged cache, rotated appends and kept paths on the GPU, against the float64 oracle.

Attention: the same sums as plain attention over fewer tokens, so the same tolerances (5e-6 in the 2-norm, and the
worst case of a value, ``Rows._bound``; see test_gpu_cache).

Turning.  The angle is the product of 64 bits that the oracle takes; the series are off by 7e-12, below 2^-37, and a
handful of roundings of 2^-53 follow: together less than 2^-34 of the pair's length.  A number that near the oracle's is
rounded to fp32 and then to bf16, so the result lies between the roundings of the oracle's value less and more 2^-34.  K
is stored from the bf16 value by exact rules, so a cache is compared byte for byte with the write of the turned rows
that the GPU returned as Q.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import bf16_bits_to_f64
from oracle import cache as oc
from oracle import tree as ot
from paper_2609_33184_amd import harness as H
from paper_2609_33184_amd import specstream as ss
from test_gpu_cache import FORMATS, IDS, Cache, Rows, _bits, _ints, _normal
from tree_inputs import as_int64, depths_of, path_to, random_parents, words_of

pytestmark = pytest.mark.gpu


class TreeRows(Rows):
    """Queries of a call whose requests' last tokens are trees (words: per request)."""

    def __init__(self, c, hq, words, end, window=0, sinks=0, **kw):
        rows = [len(w) for w in words]
        self.words, self.window, self.sinks = [x for w in words for x in w], window, sinks
        most = kw.pop("max_rows", max(rows))
        super().__init__(c, hq, rows, end, max_rows=1, **kw)
        self.desc.max_rows = most
        n = ss.ss_cache_attend_tree_workspace_bytes(self.desc)
        assert n > 0, ss.ss_last_error()
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        self.tree = torch.from_numpy(as_int64(self.words + [-1 & (1 << 64) - 1] * (self.T - len(self.words)))).cuda()

    def run(self, stream=None):
        s = torch.cuda.current_stream() if stream is None else stream
        po, pl = (None, None) if self.prev is None else (self.prev[0].data_ptr(), self.prev[1].data_ptr())
        ss.ss_cache_attend_tree(self.desc, *self.c.at(), self.q.data_ptr(), self.T, self.dend.data_ptr(), self.tree.data_ptr(),
                                self.out.data_ptr(), self.lse.data_ptr(), self.dstart.data_ptr(), self.window, self.sinks, po, pl,
                                self.ws.data_ptr(), self.ws.numel(), self.stride, s.cuda_stream)
        return self

    def want(self):
        prev = None if self.prev is None else (self.prev[0].cpu().numpy(), self.prev[1].cpu().numpy())
        n = int(self.start[-1])
        return ot.attend(_bits(self.q)[:n], self.c.pages, self.c.fmt, self.c.page, self.c.table, self.start, self.end, self.scale,
                         lambda row, i, n, end: ot.tree_sees(self.words[row], i, n, end, self.window, self.sinks), prev)


class WindowRows(Rows):
    def __init__(self, c, hq, rows, end, window, sinks, **kw):
        self.window, self.sinks = window, sinks
        super().__init__(c, hq, rows, end, **kw)

    def run(self, stream=None):
        s = torch.cuda.current_stream() if stream is None else stream
        po, pl = (None, None) if self.prev is None else (self.prev[0].data_ptr(), self.prev[1].data_ptr())
        ss.ss_cache_attend_window(self.desc, *self.c.at(), self.q.data_ptr(), self.T, self.dend.data_ptr(), self.out.data_ptr(),
                                  self.window, self.sinks, self.lse.data_ptr(), self.dstart.data_ptr(), po, pl, self.ws.data_ptr(),
                                  self.ws.numel(), self.stride, s.cuda_stream)
        return self

    def want(self):
        prev = None if self.prev is None else (self.prev[0].cpu().numpy(), self.prev[1].cpu().numpy())
        n = int(self.start[-1])
        return ot.attend(_bits(self.q)[:n], self.c.pages, self.c.fmt, self.c.page, self.c.table, self.start, self.end, self.scale,
                         lambda row, i, n, end: ot.window_sees(i, n, end, self.window, self.sinks), prev)


def _trees(rng, sizes):
    return [words_of(random_parents(rng, n)) if n else [] for n in sizes]


# ---- windows -------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("window,sinks", ((1, 0), (3, 1), (32, 0), (33, 4), (64, 32), (100, 33), (5, 200), (1 << 30, 0), (2147483647, 2147483647)))
def test_window_lengths(fmt, window, sinks):
    """Lengths around tiles and pages; windows that hold less than the rows, part of a tile, or everything."""
    end = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700, 3]
    rows = [1, 1, 4, 3, 2, 1, 4, 4, 2, 3, 1, 2, 4, 4, 4, 1, 3, 2, 4, 4]
    c = Cache(fmt, 2, 16, end)
    c.fill_tokens(end, 9)
    WindowRows(c, 8, rows, end, window, sinks).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,hkv,n", ((1, 1, 1), (8, 2, 5), (32, 8, 6), (48, 8, 5), (64, 8, 8), (17, 1, 3)))
def test_window_heads(fmt, hq, hkv, n):
    rng = np.random.default_rng(hq)
    rows = [n, 0] + list(rng.integers(1, n + 1, 3))
    end = [1300, 40, 333, 257, 7]
    c = Cache(fmt, hkv, 32, end)
    c.fill_tokens(end, 5)
    WindowRows(c, hq, rows, end, 200, 3, extra=3, wide=2).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
def test_window_requests_by_the_hundred(fmt):
    """Waves that work alone, requests of every length around the window."""
    rng = np.random.default_rng(3)
    B, hkv = 140, 8
    end = rng.integers(0, 260, B) * (rng.random(B) < 0.8)
    end[70] = 2100
    c = Cache(fmt, hkv, 32, end)
    c.fill_tokens(end, 3)
    WindowRows(c, 16, rng.integers(0, 4, B), end, 70, 5).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hkv,window", ((1, 700), (2, 1500), (16, 600), (48, 700)))
@pytest.mark.parametrize("tree", (0, 1))
def test_window_parts(fmt, hkv, window, tree):
    """A window among short requests: a request's tiles in many parts, fewer tiles than parts, one, none; joined in place."""
    rng = np.random.default_rng(window + hkv)
    end = [3000, 0, 5, 1400, 70, 33, 1]
    rows = [4, 3, 2, 1, 0, 4, 1]
    if tree:
        rows = [24, 5, 9, 40, 0, 33, 1] if hkv < 16 else [6, 5, 3, 2, 0, 6, 1]
    c = Cache(fmt, hkv, 32, end)
    c.fill_tokens(end, 3)
    T, hq = sum(rows), 4 * hkv
    prev = (torch.randn(T, hq, 128, generator=torch.Generator().manual_seed(1)).cuda(), torch.randn(T, hq, generator=torch.Generator().manual_seed(2)).cuda())
    prev[1][::5] = float("-inf")
    r = TreeRows(c, hq, _trees(rng, rows), end, window, 40, prev=prev) if tree else WindowRows(c, hq, rows, end, window, 40, prev=prev)
    r.run().check()
    first = r.out.clone()
    r.out.copy_(prev[0])
    r.lse.copy_(prev[1])
    r.prev = (r.out, r.lse)
    r.run()
    torch.cuda.synchronize()
    assert torch.equal(first, r.out)


@pytest.mark.parametrize("hkv,hq,tree,window", ((2, 8, 0, 600), (1, 16, 1, 600), (2, 64, 0, 40), (1, 8, 1, 100)))
def test_window_parts_of_many_requests(hkv, hq, tree, window):
    """More than 64 requests, most of them short or empty, a workgroup to each (request, head) and block of rows."""
    rng = np.random.default_rng(window)
    B = 131
    end = rng.integers(0, 40, B) * (rng.random(B) < 0.7)
    end[[3, 63, 64, 130]] = 1400, 33, 900, 1200
    rows = rng.integers(0, 13 if tree else 3, B)
    rows[[3, 64, 130]] = (12, 11, 9) if tree else (2, 1, 2)
    c = Cache(oc.MXFP8, hkv, 32, end)
    c.fill_tokens(end, 3)
    r = TreeRows(c, hq, _trees(rng, rows), end, window, 7, extra=2) if tree else WindowRows(c, hq, rows, end, window, 7, extra=2)
    r.run().check()


def test_window_of_everything_equals_plain_attention():
    """No token is hidden and none skipped: the same tiles in the same shares give the same bits."""
    end, rows = [700, 33, 0, 64], [3, 1, 2, 4]
    c = Cache(oc.MXFP8, 2, 32, end)
    c.fill_tokens(end, 9)
    a = Rows(c, 8, rows, end).run().check()
    b = WindowRows(c, 8, rows, end, 1 << 20, 0).run().check()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
def test_window_pages_given_back(fmt):
    """Pages behind the sinks and before the window have no number; what they held is not needed."""
    end, rows, window, sinks = [900, 650], [2, 3], 100, 5
    c = Cache(fmt, 2, 16, end)
    c.fill_tokens(end, 5)
    r = WindowRows(c, 8, rows, end, window, sinks).run().check()
    before = r.out.clone()
    for b in range(2):
        c.table[b, 2:(end[b] - rows[b] - window) // 32 * 2] = -1      # whole tiles behind the sinks'
    c.dtable = _ints(c.table)
    r.out.fill_(7.0)
    r.run().check()
    assert torch.equal(before, r.out)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((4, 1), (8, 5), (16, 8)))
@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_window_no_number_outside(fmt, hq, n, value):
    """A NaN or infinity in K or V reaches the rows that see it and no other: at the window's edges, among the sinks."""
    hkv, end0, window, sinks = max(1, hq * n // 64), 200, 50, 3
    G = hq // hkv
    first = end0 - n
    for t in (0, sinks - 1, sinks, 31, 100, first - window, first - window + 1, first - window + 2, first, end0 - 1):
        end = [end0, 50]
        for which in (0, 1):
            kv = [_normal(5, sum(end), hkv, 128), _normal(6, sum(end), hkv, 128)]
            kv[which][t, 0, 77] = value
            c = Cache(fmt, hkv, 32, end)
            c.fill_tokens(end, 5, *kv)
            r = WindowRows(c, hq, [n, 2], end, window, sinks).run()
            torch.cuda.synchronize()
            want, _ = r.want()
            got = r.out.cpu().numpy()
            for i in range(n):
                if t in ot.window_sees(i, n, end0, window, sinks):
                    assert not np.isfinite(got[i, :G, 77]).any() or which == 0 and fmt == oc.BF16
                    assert np.abs(got[i, G:] - want[i, G:]).max(initial=0) <= r._bound()
                else:
                    assert np.abs(got[i] - want[i]).max() <= r._bound()
            assert np.abs(got[n:] - want[n:]).max() <= r._bound()


def test_window_joined():
    end, rows = [300, 0, 64, 0], [3, 2, 1, 2]
    c = Cache(oc.MXFP8, 2, 32, end)
    c.fill_tokens(end, 5)
    T = sum(rows)
    po, pl = torch.randn(T, 8, 128, generator=torch.Generator().manual_seed(1)).cuda(), (torch.rand(T, 8, generator=torch.Generator().manual_seed(2)) * 12 - 2).cuda()
    pl[1], po[1] = float("-inf"), float("nan")
    pl[3], po[3] = float("-inf"), float("nan")
    r = WindowRows(c, 8, rows, end, 40, 2, prev=(po, pl)).run()
    r.check(r._bound() + 8e-6 * 5)


# ---- trees ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,hkv,sizes", (
    (8, 2, (1, 4, 3, 2, 8)), (8, 2, (16, 0, 64, 33, 1)), (32, 8, (7, 8)), (32, 8, (64, 17, 0, 40)), (48, 8, (60, 10, 11)),
    (64, 8, (64, 3, 31)), (4, 4, (64, 1, 32, 33)), (17, 1, (30, 4)), (64, 1, (8, 1)), (6, 2, (5, 21, 22, 43))))
def test_tree_heads(fmt, hq, hkv, sizes):
    """One to 512 rows per KV head, blocks of rows that end inside a node's heads, requests without rows."""
    rng = np.random.default_rng(hq)
    end = [n + int(x) for n, x in zip(sizes, (130, 33, 0, 257, 7))]
    c = Cache(fmt, hkv, 32, end)
    c.fill_tokens(end, 5)
    TreeRows(c, hq, _trees(rng, sizes), end, extra=3, wide=2).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("page", (16, 64, 256))
def test_tree_lengths(fmt, page):
    """Trees that start and end at every place of a tile; rows whose word is empty, of all nodes, of nodes behind their own."""
    rng = np.random.default_rng(page)
    sizes = [1, 2, 31, 32, 33, 63, 64, 64, 5, 40, 64, 20]
    before = [0, 0, 1, 0, 31, 1, 0, 17, 33, 600, 32, 95]
    end = [n + x for n, x in zip(sizes, before)]
    words = _trees(rng, sizes)
    words[2][3] = 0                                     # sees the history alone
    words[3][0] = words[3][7] = 0                       # ... of which there is none: an empty row
    words[4][2] = (1 << 64) - 1
    words[6] = [int(x) for x in rng.integers(0, 1 << 63, 64)]
    words[9] = [1 << 63 | x for x in words[9]]          # a bit without a node
    c = Cache(fmt, 2, page, end)
    c.fill_tokens(end, 9)
    TreeRows(c, 8, words, end).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 7), (8, 64), (16, 33)))
def test_tree_long(fmt, hq, n):
    """A long request among short ones, split over every workgroup."""
    rng = np.random.default_rng(n)
    end = [9000 + n, 5, 0, 1200]
    c = Cache(fmt, 2, 16, end)
    c.fill_tokens(end, 31)
    TreeRows(c, hq, _trees(rng, (n, 1, 0, n)), end).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("B,hq,hkv,most", ((100, 8, 2, 3), (140, 16, 8, 16), (131, 8, 8, 30), (70, 8, 1, 64)))
def test_tree_requests_by_the_hundred(fmt, B, hq, hkv, most):
    rng = np.random.default_rng(B)
    sizes = rng.integers(0, most + 1, B)
    sizes[0] = most
    end = sizes + rng.integers(0, 70, B) * (rng.random(B) < 0.7)
    end[B // 2] += 1100
    c = Cache(fmt, hkv, 32, end)
    c.fill_tokens(end, 3)
    TreeRows(c, hq, _trees(rng, sizes), end).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("window,sinks", ((1, 0), (20, 4), (64, 40), (500, 0)))
@pytest.mark.parametrize("hq", (2, 16))
def test_tree_in_a_window(fmt, window, sinks, hq):
    rng = np.random.default_rng(window)
    sizes = [9, 64, 1, 30, 20]
    end = [n + x for n, x in zip(sizes, (700, 130, 0, 20, 64))]
    words = _trees(rng, sizes)
    words[1][5] = 0
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5)
    TreeRows(c, hq, words, end, window=window, sinks=sinks).run().check()


def test_tree_of_a_chain_equals_plain_attention():
    end, rows = [700, 33, 0, 64], [8, 1, 0, 4]
    c = Cache(oc.MXFP4, 2, 32, end)
    c.fill_tokens(end, 9)
    a = Rows(c, 8, rows, end).run().check()
    b = TreeRows(c, 8, [words_of(range(-1, n - 1)) for n in rows], end).run().check()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((4, 6), (8, 40), (8, 64)))
@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_tree_no_number_among_the_nodes(fmt, hq, n, value):
    """A NaN or infinity in a node's K or V reaches the rows that see it and no other."""
    rng = np.random.default_rng(n)
    for end0, node in ((n, 0), (33 + n, n - 1), (40 + n, n // 2), (64 + n, 2)):
        end, words = [end0, 50], _trees(rng, (n, 20))
        t = end0 - n + node
        for which in (0, 1):
            kv = [_normal(5, sum(end), 1, 128), _normal(6, sum(end), 1, 128)]
            kv[which][t, 0, 77] = value
            c = Cache(fmt, 1, 32, end)
            c.fill_tokens(end, 5, *kv)
            r = TreeRows(c, hq, words, end).run()
            torch.cuda.synchronize()
            want, _ = r.want()
            got = r.out.cpu().numpy()
            for i in range(n):
                if words[0][i] >> node & 1:
                    if which:
                        assert not np.isfinite(got[i, :, 77]).any()
                        assert np.isfinite(got[i, :, :64]).all() and np.isfinite(got[i, :, 96:]).all()
                    elif fmt != oc.BF16 or np.isnan(value):
                        assert np.isnan(got[i]).all()
                else:
                    assert np.abs(got[i] - want[i]).max() <= r._bound()
            assert np.abs(got[n:] - want[n:]).max() <= r._bound()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("fill", (0xFF, 0x7F, 0x80))
def test_tree_leftovers_in_pages(fmt, fill):
    rng = np.random.default_rng(fill)
    sizes = [1, 17, 45, 64]
    c = Cache(fmt, 2, 64, sizes, fill=fill)
    c.fill_tokens(sizes, 5)
    TreeRows(c, 8, _trees(rng, sizes), sizes).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
def test_tree_pages_that_are_none(fmt):
    """Nodes and history tokens of a page without a number, and behind the table, are not seen."""
    rng = np.random.default_rng(4)
    end = [200, 300, 100, 5000, -4, 270]
    have = [200, 256, 100, 256, 0, 256]
    c = Cache(fmt, 2, 16, have)
    c.fill_tokens(have, 5)
    c.table[0, 1], c.table[0, 11], c.table[1, 0], c.table[2, :] = -1, -1, c.num_pages, -7
    c.table[3, :-1] = 1 << 30
    c.dtable = _ints(c.table)
    TreeRows(c, 8, _trees(rng, (40, 64, 30, 20, 5, 33)), end).run().check()
    TreeRows(c, 8, _trees(rng, (40, 64, 30, 20, 5, 33)), end, window=90, sinks=20).run().check()


def test_tree_strange_row_starts():
    end = [40, 50, 60, 30]
    rng = np.random.default_rng(6)
    c = Cache(oc.MXFP8, 2, 32, end)
    c.fill_tokens(end, 5)
    words = _trees(rng, (20, 20, 20, 20))
    r = TreeRows(c, 8, words, end, extra=4, max_rows=20)
    r.dstart = _ints([0, 20, 41, 40, 60])            # 20, 21, -1 and 20 rows
    r.run()
    torch.cuda.synchronize()
    got = r.out.cpu().numpy()
    r2 = TreeRows(c, 8, words, end, extra=4, max_rows=20).run()
    torch.cuda.synchronize()
    assert np.array_equal(got[:20], r2.out[:20].cpu().numpy()) and (got[20:40] == 7).all() and (got[60:] == 7).all()
    r.dstart = _ints([-2, 18, 1 << 30, (1 << 30) + 20, (1 << 30) + 40])
    r.out.fill_(7.0)
    r.run()
    torch.cuda.synchronize()
    assert (r.out[18:] == 7).all()


def test_tree_joined_without_row_start_and_repeats():
    rng = np.random.default_rng(8)
    B, n = 5, 24
    end = [n + x for x in (300, 0, 64, 1000, 3)]
    c = Cache(oc.MXFP4, 2, 32, end)
    c.fill_tokens(end, 5)
    T = B * n
    po, pl = torch.randn(T, 16, 128, generator=torch.Generator().manual_seed(1)).cuda(), (torch.rand(T, 16, generator=torch.Generator().manual_seed(2)) * 12 - 2).cuda()
    pl[1], po[1] = float("-inf"), float("nan")
    words = _trees(rng, [n] * B)
    words[1][3] = 0
    pl[n + 3], po[n + 3] = float("-inf"), float("nan")       # nothing at all
    r = TreeRows(c, 16, words, end, prev=(po, pl)).run()
    r.check(r._bound() + 8e-6 * 5)
    first, fl = r.out.clone(), r.lse.clone()
    r.dstart = torch.empty(0)
    ss.ss_cache_attend_tree(r.desc, *c.at(), r.q.data_ptr(), T, r.dend.data_ptr(), r.tree.data_ptr(), r.out.data_ptr(), None, None,
                            0, 0, po.data_ptr(), pl.data_ptr(), r.ws.data_ptr(), r.ws.numel(), r.stride,
                            torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(first, r.out) and torch.equal(fl, r.lse)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 7), (8, 40), (16, 64)))
@pytest.mark.parametrize("factor", (2.0 ** 14, 2.0 ** -40, 0.0))
def test_tree_values_of_every_size(fmt, hq, n, factor):
    """Values far above and below the others, and zeros, in history tiles, in the tree's, in all tokens."""
    rng = np.random.default_rng(n)
    end = [400 + n, 70 + n, n]
    v = _normal(6, sum(end), 2, 128)
    v[100:133, 0] *= factor
    v[200, 1, 32:64] *= factor
    v[end[0] - 3:end[0], 1] *= factor
    v[end[0]:end[0] + end[1]] *= factor
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5, v=v)
    r = TreeRows(c, hq, _trees(rng, (n, n, n)), end).run()
    torch.cuda.synchronize()
    want, wl = r.want()
    got = r.out.cpu().numpy().astype(np.float64)
    # a value's error is relative to the largest |v| of its request, head and channel block: a weighted mean's weights are off by 5e-6 in the 2-norm
    for b in range(3):
        mine = slice(n * b, n * (b + 1))
        for h in range(2):
            g, x = got[mine, h * hq // 2:(h + 1) * hq // 2], want[mine, h * hq // 2:(h + 1) * hq // 2]
            assert np.linalg.norm(g - x) <= 5e-6 * np.linalg.norm(x)
    assert np.abs(r.lse.cpu().numpy() - wl).max() <= 5e-6 * max(1.0, np.abs(wl).max())


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 7), (8, 40), (16, 64)))
@pytest.mark.parametrize("where", ("history", "tree", "all"))
def test_tree_values_near_the_largest(fmt, hq, n, where):
    """Values of up to 2^114 in one block of 32 channels: each block is as near as if it were alone.

    The scores are normal numbers: exp of 500 of them adds up to less than 2^10, and the running maximum is above 2^-1. No
    sum that the formula needs passes 2^114 * 2^11, so any overflow is the kernel's own.
    """
    rng = np.random.default_rng(n)
    end = [400 + n, 70 + n]
    v = _normal(6, sum(end), 2, 128)
    which = {"history": slice(100, 133), "tree": slice(end[0] - 3, end[0]), "all": slice(0, sum(end))}[where]
    v[which, :, 32:64] *= 2.0 ** 112
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5, v=v)
    r = TreeRows(c, hq, _trees(rng, (n, n)), end).run()
    torch.cuda.synchronize()
    want, wl = r.want()
    got = r.out.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    for b in range(4):
        g, x = got[..., 32 * b:32 * b + 32], want[..., 32 * b:32 * b + 32]
        for mine in (slice(0, n), slice(n, 2 * n)):
            assert np.linalg.norm(g[mine] - x[mine]) <= 5e-6 * np.linalg.norm(x[mine])
    assert np.abs(r.lse.cpu().numpy() - wl).max() <= 5e-6 * max(1.0, np.abs(wl).max())


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 7), (8, 40), (16, 64)))
@pytest.mark.parametrize("gap", (18, 24, 27))
def test_tree_long_tail(fmt, hq, n, gap):
    """A first token that outweighs each other by e^gap, whose values the others' are 256 times: with gap 24 each of 6000 tokens
    weighs 2^-34.6 and all their values make 6e-5 of the result, which the sum of what is small must not lose."""
    rng = np.random.default_rng(n)
    end = [6000 + n]
    q = torch.full((n, hq, 128), 1.0).to(torch.bfloat16) + 0.25 * _normal(4, n, hq, 128).cpu()
    k = 0.25 * _normal(5, sum(end), 2, 128)
    k[0] = gap / 128 ** 0.5
    v = 256 * (1 + 0.25 * _normal(6, sum(end), 2, 128).float()).to(torch.bfloat16)
    v[0] = 1.0
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5, k, v)
    TreeRows(c, hq, _trees(rng, (n,)), end, q=q.cuda().to(torch.bfloat16).contiguous()).run().check()


@pytest.mark.parametrize("hq,n", ((4, 7), (8, 40), (8, 64)))
def test_tree_codes_that_are_no_numbers(hq, n):
    """An e4m3 code that is none, under an ordinary scale, in a node's V: rows that do not see it stay as they are."""
    rng = np.random.default_rng(n)
    end, words = [64 + n], _trees(rng, (n,))
    node = n // 2
    t = 64 + node
    c = Cache(oc.MXFP8, 1, 32, end)
    c.fill_tokens(end, 5)
    oc.parts(c.pages, oc.MXFP8, 32)[1][c.table[0, t // 32], 0, t % 32, 77] = 0x7F
    c.dev.copy_(torch.from_numpy(c.pages))
    r = TreeRows(c, hq, words, end).run()
    torch.cuda.synchronize()
    want, _ = r.want()
    got = r.out.cpu().numpy()
    for i in range(n):
        if words[0][i] >> node & 1:
            assert np.isnan(got[i, :, 77]).all() and np.isnan(want[i, :, 77]).all()
            got[i, :, 77] = want[i, :, 77] = 0
    assert np.abs(got - want).max() <= r._bound()


# ---- appending -----------------------------------------------------------------------------------
def _freq(half, base=10000.0):
    return (base ** (-torch.arange(half, dtype=torch.float64) / max(1, half))).float()


def _append(c, hq, rows, end, rotary, interleaved, positions=None, scale=1.0, seed=7, in_place=False, extra=0, row_start=True):
    start = np.cumsum([0] + list(rows))
    T = int(start[-1]) + extra
    fused = _normal(seed, T, hq + 2 * c.hkv, 128)
    q, k, v = fused[:, :hq], fused[:, hq:hq + c.hkv], fused[:, hq + c.hkv:]
    before = [_bits(x) for x in (q, k, v)]
    freq = _freq(rotary // 2).cuda()
    out = q if in_place else torch.full((T, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rope = ss.make_rope_desc(rotary, freq.data_ptr(), interleaved, scale)
    at = None if positions is None else _ints(positions)
    dstart, dend = _ints(start) if row_start else None, _ints(end)
    ss.ss_cache_append(c.desc(num_q_heads=hq, max_rows=max(rows)), *c.at(), rope, k.data_ptr(), v.data_ptr(), T, dend.data_ptr(),
                       None if dstart is None else dstart.data_ptr(), fused.stride(0), None if at is None else at.data_ptr(),
                       q.data_ptr(), out.data_ptr(), fused.stride(0), fused.stride(0) if in_place else 0,
                       torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    own = np.concatenate([np.arange(e - n, e) for n, e in zip(rows, end)])
    pos = own if positions is None else positions[:len(own)]
    return before, out, start, pos, freq.cpu().numpy()


def _close(got_bits, want, rotary, interleaved):
    """Between the roundings of what is 2^-34 of the pair's length off either way; channels that do not turn are equal."""
    def rounded(x):
        bits = x.astype(np.float32).view(np.uint32)
        return bf16_bits_to_f64(((bits + 0x7fff + (bits >> 16 & 1)) >> 16).astype(np.uint16))
    got = bf16_bits_to_f64(got_bits)
    half = rotary // 2
    a, b = (np.arange(0, rotary, 2), np.arange(1, rotary, 2)) if interleaved else (np.arange(half), np.arange(half, rotary))
    length = np.zeros(want.shape)
    length[..., a] = length[..., b] = np.hypot(want[..., a], want[..., b])
    off = 2.0 ** -34 * length + 2.0 ** -134
    assert (rounded(want - off) <= got).all() and (got <= rounded(want + off)).all()
    assert np.array_equal(got[..., rotary:], want[..., rotary:])


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("rotary,interleaved", ((128, 0), (128, 1), (64, 0), (64, 1), (16, 0), (16, 1), (96, 0), (112, 1)))
@pytest.mark.parametrize("hq,hkv,rows,before", ((8, 2, (1, 1, 1, 1, 1), (15, 16, 17, 0, 400)), (9, 3, (5, 0, 33, 1), (30, 7, 0, 63)),
                                                (16, 16, (700, 350, 3), (0, 5, 100))))
def test_append(fmt, rotary, interleaved, hq, hkv, rows, before):
    end = [n + x for n, x in zip(rows, before)]
    c = Cache(fmt, hkv, 32, end)
    (q, k, v), out, start, pos, freq = _append(c, hq, rows, end, rotary, interleaved)
    some = np.arange(0, len(q), max(1, len(q) // 40))             # rows that the oracle turns one by one
    _close(_bits(out)[some], ot.turned(q[some], pos[some], freq, interleaved), rotary, interleaved)
    # K: what the pages hold is within its rounding of the turned rows; V and every other byte exactly what a write gives
    places = oc.row_places(start, end, c.table, 32, c.num_pages)
    K, V, KS, VS = oc.parts(c.dev.cpu().numpy(), fmt, 32)
    at, slot = np.array([p[1] for p in places]), np.array([p[2] for p in places])
    got = oc.decode(K[at, :, slot], KS[at, :, slot], fmt)
    turned = ot.turned(k[some], pos[some], freq, interleaved)
    if fmt == oc.BF16:
        _close(np.ascontiguousarray(K[at, :, slot]).view(np.uint16)[some], turned, rotary, interleaved)
    else:
        peak = np.abs(turned.reshape(len(some), hkv, 4, 32)).max(-1).repeat(32, -1)
        # half a step of the largest code, of a bf16 value: e4m3's top step is 32 of 448, e2m1's 2 of 6, twice that of the
        # peak where the exponent has just risen
        step = 32 / 448 if fmt == oc.MXFP8 else 2 / 6
        assert (np.abs(got[some] - turned) <= peak * (step + 2.0 ** -8)).all()
    # the same rows, turned by the call as queries, written plainly: the same bytes
    if hq == hkv:
        c2 = Cache(fmt, hkv, 32, end)
        fused = torch.empty(len(k), 3 * hkv, 128, dtype=torch.bfloat16, device="cuda")
        fused[:, :hkv] = torch.from_numpy(k.view(np.int16)).cuda().view(torch.bfloat16)
        fused[:, hkv:2 * hkv] = 0
        f, d, e = torch.from_numpy(freq).cuda(), _ints(start), _ints(end)
        rope = ss.make_rope_desc(rotary, f.data_ptr(), interleaved)
        s = torch.cuda.current_stream().cuda_stream
        kt = torch.empty(len(k), hkv, 128, dtype=torch.bfloat16, device="cuda")
        ss.ss_cache_append(c2.desc(num_q_heads=hkv, max_rows=max(rows)), *c2.at(), rope, fused[:, hkv:].data_ptr(), fused[:, hkv:].data_ptr(),
                           len(k), e.data_ptr(), d.data_ptr(), fused.stride(0), None, fused.data_ptr(), kt.data_ptr(), fused.stride(0), 0, s)
        torch.cuda.synchronize()
        c3 = Cache(fmt, hkv, 32, end)
        want = oc.write(c3.pages, fmt, 32, c3.table, _bits(kt), v, start, end)
        assert np.array_equal(c.dev.cpu().numpy(), want)


@pytest.mark.parametrize("interleaved", (0, 1))
def test_append_far_positions(interleaved):
    """Positions up to 2^31 - 1, negative ones, zero, siblings at one position; a scale."""
    rows = (40, 24)
    end = [100, 24]
    positions = np.array([0, 1, -1, 2147483647, -2147483648, 1 << 30, 1000003, 131071] + [777] * 24 + list(range(1 << 20, (1 << 20) + 32)), np.int64)
    c = Cache(oc.BF16, 2, 32, end)
    (q, k, v), out, start, pos, freq = _append(c, 8, rows, end, 128, interleaved, positions=positions, scale=1.25)
    _close(_bits(out), ot.turned(q, pos, freq, interleaved, 1.25), 128, interleaved)


def test_append_places_rows_and_leaves_the_rest():
    """Tokens without a place are not written but their q turns; q_out's rows of no request stay; in place; without
    row_start; other bytes of the pages stay."""
    rows, end = (6, 30, 40, 10), (3, 40, 40, 53)
    c = Cache(oc.MXFP8, 2, 16, [40, 40, 40, 40], width=3)
    c.table[1, 1], c.table[2, 0] = -1, c.num_pages
    c.dtable = _ints(c.table)
    (q, k, v), out, start, pos, freq = _append(c, 4, rows, end, 128, 0, extra=5)
    n = int(start[-1])
    _close(_bits(out)[:n], ot.turned(q[:n], pos, freq), 128, 0)
    assert (out[n:] == 7).all()
    got = c.dev.cpu().numpy()
    same = oc.write(c.pages, oc.MXFP8, 16, c.table, k[:n], v[:n], start, end)
    parts, mine = oc.parts(got, oc.MXFP8, 16), oc.parts(same, oc.MXFP8, 16)
    assert np.array_equal(parts[1], mine[1]) and np.array_equal(parts[3], mine[3])         # V as a write leaves it
    untouched = (mine[1] == 0xA5).all(-1).all(1)                                           # [page, slot] that no row owns
    assert (parts[0].transpose(0, 2, 1, 3)[untouched] == 0xA5).all()
    # the same call, q turned in place
    c2 = Cache(oc.MXFP8, 2, 16, [40, 40, 40, 40], width=3)
    c2.dtable = _ints(c.table)
    _, out2, _, _, _ = _append(c2, 4, rows, end, 128, 0, extra=5, in_place=True)
    assert torch.equal(out2[:n], out[:n]) and np.array_equal(c2.dev.cpu().numpy(), got)
    assert np.array_equal(_bits(out2[n:]), q[n:])
    # without row_start
    c3, c4 = Cache(oc.BF16, 3, 32, [70, 70, 70]), Cache(oc.BF16, 3, 32, [70, 70, 70])
    a = _append(c3, 6, (64, 64, 64), [64, 66, 70], 64, 1)[1]
    b = _append(c4, 6, (64, 64, 64), [64, 66, 70], 64, 1, row_start=False)[1]
    assert torch.equal(a, b) and torch.equal(c3.dev, c4.dev)


def test_append_keys_alone_and_no_numbers():
    """Without q; infinities and NaNs turn into NaNs of their pair, and a scaled block of theirs reads NaN."""
    c = Cache(oc.MXFP8, 2, 16, [20])
    k, v = _normal(1, 20, 2, 128), _normal(2, 20, 2, 128)
    k[3, 0, 5], k[4, 1, 100] = float("inf"), float("nan")
    f, e, d = _freq(64).cuda(), _ints([20]), _ints([0, 20])
    ss.ss_cache_append(c.desc(max_rows=20), *c.at(), ss.make_rope_desc(128, f.data_ptr()), k.data_ptr(), v.data_ptr(), 20, e.data_ptr(),
                       d.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    K, V, KS, VS = oc.parts(c.dev.cpu().numpy(), oc.MXFP8, 16)
    got = np.concatenate([oc.decode(K[c.table[0, t // 16], :, t % 16], KS[c.table[0, t // 16], :, t % 16], oc.MXFP8)[None] for t in range(20)])
    bad = np.isnan(got)
    want = np.zeros_like(bad)
    want[3, 0, :32] = want[3, 0, 64:96] = True            # channels 5 and 69
    want[4, 1, 32:64] = want[4, 1, 96:] = True            # channels 36 and 100
    assert np.array_equal(bad, want)


# ---- keeping -------------------------------------------------------------------------------------
def _keep(c, paths, rows, end, row_start=True, max_rows=None, counts=None, extra=0):
    start = np.cumsum([0] + list(rows))
    listed = []
    for path, n in zip(paths, rows):
        listed += list(path) + [9999] * (n - len(path))
    kept, num = _ints(listed + [5] * extra), _ints([len(p) for p in paths] if counts is None else counts)
    d, e = _ints(start), _ints(end)
    ss.ss_cache_keep(c.desc(max_rows=max(rows) if max_rows is None else max_rows), *c.at(), kept.data_ptr(), num.data_ptr(), len(listed) + extra,
                     e.data_ptr(), d.data_ptr() if row_start else None, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return start


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("page,hkv", ((16, 1), (32, 8), (256, 3)))
def test_keep(fmt, page, hkv):
    """Paths of random trees, orders turned round, one node several times, nothing kept, everything kept."""
    rng = np.random.default_rng(page)
    rows = [1, 5, 64, 64, 33, 20, 8, 0, 64]
    end = [n + x for n, x in zip(rows, (0, 14, 100, 1, 31, 250, 16, 5, 77))]
    parents = [random_parents(rng, n) for n in rows]
    paths = [path_to(p, int(rng.integers(0, n))) if n else [] for p, n in zip(parents, rows)]
    paths[3] = list(range(64))[::-1]
    paths[5] = [7] * 20
    paths[6] = []
    paths[8] = [int(x) for x in rng.permutation(64)[:40]]
    c = Cache(fmt, hkv, page, end)
    c.fill_tokens(end, 3)
    start = _keep(c, paths, rows, end)
    assert np.array_equal(c.dev.cpu().numpy(), ot.keep(c.pages, fmt, page, c.table, paths, start, end))


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
def test_keep_what_has_no_place(fmt):
    """Indices and counts out of range, tokens before the first and behind the table, pages that are none, requests of
    too many rows, rows outside the call's."""
    rows, end = [6, 8, 10, 9, 7], [4, 30, 52, 20, 40]
    paths = [[5, 3, 2, 4, 1, 0], [-1, 7, 8, 1 << 30, 3, -5], [9, 8, 7, 6, 5], [3, 2, 1], [6, 5]]
    c = Cache(fmt, 2, 16, [48] * 5, width=3)
    c.fill_tokens([48] * 5, 3)
    c.table[3, 0], c.table[4, 2] = -1, c.num_pages
    c.dtable = _ints(c.table)
    start = _keep(c, paths, rows, end, counts=[6, 8, 5, 3, 2])
    assert np.array_equal(c.dev.cpu().numpy(), ot.keep(c.pages, fmt, 16, c.table, paths, start, end))
    c.dev.copy_(torch.from_numpy(c.pages))
    _keep(c, paths, rows, end, counts=[-1, 0, -(1 << 31), 0, 0], extra=3)
    assert np.array_equal(c.dev.cpu().numpy(), c.pages)
    _keep(c, paths, rows, end, max_rows=5)                          # more rows than max_rows: left alone
    assert np.array_equal(c.dev.cpu().numpy(), c.pages)


def test_keep_without_row_start():
    c, c2 = Cache(oc.MXFP8, 2, 32, [70, 90]), Cache(oc.MXFP8, 2, 32, [70, 90])
    c.fill_tokens([70, 90], 3)
    c2.dev.copy_(c.dev)
    paths = [[3, 2, 15], [8, 1]]
    _keep(c, paths, [16, 16], [70, 90])
    _keep(c2, paths, [16, 16], [70, 90], row_start=False)
    assert torch.equal(c.dev, c2.dev)


# ---- together ------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
def test_tree_serving_loop(fmt):
    """Prompts enter turned, then steps of drafted trees: appended, attended, the accepted path kept; a windowed layer's
    attention beside them.  What the cache holds in the end is the accepted text alone."""
    B, hq, hkv, page = 3, 8, 2, 16
    rng = np.random.default_rng(8)
    p = H.PagedCache(B, hq, hkv, 600, fmt, page, max_rows=2, tree_rows=20)
    freq = _freq(64).cuda()
    s = torch.cuda.current_stream().cuda_stream
    text = [[] for _ in range(B)]             # codes of every token's K and V, as the pages held them when they were written

    def enter(rows, seed, positions=None):
        p.grow(rows)
        T = sum(rows)
        fused = _normal(seed, T, hq + 2 * hkv, 128)
        start = _ints(np.cumsum([0] + list(rows)))
        q = torch.empty(T, hq, 128, dtype=torch.bfloat16, device="cuda")
        p.append(fused[:, hq:hq + hkv], fused[:, hq + hkv:], freq, s, start, positions, fused[:, :hq], q)
        return q, start

    def held(b, upto):
        pages, table = p.pages.cpu().numpy(), p.table.cpu().numpy()
        P = oc.parts(pages, fmt, page)
        t = np.arange(upto)
        return [x[table[b][t // page], :, t % page] for x in P]

    rows = [100, 33, 1]
    enter(rows, 1)
    for b in range(B):
        text[b] = [[x[t] for x in held(b, rows[b])] for t in range(rows[b])]
    for step in range(5):
        rows = [int(x) for x in rng.integers(1, 21, B)]
        parents = [random_parents(rng, n) for n in rows]
        positions = _ints([p.tokens[b] + d for b in range(B) for d in depths_of(parents[b])])
        q, start = enter(rows, 10 + step, positions)
        words = [words_of(x) for x in parents]
        tree = torch.from_numpy(as_int64([w for ws in words for w in ws])).cuda()
        T = sum(rows)
        out, lse = torch.empty(T, hq, 128, device="cuda"), torch.empty(T, hq, device="cuda")
        window, sinks = ((0, 0), (30, 2))[step % 2]
        p.attend_tree(q, tree, out, lse, s, start, window=window, sinks=sinks)
        torch.cuda.synchronize()
        pages, table = p.pages.cpu().numpy(), p.table.cpu().numpy()
        flat = [w for ws in words for w in ws]
        want, wl = ot.attend(_bits(q), pages, fmt, page, table, start.cpu().numpy(), p.tokens, 128 ** -0.5,
                             lambda row, i, n, end: ot.tree_sees(flat[row], i, n, end, window, sinks))
        assert np.linalg.norm(out.cpu().numpy() - want) <= 5e-6 * np.linalg.norm(want)
        assert np.abs(lse.cpu().numpy() - wl).max() <= 5e-6 * max(1.0, np.abs(wl).max())
        paths = [path_to(x, int(rng.integers(0, n))) for x, n in zip(parents, rows)]
        paths[step % B] = []
        for b in range(B):
            now = held(b, p.tokens[b])
            first = p.tokens[b] - rows[b]
            text[b] += [[x[first + i] for x in now] for i in paths[b]]
        p.keep(paths, rows)
        torch.cuda.synchronize()
        assert p.end.tolist() == p.tokens == [len(x) for x in text]
        for b in range(B):
            now = held(b, p.tokens[b])
            for t, token in enumerate(text[b]):
                assert all(np.array_equal(x[t], y) for x, y in zip(now, token))
        # the next token of a windowed layer
        q1, start1 = enter([1] * B, 50 + step)
        out1, lse1 = torch.empty(B, hq, 128, device="cuda"), torch.empty(B, hq, device="cuda")
        p.attend(q1, out1, lse1, s, start1, window=25, sinks=3)
        torch.cuda.synchronize()
        pages, table = p.pages.cpu().numpy(), p.table.cpu().numpy()
        want, _ = ot.attend(_bits(q1), pages, fmt, page, table, np.arange(B + 1), p.tokens, 128 ** -0.5,
                            lambda row, i, n, end: ot.window_sees(i, n, end, 25, 3))
        assert np.linalg.norm(out1.cpu().numpy() - want) <= 5e-6 * np.linalg.norm(want)
        p.release([1] * B)


def test_tree_step_in_a_graph():
    """A captured step (append, tree attention, keep) follows tables, ends, rows and trees from replay to replay; two
    graphs share a workspace."""
    B, hq, hkv, page, n = 4, 16, 2, 16, 12
    c = Cache(oc.MXFP8, hkv, page, [500] * B)
    ends = [3, 100, 16, 250]
    c.fill_tokens(ends, 5)
    rng = np.random.default_rng(2)
    fused = torch.empty(B * n, hq + 2 * hkv, 128, dtype=torch.bfloat16, device="cuda")
    qt = torch.empty(B * n, hq, 128, dtype=torch.bfloat16, device="cuda")
    end, start = _ints([e + n for e in ends]), _ints(np.arange(B + 1) * n)
    positions, kept, num = _ints(np.zeros(B * n)), _ints(np.zeros(B * n)), _ints(np.zeros(B))
    tree = torch.zeros(B * n, dtype=torch.int64, device="cuda")
    freq = _freq(64).cuda()
    rope = ss.make_rope_desc(128, freq.data_ptr())
    d = c.desc(num_q_heads=hq, max_rows=n)
    ws = torch.empty(ss.ss_cache_attend_tree_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(B * n, hq, 128, device="cuda"), torch.empty(B * n, hq, device="cuda")

    def step(s):
        ss.ss_cache_append(d, *c.at(), rope, fused[:, hq:].data_ptr(), fused[:, hq + hkv:].data_ptr(), B * n, end.data_ptr(), start.data_ptr(),
                           fused.stride(0), positions.data_ptr(), fused.data_ptr(), qt.data_ptr(), fused.stride(0), 0, s)
        ss.ss_cache_attend_tree(d, *c.at(), qt.data_ptr(), B * n, end.data_ptr(), tree.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                start.data_ptr(), 0, 0, None, None, ws.data_ptr(), ws.numel(), 0, s)
        ss.ss_cache_keep(d, *c.at(), kept.data_ptr(), num.data_ptr(), B * n, end.data_ptr(), start.data_ptr(), s)

    graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    for graph in graphs:
        with torch.cuda.graph(graph):
            step(torch.cuda.current_stream().cuda_stream)
    for i in range(6):
        rows = [int(x) for x in rng.integers(0, n + 1, B)]
        rows[i % B] = n
        parents = [random_parents(rng, m) if m else [] for m in rows]
        flat = [w for x in parents for w in words_of(x)]
        fill = B * n - len(flat)
        fused.copy_(_normal(50 + i, B * n, hq + 2 * hkv, 128))
        tree.copy_(torch.from_numpy(as_int64(flat + [0] * fill)))
        start.copy_(_ints(np.cumsum([0] + rows)))
        end.copy_(_ints([e + m for e, m in zip(ends, rows)]))
        positions.copy_(_ints([e + x for e, par in zip(ends, parents) for x in depths_of(par)] + [0] * fill))
        paths = [path_to(x, len(x) - 1) for x in parents]
        kept.copy_(_ints([y for x, m in zip(paths, rows) for y in x + [0] * (m - len(x))] + [0] * fill))
        num.copy_(_ints([len(x) for x in paths]))
        for t in (qt, out, lse):
            t.fill_(7.0)
        torch.cuda.synchronize()
        before = c.dev.clone()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (c.dev, qt, out, lse)]
        c.dev.copy_(before)
        for t in (qt, out, lse):
            t.fill_(7.0)
        ws.fill_(255)
        step(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (c.dev, qt, out, lse)))
        ends = [e + len(x) for e, x in zip(ends, paths)]


def test_window_in_a_graph():
    """A captured call goes on with other lengths: parts without tiles, of requests that grow past the window."""
    end = [2500, 700, 3, 0]
    rows = [4, 2, 3, 1]
    c = Cache(oc.MXFP8, 2, 32, end, width=96)
    c.fill_tokens(end, 5)
    r = WindowRows(c, 32, rows, end, 600, 30)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.run(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.run()
    for shorter in ([0, 0, 0, 0], [2490, 699, 3, 0], [1, 640, 0, 0], [400, 0, 2, 0]):
        r.end = [e - s for e, s in zip(end, shorter)]
        r.dend.copy_(_ints(r.end))
        r.out.fill_(7.0)
        r.lse.fill_(7.0)
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        out, lse = r.out.clone(), r.lse.clone()
        r.check()
        r.run()
        torch.cuda.synchronize()
        assert torch.equal(out, r.out) and torch.equal(lse, r.lse)


def test_tree_pages_beyond_32_bits_on_another_stream():
    """Pages more than 2^32 bytes into the cache, interleaved with other layers' by page_stride; a side stream."""
    hkv, page, fmt = 1, 16, oc.BF16
    own = oc.page_bytes(fmt, hkv, page)
    stride, num_pages = 1 << 20, 4600
    pool = torch.zeros(num_pages * stride, dtype=torch.uint8, device="cuda")
    sizes, before = [20, 64], [30, 50]
    end = [a + b for a, b in zip(sizes, before)]
    ids = [4599, 4598, 1, 4200, 4300, 4400, 4500, 0, 4597, 4100, 4000, 3900]
    table = np.full((2, 8), -1, np.int32)
    table[0, :4], table[1] = ids[:4], ids[4:]
    small = Cache(fmt, hkv, page, [64, 128], spare=0)
    small.fill_tokens([64, 128], 5)
    for b in range(2):
        for j in range(8):
            if table[b, j] >= 0:
                at = int(table[b, j]) * stride
                pool[at:at + own] = small.dev[small.table[b, j]].flatten()
    rng = np.random.default_rng(1)
    r = TreeRows(small, 4, _trees(rng, sizes), end).run().check()
    d = ss.make_cache_desc(2, hkv, fmt, page, num_pages, 8, num_q_heads=4, page_stride=stride, max_rows=64)
    ws = torch.empty(ss.ss_cache_attend_tree_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    out, lse, dt = torch.full_like(r.out, 7.0), torch.full_like(r.lse, 7.0), _ints(table)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ss.ss_cache_attend_tree(d, pool.data_ptr(), dt.data_ptr(), r.q.data_ptr(), r.T, r.dend.data_ptr(), r.tree.data_ptr(), out.data_ptr(),
                            lse.data_ptr(), r.dstart.data_ptr(), 0, 0, None, None, ws.data_ptr(), ws.numel(), r.stride, side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(out, r.out) and torch.equal(lse, r.lse)
    # a path kept there
    kept, num = _ints([5, 3] + [0] * 18 + [63, 62, 0] + [0] * 61), _ints([2, 3])
    ss.ss_cache_keep(d, pool.data_ptr(), dt.data_ptr(), kept.data_ptr(), num.data_ptr(), 84, r.dend.data_ptr(), r.dstart.data_ptr(), side.cuda_stream)
    torch.cuda.synchronize()
    want = ot.keep(small.pages, fmt, page, small.table, [[5, 3], [63, 62, 0]], r.start, end)
    for b in range(2):
        for j in range(8):
            if table[b, j] >= 0:
                at = int(table[b, j]) * stride
                assert np.array_equal(pool[at:at + own].cpu().numpy(), want[small.table[b, j]].ravel())
