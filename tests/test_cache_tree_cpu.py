"""Rotated appends, trees, windows and kept paths without a GPU: workspaces, refusals, the oracle's pins, and
PagedCache's bookkeeping.  Every call here is refused before it looks at a device, or does not reach the library."""
from __future__ import annotations

from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from oracle import bf16_bits_to_f64
from oracle import cache as oc
from oracle import tree as ot
from paper_2609_33184_amd import harness as H
from paper_2609_33184_amd import specstream as ss
from test_cache_cpu import BAD, END, K, PAGES, ROWS, TABLE, V, WS, _desc, _refused, lib  # noqa: F401
from tree_inputs import depths_of, path_to, random_parents, words_of

FREQ, TREE = 0x7F0010000000, 0x7F0011000000
INVALID, UNSUPPORTED = ss.SS_ERR_INVALID_ARGUMENT, ss.SS_ERR_UNSUPPORTED


def _append(d, pages=PAGES, table=TABLE, k=K, v=V, num_rows=8, end=END, rotary=128, freq=FREQ, interleaved=0, scale=1.0, **kw):
    ss.ss_cache_append(d, pages, table, ss.make_rope_desc(rotary, freq, interleaved, scale), k, v, num_rows, end, **kw)


def _tree(d, pages=PAGES, table=TABLE, q=K, num_rows=8, end=END, tree=TREE, out=V, workspace=WS, workspace_bytes=1 << 32, **kw):
    ss.ss_cache_attend_tree(d, pages, table, q, num_rows, end, tree, out, workspace=workspace, workspace_bytes=workspace_bytes, **kw)


def _window(d, pages=PAGES, table=TABLE, q=K, num_rows=8, end=END, out=V, window=4, sinks=0, workspace=WS, workspace_bytes=1 << 32, **kw):
    ss.ss_cache_attend_window(d, pages, table, q, num_rows, end, out, window, sinks, workspace=workspace, workspace_bytes=workspace_bytes, **kw)


def _keep(d, pages=PAGES, table=TABLE, kept=K, num_kept=V, num_rows=8, end=END, **kw):
    ss.ss_cache_keep(d, pages, table, kept, num_kept, num_rows, end, **kw)


CALLS = (_append, _tree, _window, _keep)


@pytest.mark.parametrize("kw,word,status", BAD, ids=lambda x: str(x)[:40])
def test_descriptors_that_every_call_refuses(kw, word, status):
    d = _desc(**kw)
    assert ss.ss_cache_attend_tree_workspace_bytes(d) == 0 and word in ss.ss_last_error()
    for call in CALLS:
        _refused(status, word, call, d)


@pytest.mark.parametrize("call", CALLS)
def test_shared_arguments(call):
    for kw in (dict(pages=0), dict(pages=PAGES + 8), dict(table=0), dict(table=TABLE + 2), dict(end=0), dict(end=END + 1),
               dict(row_start=ROWS + 2, num_rows=3), dict(num_rows=0), dict(num_rows=-1), dict(num_rows=7)):
        _refused(INVALID, "", call, _desc(), **kw)


ATTEND = [(dict(num_q_heads=0), "num_q_heads", INVALID), (dict(num_q_heads=9), "num_q_heads", INVALID),
          (dict(softmax_scale=0.0), "softmax_scale", INVALID), (dict(softmax_scale=3e38), "softmax_scale", INVALID), (dict(causal=2), "causal", INVALID)]


@pytest.mark.parametrize("kw,word,status", ATTEND + [
    (dict(max_rows=65), "max_rows", INVALID), (dict(max_rows=64, num_q_heads=18), "rows per KV head", UNSUPPORTED),
    (dict(max_rows=1, num_q_heads=130), "query heads per KV head", UNSUPPORTED),
    (dict(max_rows=64, num_kv_heads=512, num_q_heads=1024, num_requests=1), "max_rows x num_q_heads", UNSUPPORTED),
    (dict(max_rows=64, num_requests=256, table_stride=1 << 21, num_q_heads=16), "blocks of rows", UNSUPPORTED)], ids=lambda x: str(x)[:40])
def test_descriptors_that_a_tree_refuses(kw, word, status):
    d = _desc(**kw)
    assert ss.ss_cache_attend_tree_workspace_bytes(d) == 0 and word in ss.ss_last_error()
    _refused(status, word, _tree, d)


@pytest.mark.parametrize("kw,word,status", ATTEND + [(dict(max_rows=9), "max_rows", INVALID), (dict(causal=0), "causal", INVALID),
                                                     (dict(max_rows=8, num_q_heads=18), "rows per KV head", UNSUPPORTED)], ids=lambda x: str(x)[:40])
def test_descriptors_that_a_window_refuses(kw, word, status):
    _refused(status, word, _window, _desc(**kw))


def test_workspaces():
    """Whatever the length; 512 rows per KV head are attended in blocks of 64 and need no more than 64 do."""
    for rows, hq in ((1, 2), (8, 8), (16, 8), (64, 16)):
        n = ss.ss_cache_attend_tree_workspace_bytes(_desc(max_rows=rows, num_q_heads=hq, causal=0))
        assert n > 0 and n % 256 == 0
    assert ss.ss_cache_attend_tree_workspace_bytes(_desc(max_rows=8)) == ss.ss_cache_attend_workspace_bytes(_desc(max_rows=8))
    assert ss.load().ss_cache_attend_tree_workspace_bytes(None) == 0


@pytest.mark.parametrize("call", (_tree, _window))
def test_attention_arguments(call):
    d = _desc()
    for kw in (dict(q=0), dict(q=K + 8), dict(out=0), dict(out=V + 4), dict(lse=V + 2), dict(q_row_stride=1016), dict(q_row_stride=1028),
               dict(prev_out=V), dict(prev_lse=V), dict(prev_out=V + 8, prev_lse=V), dict(prev_out=V, prev_lse=V + 1),
               dict(window=-1), dict(sinks=-1, window=4)):
        _refused(INVALID, "", call, d, **kw)
    need = ss.ss_cache_attend_tree_workspace_bytes(d)
    for kw in (dict(workspace=0), dict(workspace=WS + 64), dict(workspace_bytes=need - 1)):
        _refused(ss.SS_ERR_WORKSPACE, "workspace", call, d, **kw)
    _refused(INVALID, "window", _window, d, window=0)
    for tree in (0, TREE + 4):
        _refused(INVALID, "tree", _tree, d, tree=tree)


def test_append_arguments():
    d = _desc()
    for kw in (dict(k=0), dict(v=0), dict(k=K + 8), dict(v=V + 2)):
        _refused(INVALID, "k and v", _append, d, **kw)
    for stride in (-256, 248, 260):
        _refused(INVALID, "row_stride", _append, d, row_stride=stride)
    for rotary in (0, -16, 129, 144):
        _refused(INVALID, "rotary_dim", _append, d, rotary=rotary)
    for rotary in (2, 8, 100, 120):
        _refused(UNSUPPORTED, "rotary_dim", _append, d, rotary=rotary)
    for kw in (dict(interleaved=2), dict(interleaved=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(freq=0), dict(freq=FREQ + 2), dict(positions=ROWS + 1), dict(q=K), dict(q_out=K), dict(q=K + 8, q_out=V), dict(q=K, q_out=V + 8),
               dict(q=K, q_out=V, q_row_stride=1016), dict(q=K, q_out=V, q_out_row_stride=1028), dict(q=K, q_out=K, q_row_stride=2048)):
        _refused(INVALID, "", _append, d, **kw)
    for heads, status in ((0, INVALID), (9, INVALID), (131072, UNSUPPORTED)):
        _refused(status, "num_q_heads", _append, _desc(num_q_heads=heads), q=K, q_out=V)
    _refused(UNSUPPORTED, "num_rows", _append, d, num_rows=1 << 28, row_start=ROWS)
    assert ss.load().ss_cache_append(d, PAGES, TABLE, None, None, K, V, 0, None, 0, None, 0, 8, None, END, None) == INVALID


def test_keep_arguments():
    for kw in (dict(kept=0), dict(num_kept=0), dict(kept=K + 2), dict(num_kept=V + 1)):
        _refused(INVALID, "kept", _keep, _desc(), **kw)
    _refused(INVALID, "max_rows", _keep, _desc(max_rows=65), num_rows=260)


# ---- the oracle -----------------------------------------------------------------------------------
def test_bf16_rounding():
    x = np.array([1.0, 1.00390625, 1.01171875, 1.0039062500001, -1.00390625, 2.0 ** -130, 3e38, 0.0, 2.0 ** -133 * 2.5])
    want = [1.0, 1.0, 1.015625, 1.0078125, -1.0, 2.0 ** -130, 3.0040553e38, 0.0, 2.0 ** -133 * 2]
    assert np.allclose(bf16_bits_to_f64(ot.bf16_bits(x)), want, rtol=1e-6, atol=0)
    r = np.random.default_rng(1).standard_normal(4000) * np.exp2(np.random.default_rng(2).integers(-30, 30, 4000))
    want = torch.from_numpy(r.astype(np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(ot.bf16_bits(r.astype(np.float32).astype(np.float64)), want)


@pytest.mark.parametrize("interleaved", (False, True))
def test_turning_by_multiples_keeps_what_it_must(interleaved):
    """Lengths of pairs stay, turning adds positions, dot products depend on the difference alone, and a quarter turn
    is (x1, x2) -> (-x2, x1)."""
    rng = np.random.default_rng(4)
    bits = ot.bf16_bits(rng.standard_normal((6, 2, 128)))
    x = bf16_bits_to_f64(bits)
    f = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    y = ot.turned(bits, [0, 1, 5, -3, 1000, 77], f, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 64:], x[..., 64:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-13)
    a = np.stack([bits[0], bits[1]])
    d1, d2 = ot.turned(a, [9, 4], f, interleaved), ot.turned(a, [105, 100], f, interleaved)
    assert np.allclose((d1[0] * d1[1]).sum(-1), (d2[0] * d2[1]).sum(-1), rtol=1e-12)
    q = ot.turned(bits[:1], [1], np.array([np.pi / 2], np.float32), interleaved, scale=2.0)[0]
    i, j = (0, 1)
    assert np.allclose(q[:, i], -2 * x[0, :, j], atol=1e-6) and np.allclose(q[:, j], 2 * x[0, :, i], atol=1e-6)


def test_what_rows_see():
    """By hand: a tree of five nodes, two of them roots, behind three tokens."""
    words = words_of([-1, 0, 0, -1, 2])
    assert words == [1, 3, 5, 8, 21] and depths_of([-1, 0, 0, -1, 2]) == [0, 1, 1, 0, 2] and path_to([-1, 0, 0, -1, 2], 4) == [0, 2, 4]
    assert [ot.tree_sees(w, i, 5, 8) for i, w in enumerate(words)] == [[0, 1, 2, 3], [0, 1, 2, 3, 4], [0, 1, 2, 3, 5], [0, 1, 2, 6], [0, 1, 2, 3, 5, 7]]
    assert ot.tree_sees(words[4], 4, 5, 8, window=4) == [2, 3, 5, 7]        # it stands at 5: 2, 3, 4, 5
    assert ot.tree_sees(words[4], 4, 5, 8, window=2, sinks=1) == [0, 3, 5, 7]
    assert ot.tree_sees(1 << 9, 1, 5, 3) == [] and ot.tree_sees(31, 0, 5, 3) == [0, 1, 2]
    assert ot.window_sees(1, 2, 10, 3, 0) == [7, 8, 9] and ot.window_sees(0, 2, 10, 3, 2) == [0, 1, 6, 7, 8] and ot.window_sees(0, 4, 2, 3, 9) == []


def test_attention_of_a_tree_in_decimals():
    """A small tree, element by element with 40 digits."""
    getcontext().prec = 40
    rng = np.random.default_rng(7)
    page, end, n = 16, 9, 4
    bits = lambda *s: ot.bf16_bits(rng.standard_normal(s))
    table = np.array([[1, 0]], np.int32)
    pages = np.zeros((2, 1, oc.page_bytes(oc.BF16, 1, page)), np.uint8)
    pages = oc.write(pages, oc.BF16, page, table, bits(end, 1, 128), bits(end, 1, 128), [0, end], [end])
    words, q = words_of([-1, 0, 0, 1]), bits(n, 2, 128)
    out, lse = ot.attend(q, pages, oc.BF16, page, table, [0, n], [end], 0.125, lambda row, i, n, end: ot.tree_sees(words[row], i, n, end, 5, 1))
    k, v, _ = oc.tokens(pages, oc.BF16, page, table, 0, end)
    for i, sees in enumerate(([0, 1, 2, 3, 4, 5], [0, 2, 3, 4, 5, 6], [0, 2, 3, 4, 5, 7], [0, 3, 4, 5, 6, 8])):
        for h in range(2):
            x = [Decimal(float(a)) for a in bf16_bits_to_f64(q[i, h])]
            w = [(sum(a * Decimal(float(b)) for a, b in zip(x, k[0, t])) * Decimal("0.125")).exp() for t in sees]
            for c in (0, 77):
                o = sum(a * Decimal(float(v[0, t, c])) for a, t in zip(w, sees)) / sum(w)
                assert abs(float(o) - out[i, h, c]) <= 1e-13
            assert abs(float(sum(w).ln()) - lse[i, h]) <= 1e-13


def test_kept_paths_by_hand():
    page, table = 16, np.array([[2, 0], [1, -1]], np.int32)
    pages = np.random.default_rng(3).integers(0, 256, (3, 2, oc.page_bytes(oc.MXFP4, 1, page))).astype(np.uint8)
    got = ot.keep(pages, oc.MXFP4, page, table, [[3, 0, 1], [0, 2]], [0, 4, 7], [18, 5])
    for old, new in zip(oc.parts(pages, oc.MXFP4, page), oc.parts(got, oc.MXFP4, page)):
        assert np.array_equal(new[2, :, 14], old[0, :, 1]) and np.array_equal(new[2, :, 15], old[2, :, 14])     # tokens 17, 14 -> 14, 15
        assert np.array_equal(new[0, :, 0], old[2, :, 15]) and np.array_equal(new[0, :, 1:], old[0, :, 1:])     # 15 -> 16; 17 stays
        assert np.array_equal(new[1, :, 3], old[1, :, 4]) and np.array_equal(new[1, :, 2], old[1, :, 2])


# ---- PagedCache -----------------------------------------------------------------------------------
BF = torch.bfloat16


@pytest.fixture
def reached(monkeypatch):
    calls = []
    for name in ("ss_cache_append", "ss_cache_attend", "ss_cache_attend_tree", "ss_cache_attend_window", "ss_cache_keep"):
        monkeypatch.setattr(ss, name, lambda *a, _name=name, **kw: calls.append((_name, a)))
    monkeypatch.setattr(H.PagedCache, "_on_current_device", lambda self: None)
    return calls


def _cache(**kw):
    p = H.PagedCache(2, 8, 2, 64, ss.SS_CACHE_BF16, 16, **{"max_rows": 4, "device": "cpu", "tree_rows": 10, **kw})
    p.grow([20, 20])
    return p


def test_paged_cache_of_trees_is_checked():
    assert _cache().workspace.numel() == max(ss.ss_cache_attend_workspace_bytes(_cache().desc), ss.ss_cache_attend_tree_workspace_bytes(_cache().tree_desc))
    for rows in (65, -1):
        with pytest.raises(ss.SpecStreamError, match="max_rows"):
            _cache(tree_rows=rows)
    p = _cache(tree_rows=0)
    q, out, lse = torch.zeros(8, 8, 128, dtype=BF), torch.zeros(8, 8, 128), torch.zeros(8, 8)
    for call in (lambda: p.attend_tree(q, torch.zeros(8, dtype=torch.int64), out, lse, 0), lambda: p.keep([[0], [0]], [1, 1])):
        with pytest.raises(ValueError, match="tree_rows"):
            call()


def test_paged_cache_append(reached):
    p = _cache()
    k, q, f = torch.zeros(8, 2, 128, dtype=BF), torch.zeros(8, 8, 128, dtype=BF), torch.zeros(64)
    pos = torch.zeros(8, dtype=torch.int32)
    p.append(k, k, f, 0, None, pos, q, q)
    p.append(k, k, f[:16], 0)
    assert len(reached) == 2
    meta = lambda x: torch.empty_like(x, device="meta")
    for call in (lambda: p.append(k.float(), k, f, 0), lambda: p.append(k, k[:7], f, 0), lambda: p.append(meta(k), k, f, 0),
                 lambda: p.append(k, k, f.double(), 0), lambda: p.append(k, k, meta(f), 0), lambda: p.append(k, k, f[::2], 0),
                 lambda: p.append(k, k, [1.0], 0), lambda: p.append(k, k, f, 0, None, pos.long()), lambda: p.append(k, k, f, 0, None, pos[:7]),
                 lambda: p.append(k, k, f, 0, pos), lambda: p.append(k, k, f, 0, q=q), lambda: p.append(k, k, f, 0, q_out=q),
                 lambda: p.append(k, k, f, 0, q=q[:7], q_out=q[:7]), lambda: p.append(k, k, f, 0, q=q, q_out=q[:1]),
                 lambda: p.append(k, k, f, 0, q=q, q_out=q[:1].expand(8, 8, 128)), lambda: p.append(k, k, f, 0, q=k, q_out=k)):
        with pytest.raises(ValueError):
            call()
    assert len(reached) == 2


def test_paged_cache_attentions(reached):
    p = _cache()
    q, out, lse, tree = torch.zeros(8, 8, 128, dtype=BF), torch.zeros(8, 8, 128), torch.zeros(8, 8), torch.zeros(8, dtype=torch.int64)
    p.attend(q, out, lse, 0)
    p.attend(q, out, None, 0, window=5, sinks=2)
    p.attend_tree(q, tree, out, lse, 0, prev=(out, lse), window=5)
    p.attend_tree(q, tree.view(torch.uint64), out, lse, 0)
    assert [c[0] for c in reached] == ["ss_cache_attend", "ss_cache_attend_window", "ss_cache_attend_tree", "ss_cache_attend_tree"]
    for call in (lambda: p.attend(q, out, lse, 0, window=2 ** 32 + 5), lambda: p.attend_tree(q, tree, out, lse, 0, window=2 ** 31),
                 lambda: p.attend(q, out, lse, 0, window=4, sinks=2 ** 33), lambda: p.attend(q, out, lse, 0, window=-1), lambda: p.attend(q, out, lse, 0, sinks=1), lambda: p.attend(q, out, lse, 0, window=2, sinks=-1),
                 lambda: p.attend_tree(q, tree, out, lse, 0, sinks=4), lambda: p.attend_tree(q, tree[:7], out, lse, 0),
                 lambda: p.attend_tree(q, tree.int(), out, lse, 0), lambda: p.attend_tree(q, [0] * 8, out, lse, 0),
                 lambda: p.attend_tree(q, torch.zeros(16, dtype=torch.int64)[::2], out, lse, 0),
                 lambda: p.attend_tree(q, torch.empty(8, dtype=torch.int64, device="meta"), out, lse, 0),
                 lambda: p.attend_tree(q, tree, out.half(), lse, 0), lambda: p.attend_tree(q, tree, out, lse[:7], 0),
                 lambda: p.attend_tree(q.float(), tree, out, lse, 0)):
        with pytest.raises(ValueError):
            call()
    assert len(reached) == 4


def test_paged_cache_keep_counts_and_refuses(reached, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("S", (), {"cuda_stream": 0})())
    p = _cache()
    state = lambda: (list(p.tokens), [list(x) for x in p.owned], list(p.free), p.table.tolist(), p.end.tolist())
    before = state()
    for kept, rows in (([[0]], [1, 1]), ([[0], [0]], [1]), ([[0], [0]], [11, 1]), ([[0], [0, 1]], [1, 1]), ([[1], [0]], [1, 1]),
                       ([[-1], [0]], [1, 1]), ([[0], [0]], [1, -1])):
        with pytest.raises(ValueError):
            p.keep(kept, rows)
        assert state() == before
    with pytest.raises(TypeError):
        p.keep([[0.5], [0]], [1, 1])
    assert state() == before and reached == []
    p.keep([[0, 1, 2], []], [3, 0])                   # nothing moves, nothing leaves
    assert state() == before and reached == []
    p.keep([[0, 1], [0]], [6, 4])                     # nothing moves
    assert p.tokens == [16, 17] and p.end.tolist() == [16, 17] and [len(x) for x in p.owned] == [1, 2] and reached == []
    p.grow([4, 4])
    p.keep([[3], [0, 2]], [4, 4])
    assert p.tokens == [17, 19] and p.end.tolist() == [17, 19] and [c[0] for c in reached] == ["ss_cache_keep"]

    def full(*a, **kw):
        raise RuntimeError("out of memory")

    before = state()
    with monkeypatch.context() as m:
        m.setattr(torch, "tensor", full)
        with pytest.raises(RuntimeError):
            p.keep([[1], [0]], [2, 2])
    assert state() == before
    monkeypatch.setattr(ss, "ss_cache_keep", full)
    with pytest.raises(RuntimeError):
        p.keep([[1], [0]], [2, 2])
    assert state() == before


def test_paged_cache_keep_hands_over_paths_and_starts(monkeypatch):
    """What the library is given: counts, row starts and nodes as int32 arrays on the cache's device."""
    seen = {}

    def keep(desc, pages, table, kept, num_kept, num_rows, end, row_start, stream):
        import ctypes
        read = lambda at, n: list((ctypes.c_int32 * n).from_address(at))
        seen.update(kept=read(kept, num_rows), num=read(num_kept, 2), start=read(row_start, 3), rows=num_rows, end=read(end, 2))

    monkeypatch.setattr(ss, "ss_cache_keep", keep)
    monkeypatch.setattr(H.PagedCache, "_on_current_device", lambda self: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("S", (), {"cuda_stream": 0})())
    p = _cache()
    p.keep([[2, 4], [0]], [5, 3])
    assert seen == {"kept": [2, 4, -1, -1, -1, 0, -1, -1], "num": [2, 1], "start": [0, 5, 8], "rows": 8, "end": [20, 20]}
    assert p.tokens == [17, 18]
