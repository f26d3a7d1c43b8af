"""Timed cases of tree drafting over a paged cache: rotated rows appended to it, a tree or a window of it attended, the
accepted path kept.

The cache is the one of ``ss_cache_write`` and ``ss_cache_attend``: pages of ``page`` tokens that a table hands out per
request, in bf16, or in 8 or 4 bits with one power-of-two scale per 32 channels; request b's rows are row_start[b] ..
row_start[b + 1] - 1 and its i-th of n_b rows stands for the token at end_b - n_b + i.

append  K rows turned by their position (pairs of channels by position times frequency), written; V rows written; Q rows
        turned too.
tree    the last n_b tokens are a tree of drafted ones: row i sees the tokens before the tree and, of the tree, those whose
        bit is set in its word (itself and what it descends from).
window  row at position p sees the tokens t <= p with t > p - window or t < sinks.
keep    of the last n_b tokens the given ones move to the first places, in the given order.

``listed`` names the cases that stand for real use, ``draw`` gives more of the same ranges, ``prepare`` makes what a
serving loop holds before the call, ``run`` is the call (or, with ``own`` false, the same in elementary torch
operations), and ``exact`` computes the definition in float64.

Layout of a page: per KV head one block of ``page`` K rows, ``page`` V rows and, for the scaled formats, ``page`` times
4 scale bytes of K and then of V.  A row is 128 channels: 256, 128 or 64 bytes, the lower channel of a 4-bit pair in
the lower bits.  A scale byte e stands for 2^(e - 127).
"""
from __future__ import annotations

import math
import random

import torch

own = False

HEAD_DIM = 128
BLOCK = 32                                               # channels that share a scale
BLOCKS = HEAD_DIM // BLOCK
FORMATS = {"bf16": 0, "mxfp8": 1, "mxfp4": 2}            # the library's numbers for them
ROW_BYTES = {"bf16": 256, "mxfp8": 128, "mxfp4": 64}
SCALE_BYTES = {"bf16": 0, "mxfp8": BLOCKS, "mxfp4": BLOCKS}
LEAST_EXPONENT = -111
MOST_NODES = 64                                          # of a tree
# query and KV heads: the 7-8B layer, the 48- and 64-head targets, the half of a 64-head one on each of two GPUs, the
# small test model, and one query head per KV head
HEADS = ((32, 8), (48, 8), (64, 8), (32, 4), (8, 2), (16, 16))


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def _case(name, op, requests, tokens, rows, heads, fmt, page, **more):
    """tokens: what the cache holds of a request before the rows of the call; rows: n_b."""
    c = {"name": name, "op": op, "requests": requests, "tokens_min": tokens[0], "tokens_max": tokens[1], "rows_min": rows[0],
         "rows_max": rows[1], "q_heads": heads[0], "kv_heads": heads[1], "format": fmt, "page": page, "shape_seed": 4,
         "window": 0, "sinks": 0, "kept_max": 8, "rotary_dim": HEAD_DIM, "interleaved": False, "before": 0,
         "drafted": False}
    c.update(more)
    return c


def listed():
    return [
        # every decode step behind a history on the host: the cache holds each request's last tokens only, whose positions
        # are far, and half of each head turns in neighbouring pairs
        _case("append_decode_64", "append", 64, (33, 3000), (1, 1), (32, 8), "mxfp8", 16, rotary_dim=64, interleaved=True,
              before=100000),
        # prompts of mixed lengths entering the cache: the most rows
        _case("append_prompts", "append", 16, (0, 0), (2048, 8191), (32, 8), "mxfp8", 64),
        # drafted trees entering the cache before they attend, siblings at one position
        _case("append_trees_16", "append", 16, (500, 8000), (16, 48), (64, 8), "bf16", 64, drafted=True),
        # the smallest call: one short chat, a handful of drafted tokens; launches and latency count
        _case("tree_chat_300", "tree", 1, (300, 300), (8, 8), (8, 2), "bf16", 16),
        # one interactive user, a long context in 8 bits, the widest tree
        _case("tree_one_32k", "tree", 1, (32768, 32768), (64, 64), (32, 8), "mxfp8", 64),
        # the benchmark's Cohort, a tree of a few branches, 96 query rows on every KV head
        _case("tree_verify_16x32k", "tree", 16, (32768, 32768), (24, 24), (32, 8), "mxfp8", 64),
        # wide trees over unquantised contexts, 256 query rows on every KV head: the most arithmetic
        _case("tree_wide_16x16k", "tree", 16, (12000, 16384), (64, 64), (32, 8), "bf16", 32),
        # contexts and trees of every size in one call, 4 bits, 6 query heads per KV head
        _case("tree_24_ragged", "tree", 24, (33, 3000), (1, 64), (48, 8), "mxfp4", 32),
        # plain decoding of a windowed layer, contexts that differ by a factor of 32
        _case("window_decode_64", "window", 64, (2048, 65536), (1, 1), (32, 8), "bf16", 16, window=4096, sinks=4),
        # the benchmark's Cohort verifying a chain of candidates in a windowed layer, 64 query rows on every KV head
        _case("window_verify_16x32k", "window", 16, (32768, 32768), (8, 8), (64, 8), "mxfp4", 64, window=1024, sinks=64),
        # the accepted paths of many short trees
        _case("keep_256", "keep", 256, (33, 3000), (1, 64), (32, 8), "bf16", 16, kept_max=12),
        # one request's accepted path in 4 bits: a launch
        _case("keep_one", "keep", 1, (32768, 32768), (64, 64), (32, 8), "mxfp4", 64),
    ]


MOST_PADDED = 16 * 32832 * 8      # tokens and KV heads that the plain form spans, every request as long as the longest
MOST_SCORES = 16 * 16448 * 8 * 256


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1

    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(("append", "append", "tree", "tree", "tree", "tree", "window", "window", "window", "keep"))
        heads = rng.choice(HEADS)
        fmt = rng.choice(("bf16", "mxfp8") if op == "append" else ("bf16", "mxfp8", "mxfp4"))
        requests = max(1, log_int(1, 256))
        hi = log_int(16, 65536)
        tokens = (hi if rng.random() < 0.3 else log_int(0, hi), hi)
        window = sinks = 0
        drafted = op == "append" and rng.random() < 0.3
        if op == "append":
            top = rng.randint(1, MOST_NODES) if drafted else max(1, log_int(1, 16384))
            tokens = (0, min(hi, 5000))
        elif op == "window":
            top = rng.randint(1, min(8, 64 // (heads[0] // heads[1])))
            window, sinks = max(1, log_int(1, 8192)), rng.choice((0, 1, 4, 64, rng.randint(0, 128)))
        else:
            top = rng.randint(1, MOST_NODES)
            if op == "tree" and rng.random() < 0.2:
                window, sinks = max(1, log_int(16, 8192)), rng.choice((0, 4))
        rows = (top if rng.random() < 0.5 else rng.randint(1, top), top)
        c = _case("", op, requests, tokens, rows, heads, fmt, rng.choice((16, 32, 64, 128, 256)), window=window, sinks=sinks,
                  kept_max=rng.randint(1, 16), rotary_dim=rng.choice((32, 64, 96, 128, 128)), interleaved=rng.random() < 0.4,
                  before=rng.choice((0, log_int(16, 1 << 20))), drafted=drafted, shape_seed=rng.randrange(1 << 30))
        del c["name"]
        n, end = _shape(c)
        w = work(c)
        span = min(max(end), window + sinks + max(n)) if window else max(end)
        padded = len(end) * span * heads[1]
        scores = padded * max(n) * (heads[0] // heads[1]) if op in ("tree", "window") else 0
        held = len(end) * max(end) * heads[1]
        if (padded <= MOST_PADDED and scores <= MOST_SCORES and held <= 4 * MOST_PADDED and w["bytes"] <= most["bytes"]
                and w["flops"] <= most["flops"]):
            return c


def _shape(case):
    """Per request: its rows n_b and its end, the tokens in the cache once they are there."""
    r = random.Random(case["shape_seed"])

    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(r.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1))

    held = [log_int(case["tokens_min"], case["tokens_max"]) for _ in range(case["requests"])]
    rows = [log_int(case["rows_min"], case["rows_max"]) for _ in range(case["requests"])]
    return rows, [h + n for h, n in zip(held, rows)]


def _trees(case):
    """Per request: the parent of each node (-1: the last token of the context, for node 0 and its siblings), and the accepted path."""
    r = random.Random(case["shape_seed"] + 1)
    parents, paths = [], []
    for n in _shape(case)[0]:
        parent = [-1] + [max(-1, i - 1 - int(r.expovariate(0.4))) for i in range(1, n)]
        path, at = [], r.randrange(n)
        while at >= 0:
            path.append(at)
            at = parent[at]
        parents.append(parent)
        paths.append(path[::-1][:case["kept_max"]])
    return parents, paths


def _depths(parent):
    depth = []
    for p in parent:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def work(case):
    rows, end = _shape(case)
    hq, hkv, op = case["q_heads"], case["kv_heads"], case["op"]
    T = sum(rows)
    held = 2 * hkv * (ROW_BYTES[case["format"]] + SCALE_BYTES[case["format"]])    # a token in the cache
    b = f = 0
    if op == "append":
        b += T * (2 * hkv * HEAD_DIM * 2 + 2 * hq * HEAD_DIM * 2 + held) + 4 * T
        f += 6 * T * (hq + hkv) * case["rotary_dim"] // 2
    if op in ("tree", "window"):
        tokens = seen = 0
        W, S = case["window"], case["sinks"]
        for n, e, parent in zip(rows, end, _trees(case)[0]):
            depth = list(range(n)) if op == "window" else _depths(parent)
            first = e - n
            low = [max(0, first + d + 1 - W) if W else 0 for d in depth]          # of the window
            for d, at in zip(depth, low):
                seen += max(0, first - at) + min(at, S, first) + min(d + 1, W or d + 1)
            least = min(low)
            tokens += e - least + min(least, S)
        b += tokens * held + T * hq * (HEAD_DIM * 2 + (HEAD_DIM + 1) * 4)
        f += 4 * seen * hq * HEAD_DIM
    if op == "keep":
        paths = _trees(case)[1]
        b += sum(sum(at != j for j, at in enumerate(p)) for p in paths) * 2 * held + 4 * sum(len(p) + 1 for p in paths)
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _parts(pages, fmt, page):
    """Views of a cache's K and V rows [pages, KV heads, page, ...] and their scales."""
    rb, sb = ROW_BYTES[fmt], SCALE_BYTES[fmt]
    k = pages[:, :, :page * rb].unflatten(-1, (page, rb))
    v = pages[:, :, page * rb:2 * page * rb].unflatten(-1, (page, rb))
    if fmt == "bf16":
        return k.view(torch.bfloat16), v.view(torch.bfloat16), None, None
    at = 2 * page * rb
    ks = pages[:, :, at:at + page * sb].unflatten(-1, (page, sb))
    vs = pages[:, :, at + page * sb:].unflatten(-1, (page, sb))
    return k, v, ks, vs


def _encode(x, fmt):
    """Rows [..., 128] of bf16 as a cache holds them: (bytes or bf16 values, scale bytes)."""
    if fmt == "bf16":
        return x, None
    most = {"mxfp8": (0.875, 9), "mxfp4": (0.75, 3)}[fmt]                 # 448 and 6 as m 2^x
    x = x.float().unflatten(-1, (BLOCKS, BLOCK))
    m, e = torch.frexp(x.abs().amax(-1))
    e = (e - most[1] + (m > most[0]).int()).clamp(min=LEAST_EXPONENT)
    e = torch.where(m == 0, LEAST_EXPONENT, e)
    x = x / ((e + 127) << 23).view(torch.float32).unsqueeze(-1)           # exact: a power of two
    scales = (e + 127).to(torch.uint8)
    if fmt == "mxfp8":
        return x.flatten(-2).to(torch.float8_e4m3fn).view(torch.uint8), scales
    a = x.abs()
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
            + 8 * torch.signbit(x)).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, scales


def _decode(rows, scales, fmt):
    """What rows of a cache stand for, in float32."""
    if fmt == "bf16":
        return rows.float()
    if fmt == "mxfp8":
        x = rows.view(torch.float8_e4m3fn).float()
    else:
        values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=rows.device)
        values = torch.cat([values, -values])
        x = torch.stack([values[(rows & 15).int()], values[(rows >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (BLOCKS, BLOCK)) * (scales.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    """The cache with its table, rows and ends on the GPU, the new rows (queries, keys, values: views of one tensor, as the
    projection leaves them), and what the drafting hands over: the tree's words, the rows' positions, the accepted paths."""
    rows, end = _shape(case)
    parents, paths = _trees(case)
    hq, hkv, page, fmt, op = case["q_heads"], case["kv_heads"], case["page"], case["format"], case["op"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev = {"device": "cuda"}

    def normal(*shape):
        return torch.randn(shape, generator=gen, dtype=torch.bfloat16, **dev)

    B, T, width = len(rows), sum(rows), max(1, -(-max(end) // page))
    need = [-(-e // page) for e in end]
    num_pages = sum(need) + 3
    ids = torch.randperm(num_pages, generator=gen, **dev).int()
    first = torch.tensor([0] + need, **dev).cumsum(0)
    at = torch.arange(width, **dev)
    table = torch.where(at < torch.tensor(need, **dev)[:, None], ids[(first[:-1, None] + at).clamp(max=num_pages - 1)], -1).int()

    channel = (torch.rand(hkv, HEAD_DIM, generator=gen, **dev) * 1.5 + 0.5).to(torch.bfloat16)     # of the keys
    held = 2 * page * (ROW_BYTES[fmt] + SCALE_BYTES[fmt])
    pages = torch.zeros(num_pages, hkv, held, dtype=torch.uint8, **dev)
    parts = _parts(pages, fmt, page)
    if op != "append":
        for rows_at, scales_at, factor in ((parts[0], parts[2], channel[:, None]), (parts[1], parts[3], None)):
            x = normal(num_pages, hkv, page, HEAD_DIM)
            if factor is not None:
                x *= factor
            codes, scales = _encode(x, fmt)
            rows_at.copy_(codes)
            if scales is not None:
                scales_at.copy_(scales)
            del x, codes, scales
    s = {"case": case, "pages": pages, "parts": parts, "table": table, "num_rows": T, "most_rows": max(rows),
         "row_start": torch.tensor([0] + rows, **dev).cumsum(0).int(), "end": torch.tensor(end, **dev).int(),
         "scale": HEAD_DIM ** -0.5}
    fused = normal(T, hq + 2 * hkv, HEAD_DIM)
    fused[:, hq:hq + hkv] *= channel
    s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    s["row_elements"] = (hq + 2 * hkv) * HEAD_DIM
    if op == "append":
        half = case["rotary_dim"] // 2
        s["inv_freq"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(**dev)
        s["q_turned"] = torch.empty(T, hq, HEAD_DIM, dtype=torch.bfloat16, **dev)
        ahead = []
        for n, e, parent in zip(rows, end, parents):
            at = _depths(parent) if case["drafted"] else range(n)
            ahead += [case["before"] + e - n + d for d in at]
        s["positions"] = torch.tensor(ahead, **dev).int() if case["drafted"] or case["before"] else None
    if op == "tree":
        words = []
        for parent in parents:
            sees = []
            for i, p in enumerate(parent):
                sees.append((sees[p] if p >= 0 else 0) | 1 << i)
            words += sees
        s["tree"] = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, **dev)
    if op in ("tree", "window"):
        s["out"] = torch.empty(T, hq, HEAD_DIM, **dev)
        s["lse"] = torch.empty(T, hq, **dev)
    if op == "keep":
        kept = []
        for n, path in zip(rows, paths):
            kept += path + [-1] * (n - len(path))
        s["kept"] = torch.tensor(kept, **dev).int()
        s["num_kept"] = torch.tensor([len(p) for p in paths], **dev).int()
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _held(state):
    """The cache's contents as the values that it holds: an 8-bit row is a float8 one, a scale a power of two; packed 4-bit
    rows, which only a move of whole tokens returns, are bytes."""
    k, v, ks, vs = state["parts"]
    if ks is None:
        return {"k": k, "v": v}
    if state["case"]["format"] == "mxfp8":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return {"k": k, "v": v, "k_scale": ks.view(torch.float8_e8m0fnu), "v_scale": vs.view(torch.float8_e8m0fnu)}


def run(state):
    op = state["case"]["op"]
    r = {}
    if own:
        _own(state)
    if op == "append":
        if not own:
            _plain_append(state)
        r["q"] = state["q_turned"]
    if op in ("tree", "window"):
        r["out"], r["lse"] = (state["out"], state["lse"]) if own else _plain_attend(state)
    if op == "keep" and not own:
        _plain_keep(state)
    if op in ("append", "keep"):
        r.update(_held(state))
    return r


def _own(state):
    from paper_2609_33184_amd import specstream as ss

    case, op = state["case"], state["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if "desc" not in state:          # a serving loop keeps the descriptors and the workspace
        state["desc"] = ss.make_cache_desc(
            len(state["end"]), case["kv_heads"], FORMATS[case["format"]], case["page"], state["pages"].shape[0],
            state["table"].shape[1], num_q_heads=case["q_heads"], max_rows=state["most_rows"], softmax_scale=state["scale"])
        n = 0
        if op == "tree":
            n = ss.ss_cache_attend_tree_workspace_bytes(state["desc"])
        elif op == "window":
            n = ss.ss_cache_attend_workspace_bytes(state["desc"])
        state["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        if op == "append":
            state["rope"] = ss.make_rope_desc(case["rotary_dim"], state["inv_freq"].data_ptr(), interleaved=int(case["interleaved"]))
    desc, cache = state["desc"], (state["pages"].data_ptr(), state["table"].data_ptr())
    where = {"num_rows": state["num_rows"], "end": state["end"].data_ptr(), "row_start": state["row_start"].data_ptr(), "stream": stream}
    if op == "append":
        positions = state["positions"]
        ss.ss_cache_append(desc, *cache, state["rope"], state["k"].data_ptr(), state["v"].data_ptr(), row_stride=state["row_elements"],
                           q=state["q"].data_ptr(), q_out=state["q_turned"].data_ptr(), q_row_stride=state["row_elements"],
                           positions=None if positions is None else positions.data_ptr(), **where)
    if op in ("tree", "window"):
        to = {"out": state["out"].data_ptr(), "lse": state["lse"].data_ptr(), "workspace": state["workspace"].data_ptr(),
              "workspace_bytes": state["workspace"].numel(), "q_row_stride": state["row_elements"], "window": case["window"], "sinks": case["sinks"]}
        if op == "window":
            ss.ss_cache_attend_window(desc, *cache, state["q"].data_ptr(), **to, **where)
        else:
            ss.ss_cache_attend_tree(desc, *cache, state["q"].data_ptr(), tree=state["tree"].data_ptr(), **to, **where)
    if op == "keep":
        ss.ss_cache_keep(desc, *cache, kept=state["kept"].data_ptr(), num_kept=state["num_kept"].data_ptr(), **where)


def _slots(state):
    """Of every row: its request and the place of its token."""
    start, end = state["row_start"].long(), state["end"].long()
    t = torch.arange(state["num_rows"], device=start.device)
    b = torch.searchsorted(start[1:], t, right=True)
    return b, end[b] - start[b + 1] + t


def _turned(x, cos, sin, dim, interleaved):
    """Rows [T, heads, 128] with the first dim channels turned, in float32, rounded once."""
    y = x.float()
    a, b = (y[..., 0:dim:2], y[..., 1:dim:2]) if interleaved else (y[..., :dim // 2], y[..., dim // 2:dim])
    c, s = a * cos - b * sin, b * cos + a * sin
    z = torch.stack([c, s], -1).flatten(-2) if interleaved else torch.cat([c, s], -1)
    return torch.cat([z, y[..., dim:]], -1).to(x.dtype)


def _plain_append(state):
    case = state["case"]
    fmt, page, dim = case["format"], case["page"], case["rotary_dim"]
    b, slot = _slots(state)
    position = slot if state["positions"] is None else state["positions"]
    angle = position.double()[:, None, None] * state["inv_freq"].double()        # far positions: float32 would lose it
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    state["q_turned"] = _turned(state["q"], cos, sin, dim, case["interleaved"])
    at, slot = state["table"].long()[b, slot // page][:, None], (slot % page)[:, None]
    head = torch.arange(case["kv_heads"], device=slot.device)[None]
    k, v, ks, vs = state["parts"]
    (kc, ksc), (vc, vsc) = _encode(_turned(state["k"], cos, sin, dim, case["interleaved"]), fmt), _encode(state["v"], fmt)
    k[at, head, slot], v[at, head, slot] = kc, vc
    if ks is not None:
        ks[at, head, slot], vs[at, head, slot] = ksc, vsc


def _plain_attend(state):
    """Every request padded to the longest, or to the window and the sinks; scores, weights and sums in float32."""
    case = state["case"]
    fmt, hq, hkv, most, page = case["format"], case["q_heads"], case["kv_heads"], state["most_rows"], case["page"]
    W, S, G = case["window"], case["sinks"], case["q_heads"] // case["kv_heads"]
    start, end, table = state["row_start"].long(), state["end"].long(), state["table"].long().clamp(min=0)
    B, reach = len(end), table.shape[1] * page
    n = start[1:] - start[:-1]
    first = (end - n)[:, None]
    i = torch.arange(most, device=end.device)
    row = (start[:-1, None] + i).clamp(max=state["num_rows"] - 1)
    q = state["q"][row].float().view(B, most, hkv, G, HEAD_DIM)
    q = q.transpose(1, 2).reshape(B, hkv, most * G, HEAD_DIM)

    t = torch.arange(reach, device=end.device)[None].expand(B, -1)                # the tokens to look at
    fresh = torch.ones_like(t, dtype=torch.bool)
    if W and W + S + most < reach:
        low = (first - W + 1).clamp(min=0)
        near = low + torch.arange(W + most, device=end.device)
        far = torch.arange(S, device=end.device)[None].expand(B, -1)
        t, fresh = torch.cat([far, near], 1), torch.cat([far < low, torch.ones_like(near, dtype=torch.bool)], 1)
    here = fresh & (t < end[:, None])
    t = t.clamp(max=reach - 1)
    if case["op"] == "window":
        ahead = i[None].expand(B, -1)
        seen = (t[:, None] <= (first + ahead)[:, :, None])
    else:
        word = state["tree"][row]
        bits = (word[:, :, None] >> torch.arange(MOST_NODES, device=end.device)) & 1
        ahead = bits.sum(-1) - 1
        node = t - first
        mine = torch.gather(bits, 2, node.clamp(0, MOST_NODES - 1)[:, None].expand(B, most, -1)).bool()
        seen = torch.where((node < 0)[:, None], True, mine)
    if W:
        inside = (t[:, None] > (first + ahead - W)[:, :, None]) | (t < S)[:, None]
        seen = seen & (inside if case["op"] == "window" else inside | (t >= first)[:, None])
    seen = seen & here[:, None]
    at, slot = torch.gather(table, 1, t // page), t % page

    def tokens(rows, scales):
        x = _decode(rows[at, :, slot], None if scales is None else scales[at, :, slot], fmt)        # [B, tokens, KV heads, 128]
        return x.transpose(1, 2).contiguous()

    k, v, ks, vs = state["parts"]
    s = torch.matmul(q, tokens(k, ks).transpose(2, 3)) * state["scale"]
    s = s.masked_fill(~seen[:, None, :, None, :].expand(B, hkv, most, G, -1).reshape(s.shape), float("-inf"))
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s = torch.exp(s - m)
    l = s.sum(-1, keepdim=True)
    o = torch.matmul(s, tokens(v, vs)) / l.clamp(min=1e-38)
    lse = (m + torch.log(l)).masked_fill(l == 0, float("-inf"))
    b, _ = _slots(state)
    at = torch.arange(state["num_rows"], device=b.device) - start[b]
    o = o.view(B, hkv, most, G, HEAD_DIM).transpose(1, 2)[b, at].reshape(-1, hq, HEAD_DIM)
    return o, lse.view(B, hkv, most, G).transpose(1, 2)[b, at].reshape(-1, hq)


def _plain_keep(state):
    page, start, end, table = state["case"]["page"], state["row_start"].long(), state["end"].long(), state["table"].long()
    b, _ = _slots(state)
    j = torch.arange(state["num_rows"], device=b.device) - start[b]
    n = (start[1:] - start[:-1])[b]
    take = j < state["num_kept"][b]
    old, new = (end[b] - n + state["kept"]).where(take, 0), (end[b] - n + j).where(take, 0)
    for part in state["parts"]:
        if part is not None:
            from_ = part[table[b, old // page], :, old % page]
            to = (table[b, new // page][take], slice(None), (new % page)[take])
            part[to] = from_[take]


# ------------------------------------------------------------------------------------------------
# the definition in float64
# ------------------------------------------------------------------------------------------------
def _values(fmt, device):
    """What each code stands for, by the formats' bits: sign, exponent, fraction."""
    ebits, mbits, bias = {"mxfp8": (4, 3, 7), "mxfp4": (2, 1, 1)}[fmt]
    c = torch.arange(1 << (1 + ebits + mbits), device=device)
    e, f = (c >> mbits) & ((1 << ebits) - 1), (c & ((1 << mbits) - 1)).double() / (1 << mbits)
    x = torch.where(e == 0, f * 2.0 ** (1 - bias), (1 + f) * torch.exp2((e - bias).double()))
    x = torch.where(c >> (ebits + mbits) == 1, -x, x)
    if fmt == "mxfp8":
        x[0x7F], x[0xFF] = float("nan"), float("nan")
    return x


def _exact_tokens(state, b, upto, which):
    """K (which 0) or V (1) of request b's tokens [0, upto) in float64, [KV heads, upto, 128]."""
    fmt, page = state["case"]["format"], state["case"]["page"]
    ids = state["table"][b, :-(-upto // page)].long()
    rows = state["parts"][which][ids]
    if fmt == "bf16":
        x = rows.double()
    else:
        if fmt == "mxfp4":
            rows = torch.stack([rows % 16, rows // 16], -1).flatten(-2)
        x = _values(fmt, rows.device)[rows.long()]
        x = x * torch.exp2(state["parts"][2 + which][ids].double() - 127).repeat_interleave(BLOCK, -1)
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, HEAD_DIM)[:, :upto]


def _exact_stored(x, fmt):
    """The codes' values that rows [..., 128] are stored as: the nearest code, the even one of two."""
    x = x.double()
    if fmt == "bf16":
        return x
    top = {"mxfp8": 448.0, "mxfp4": 6.0}[fmt]
    xb = x.unflatten(-1, (BLOCKS, BLOCK))
    peak = xb.abs().amax(-1)
    e = torch.ceil(torch.log2(peak / top)).nan_to_num(neginf=-1000)
    e = torch.where(peak > top * torch.exp2(e), e + 1, e)
    e = torch.where(peak <= top * torch.exp2(e - 1), e - 1, e).clamp(min=LEAST_EXPONENT)
    xs = xb * torch.exp2(-e)[..., None]
    grid = _values(fmt, x.device)
    grid = grid[:len(grid) // 2]
    grid = grid[~grid.isnan()]
    a = xs.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    near = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(grid[near], xs).flatten(-2)


def _exact_turn(x, position, inv_freq, interleaved):
    """Each pair of channels as a complex number times e^(i position frequency), in float64."""
    y = x.double()
    half = len(inv_freq)
    first = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=x.device), position.double()[:, None] * inv_freq.double())
    z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    op, fmt, page, hq, hkv = case["op"], case["format"], case["page"], case["q_heads"], case["kv_heads"]
    if op == "keep":
        return None                                       # nothing is computed: whole tokens move
    state = prepare(case, seed)
    rows, end = _shape(case)
    parents = _trees(case)[0]
    r = {}
    if op == "append":
        position = state["positions"]
        if position is None:
            position = torch.cat([torch.arange(e - n, e) for n, e in zip(rows, end)]).cuda()
        r["q"] = _exact_turn(state["q"], position, state["inv_freq"], case["interleaved"])
        stored = {"k": _exact_turn(state["k"], position, state["inv_freq"], case["interleaved"]).to(torch.bfloat16), "v": state["v"]}
        whole = {}
        for name, which in (("k", 0), ("v", 1)):
            part = state["parts"][which]
            whole[name] = (part.view(torch.float8_e4m3fn) if fmt == "mxfp8" else part).double()
            code = _exact_stored(stored[name], fmt)
            at = 0
            for b, n in enumerate(rows):
                pos = torch.arange(end[b] - n, end[b], device="cuda")
                whole[name][state["table"][b].long()[pos // page], :, pos % page] = code[at:at + n]
                at += n
        r.update(whole)
        if fmt != "bf16":
            r["k_scale"] = r["v_scale"] = None
    if op in ("tree", "window"):
        W, S = case["window"], case["sinks"]
        out = torch.zeros(sum(rows), hq, HEAD_DIM, dtype=torch.float64, device="cuda")
        lse = torch.full((sum(rows), hq), -math.inf, dtype=torch.float64, device="cuda")
        at = 0
        for b, (n, e) in enumerate(zip(rows, end)):
            k, v = _exact_tokens(state, b, e, 0), _exact_tokens(state, b, e, 1)
            queries = state["q"][at:at + n].double()
            for i in range(n):
                if op == "window":
                    line, p = list(range(i + 1)), e - n + i
                    line = [x for x in line if e - n + x > p - W or e - n + x < S]
                else:
                    line, x = [], i
                    while x >= 0:
                        line.append(x)
                        x = parents[b][x]
                    p = e - n + len(line) - 1
                past = list(range(0, min(S, e - n))) + list(range(max(min(S, e - n), p - W + 1), e - n)) if W else range(0, e - n)
                if W:
                    see = torch.tensor(list(past) + [e - n + x for x in line], dtype=torch.long, device="cuda")
                    ks, vs = k[:, see], v[:, see]
                else:
                    see = torch.tensor([e - n + x for x in line], dtype=torch.long, device="cuda")
                    ks, vs = torch.cat([k[:, :e - n], k[:, see]], 1), torch.cat([v[:, :e - n], v[:, see]], 1)
                s = torch.bmm(queries[i].view(hkv, -1, HEAD_DIM), ks.transpose(1, 2).contiguous()) * state["scale"]
                out[at + i] = torch.bmm(torch.softmax(s, -1), vs).reshape(hq, HEAD_DIM)
                lse[at + i] = torch.logsumexp(s, -1).reshape(hq)
            at += n
        r["out"], r["lse"] = out, lse
    return r
