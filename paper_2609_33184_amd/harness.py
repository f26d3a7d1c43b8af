"""Device buffers and round drivers over the C ABI (used by tests, bench, smoke).

Torch provides device memory, pinned host memory and streams only; every step
of the round runs in libspecstream's kernels through the binding.
"""
from __future__ import annotations

import itertools
import operator
from typing import Callable, Dict, List, Optional, Sequence, Tuple

import torch

from . import specstream as ss
from .workloads import Workload

BF16_BYTES = 2


class RoundBuffers:
    """Queries, candidate K/V, workspace and outputs of one layer's round."""

    def __init__(self, w: Workload, layer: int = 0, device="cuda", split_tokens: int = 0,
                 mfma_min_rows: int = 0, max_chunk_tokens: Optional[int] = None,
                 kv_layout: int = ss.SS_KV_TOKEN_MAJOR, balance_permille: int = 0, counters_zeroed: int = 0):
        self.w = w
        self.layer = layer
        self.device = device
        self.q = w.q_all(layer, device)
        self.kc = w.k_cand_all(layer, device)
        self.vc = w.v_cand_all(layer, device)
        mct = max_chunk_tokens or max(1, max(sum(w.chunk_lens(j)) for j in range(max(1, w.num_chunks))))
        self.kv_layout = kv_layout
        self.desc = ss.make_desc(w.num_cand, w.num_q_heads, w.num_kv_heads, w.head_dim, w.softmax_scale,
                                 mct, split_tokens, mfma_min_rows, kv_layout, balance_permille, counters_zeroed)
        self.ws_bytes = ss.ss_round_workspace_bytes(self.desc)
        if self.ws_bytes == 0:
            raise ss.SpecStreamError(ss.SS_ERR_INVALID_ARGUMENT, "ss_round_workspace_bytes", ss.ss_last_error())
        # with counters_zeroed the rounds rely on the workspace's counter block being zero: zero-fill it once
        alloc = torch.zeros if counters_zeroed else torch.empty
        self.ws = alloc(self.ws_bytes, dtype=torch.uint8, device=device)
        rows = w.total_rows
        self.out = torch.empty(rows, w.num_q_heads, w.head_dim, dtype=torch.float32, device=device)
        self.lse = torch.empty(rows, w.num_q_heads, dtype=torch.float32, device=device)

    def set_layer(self, layer: int) -> None:
        """New per-layer queries (candidates and history are shared by layers)."""
        self.layer = layer
        self.q.copy_(self.w.q_all(layer, self.device))


def hbm_history(w: Workload, layer: int = 0, device="cuda", kv_layout: int = ss.SS_KV_TOKEN_MAJOR
                ) -> List[Tuple[torch.Tensor, torch.Tensor]]:
    """Every history chunk resident in device memory: [(k_j, v_j)] in the
    given chunk layout."""
    return [w.chunk_kv(j, layer, device, head_major=kv_layout == ss.SS_KV_HEAD_MAJOR,
                       kv_interleaved=kv_layout == ss.SS_KV_HEAD_MAJOR_KV) for j in range(w.num_chunks)]


def run_round(b: RoundBuffers, chunks: Sequence[Tuple[torch.Tensor, torch.Tensor]], stream: int,
              order: Optional[Sequence[int]] = None, cand_position: Optional[int] = None,
              lens: Optional[Sequence[Sequence[int]]] = None, batch: int = 1, scratch: bool = False) -> None:
    """Enqueue one whole round (init, history chunks, candidates, finalize)
    on `stream`; results land in b.out / b.lse.  ``batch`` > 1 groups that
    many consecutive chunks into one ss_attend_history_chunks call.  With
    ``scratch`` the round starts with ss_round_init_scratch (the
    library's own workspace) instead of b.ws."""
    w = b.w
    order = list(range(len(chunks))) if order is None else list(order)
    pos = len(order) if cand_position is None else cand_position
    step = max(1, batch)
    groups = [order[i0:i0 + step] for i0 in range(0, len(order), step)]
    if scratch:
        r = ss.ss_round_init_scratch(b.desc, b.q.data_ptr(), stream)
    else:
        r = ss.ss_round_init(b.desc, b.q.data_ptr(), b.ws.data_ptr(), b.ws_bytes, stream)

    def args(grp):
        ks = [chunks[j][0].data_ptr() if chunks[j][0].numel() else 0 for j in grp]
        vs = [chunks[j][1].data_ptr() if chunks[j][1].numel() else 0 for j in grp]
        ls = [w.chunk_lens(j) if lens is None else lens[j] for j in grp]
        return ks, vs, ls

    try:
        done = 0
        for gi, grp in enumerate(groups):
            if done <= pos < done + len(grp) or (pos == done and gi == 0):
                ss.ss_attend_local_candidates(r, b.kc.data_ptr(), b.vc.data_ptr(), stream)
            ks, vs, ls = args(grp)
            if batch > 1:
                ss.ss_attend_history_chunks(r, ks, vs, ls, None, None, stream)
            else:
                ss.ss_attend_history_chunk(r, ks[0], vs[0], ls[0], None, None, stream)
            done += len(grp)
        if pos >= len(order):
            ss.ss_attend_local_candidates(r, b.kc.data_ptr(), b.vc.data_ptr(), stream)
        ss.ss_round_finalize(r, b.out.data_ptr(), b.lse.data_ptr(), stream)
    finally:
        ss.ss_round_destroy(r)


def capture_round(b: RoundBuffers, chunks: Sequence[Tuple[torch.Tensor, torch.Tensor]], batch: int = 1,
                  pool=None) -> "torch.cuda.CUDAGraph":
    """Capture one whole round (the same calls as run_round) into a HIP graph.

    Every step the library enqueues is a kernel launch with its arguments by
    value (no memsets, no host waits), so a replay redoes the round on the
    buffers it was captured with: b.q, b.kc, b.vc, the chunks, b.ws and
    b.out / b.lse.  Replays serve loops that re-run a round of the same
    shape with new contents in those buffers, without the host's per-call
    work."""
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, pool=pool):
        run_round(b, chunks, torch.cuda.current_stream().cuda_stream, batch=batch)
    return g


class HostHistory:
    """One layer's history in pinned host memory, chunk j as its K then its V
    (each in the round's chunk layout; with the interleaved layout the chunk's
    one K-and-V buffer), for streaming through the two-slot pipeline."""

    def __init__(self, w: Workload, layer: int = 0, gen_device="cuda", kv_layout: int = ss.SS_KV_TOKEN_MAJOR):
        self.w = w
        hm = kv_layout == ss.SS_KV_HEAD_MAJOR
        il = kv_layout == ss.SS_KV_HEAD_MAJOR_KV
        tb = w.num_kv_heads * w.head_dim * BF16_BYTES
        self.sizes = [2 * sum(w.chunk_lens(j)) * tb for j in range(w.num_chunks)]
        self.offsets = []
        acc = 0
        for s in self.sizes:
            self.offsets.append(acc)
            acc += s
        self.total_bytes = acc
        self.buf = torch.empty(max(1, acc), dtype=torch.uint8, pin_memory=True)
        for j in range(w.num_chunks):
            if self.sizes[j] == 0:
                continue
            k, v = w.chunk_kv(j, layer, gen_device, head_major=hm, kv_interleaved=il)
            half = self.sizes[j] // 2
            o = self.offsets[j]
            if il:      # one buffer: the views' base holds K and V rows
                kv = torch.as_strided(k, (self.sizes[j] // BF16_BYTES,), (1,))
                self.buf[o:o + 2 * half].copy_(kv.view(torch.uint8).cpu())
            else:
                self.buf[o:o + half].copy_(k.view(-1).view(torch.uint8).cpu())
                self.buf[o + half:o + 2 * half].copy_(v.view(-1).view(torch.uint8).cpu())
            del k, v

    def chunk_ptr(self, j: int) -> int:
        return self.buf.data_ptr() + self.offsets[j]

    def max_chunk_bytes(self) -> int:
        return max(self.sizes) if self.sizes else 0


class Pipeline:
    """The library's two-slot pipeline with its staging buffers and copy stream."""

    def __init__(self, slot_bytes: int, device="cuda"):
        self.slot_bytes = max(256, slot_bytes)
        self.staging = [torch.empty(self.slot_bytes, dtype=torch.uint8, device=device) for _ in range(2)]
        self.copy_stream = torch.cuda.Stream(device=device)          # default priority
        self.handle = ss.ss_pipeline_create(self.staging[0].data_ptr(), self.staging[1].data_ptr(),
                                            self.slot_bytes, self.copy_stream.cuda_stream)

    def close(self) -> None:
        if self.handle:
            torch.cuda.synchronize()
            ss.ss_pipeline_destroy(self.handle)
            self.handle = None


def batch_bytes(host: HostHistory, batch: int) -> int:
    """Largest staging slot a transfer batch of `batch` adjacent chunks needs."""
    n = len(host.sizes)
    return max([sum(host.sizes[j:j + batch]) for j in range(0, n, batch)] or [0])


def run_round_streamed(b: RoundBuffers, host: HostHistory, pipe: Pipeline, stream: int,
                       order: Optional[Sequence[int]] = None, batch: int = 1) -> None:
    """Enqueue one round whose history streams from pinned host memory; with
    ``batch`` > 1, groups of that many adjacent chunks travel as one transfer
    batch (one copy, one attention launch)."""
    w = b.w
    if batch > 1 and order is not None:
        raise ValueError("transfer batches take the chunks in their host order")
    order = list(range(w.num_chunks)) if order is None else list(order)
    r = ss.ss_round_init(b.desc, b.q.data_ptr(), b.ws.data_ptr(), b.ws_bytes, stream)
    try:
        if batch > 1:
            for j0 in range(0, w.num_chunks, batch):
                grp = range(j0, min(w.num_chunks, j0 + batch))
                ss.ss_pipeline_attend_chunks(pipe.handle, r, host.chunk_ptr(j0), [w.chunk_lens(j) for j in grp],
                                             stream)
        for j in (order if batch <= 1 else []):
            ss.ss_pipeline_attend_chunk(pipe.handle, r, host.chunk_ptr(j), w.chunk_lens(j), stream)
        ss.ss_attend_local_candidates(r, b.kc.data_ptr(), b.vc.data_ptr(), stream)
        ss.ss_round_finalize(r, b.out.data_ptr(), b.lse.data_ptr(), stream)
    finally:
        ss.ss_round_destroy(r)


def _chunk_vofs(w: Workload, host: HostHistory, j: int, kv_layout: int) -> int:
    """Bytes from a chunk's K to its V in a staging buffer holding the chunk."""
    return 2 * w.head_dim if kv_layout == ss.SS_KV_HEAD_MAJOR_KV else host.sizes[j] // 2


def run_round_restored(b: RoundBuffers, host: HostHistory, dev: Sequence[torch.Tensor], copy: "torch.cuda.Stream",
                       stream: int) -> None:
    """Restore, then attend: every chunk of the history goes to its own
    device buffer (``dev[j]``, at least host.sizes[j] bytes) on the copy
    stream, and one batched call attends all of them once the last upload is
    done."""
    w = b.w
    n = w.num_chunks
    done = ss.ss_event_create()
    try:
        last = max([j for j in range(n) if host.sizes[j]], default=-1)
        for j in range(n):
            if host.sizes[j]:
                ss.ss_upload_chunk(dev[j].data_ptr(), host.chunk_ptr(j), host.sizes[j], copy.cuda_stream, None,
                                   done if j == last else None)
        r = ss.ss_round_init(b.desc, b.q.data_ptr(), b.ws.data_ptr(), b.ws_bytes, stream)
        try:
            ks = [dev[j].data_ptr() for j in range(n)]
            vs = [dev[j].data_ptr() + _chunk_vofs(w, host, j, b.kv_layout) for j in range(n)]
            ss.ss_attend_history_chunks(r, ks, vs, [w.chunk_lens(j) for j in range(n)],
                                        done if last >= 0 else None, None, stream)
            ss.ss_attend_local_candidates(r, b.kc.data_ptr(), b.vc.data_ptr(), stream)
            ss.ss_round_finalize(r, b.out.data_ptr(), b.lse.data_ptr(), stream)
        finally:
            ss.ss_round_destroy(r)
    finally:
        torch.cuda.synchronize()      # the events are destroyed only after the work that uses them
        ss.ss_event_destroy(done)


def run_round_single_slot(b: RoundBuffers, host: HostHistory, slot: torch.Tensor, copy: "torch.cuda.Stream",
                          stream: int) -> None:
    """Chunk by chunk through one staging buffer: chunk j is uploaded into
    ``slot`` once chunk j-1's attention has read it (its free event), and
    attended once its upload is done (its ready event), so uploads and
    attention alternate without overlapping."""
    w = b.w
    ready, free = ss.ss_event_create(), ss.ss_event_create()
    try:
        r = ss.ss_round_init(b.desc, b.q.data_ptr(), b.ws.data_ptr(), b.ws_bytes, stream)
        try:
            used = False
            for j in range(w.num_chunks):
                if not host.sizes[j]:
                    continue
                ss.ss_upload_chunk(slot.data_ptr(), host.chunk_ptr(j), host.sizes[j], copy.cuda_stream,
                                   free if used else None, ready)
                ss.ss_attend_history_chunk(r, slot.data_ptr(), slot.data_ptr() + _chunk_vofs(w, host, j, b.kv_layout),
                                           w.chunk_lens(j), ready, free, stream)
                used = True
            ss.ss_attend_local_candidates(r, b.kc.data_ptr(), b.vc.data_ptr(), stream)
            ss.ss_round_finalize(r, b.out.data_ptr(), b.lse.data_ptr(), stream)
        finally:
            ss.ss_round_destroy(r)
    finally:
        torch.cuda.synchronize()
        ss.ss_event_destroy(ready)
        ss.ss_event_destroy(free)


class _Order:
    """Streams of a cache's calls and of the changes of its table.  A change comes after the calls before it, a call
    after the last change, an attention after the last attention (they share a workspace); calls on the changes' own
    stream need nothing for that."""

    def __init__(self, device):
        self.device = device
        self.home = torch.cuda.current_stream(device)      # of the last change
        self.changed = torch.cuda.Event()
        self.changed.record(self.home)
        self.calls: Dict[int, torch.cuda.Event] = {}       # since then, on other streams, by handle
        self.attended: Optional[int] = None                # the last attention's stream, if there was one since

    def change_begins(self) -> None:
        now = torch.cuda.current_stream(self.device)
        if now.cuda_stream != self.home.cuda_stream:
            now.wait_stream(self.home)
        for handle, done in self.calls.items():
            if handle != now.cuda_stream:
                now.wait_event(done)
        self.home = now

    def change_ends(self) -> None:
        self.changed.record(self.home)
        self.calls.clear()
        self.attended = None

    def call_begins(self, handle: int, attends: bool) -> Optional["torch.cuda.Stream"]:
        """The call's stream, where ``call_ends`` has to mark it."""
        home = self.home.cuda_stream
        waits = attends and self.attended is not None and self.attended != handle
        if handle == home and not waits:
            if attends:
                self.attended = handle
            return None
        stream = torch.cuda.ExternalStream(handle, device=self.device) if handle else torch.cuda.default_stream(self.device)
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():   # its replays are the caller's to order
                return None
        if handle != home:
            stream.wait_event(self.changed)
        if waits:
            if self.attended == home:
                stream.wait_stream(self.home)
            else:
                stream.wait_event(self.calls[self.attended])
        return stream

    def call_ends(self, stream: "torch.cuda.Stream", attends: bool) -> None:
        handle = stream.cuda_stream
        if handle != self.home.cuda_stream:
            self.calls.setdefault(handle, torch.cuda.Event()).record(stream)
        if attends:
            self.attended = handle


class PagedCache:
    """A paged cache with its table and free pages, for a Cohort's requests.

    ``end[b]`` counts request b's tokens on the device, ``tokens[b]`` on the
    host, so that ``grow`` can hand out pages without waiting for the GPU.  The
    table and ``end`` change on torch's current stream.  A call may go to any
    stream: it comes after the changes made before it and before those made
    after it, and one attention after the other (they share ``workspace``).
    What calls on several streams write and read in the same pages is the
    caller's to order, and so are a captured call's replays: behind the changes
    that they need, never beside a change or another attention.  One host
    thread uses a cache at a time.

    ``tree_rows``: most nodes of a request's tree of drafted tokens (0: none).
    A step with trees is ``grow``, ``append`` (or ``write``), ``attend_tree``
    and ``keep``.

    ``row_start``: where each request's rows begin, and the last one's end.
    Without it every request has ``max_rows`` rows, in ``attend_tree``
    ``tree_rows``: a step whose calls take one batch of trees gives it, unless
    the two are one number."""

    def __init__(self, num_requests: int, num_q_heads: int, num_kv_heads: int, max_tokens: int, fmt: int = ss.SS_CACHE_MXFP8,
                 page_tokens: int = 64, num_pages: Optional[int] = None, max_rows: int = 1,
                 softmax_scale: Optional[float] = None, causal: int = 1, device="cuda", tree_rows: int = 0):
        width = -(-max_tokens // page_tokens)
        pages = num_requests * width if num_pages is None else num_pages
        self.desc = ss.make_cache_desc(num_requests, num_kv_heads, fmt, page_tokens, pages, width, num_q_heads,
                                       max_rows=max_rows, softmax_scale=softmax_scale, causal=causal)
        page_bytes = ss.ss_cache_page_bytes(self.desc)
        ws_bytes = ss.ss_cache_attend_workspace_bytes(self.desc)
        self.tree_desc: Optional[ss.ss_cache_desc] = None
        if tree_rows != 0 and ws_bytes != 0:
            self.tree_desc = ss.make_cache_desc(num_requests, num_kv_heads, fmt, page_tokens, pages, width, num_q_heads,
                                                max_rows=tree_rows, softmax_scale=softmax_scale, causal=causal)
            tree_bytes = ss.ss_cache_attend_tree_workspace_bytes(self.tree_desc)
            ws_bytes = max(ws_bytes, tree_bytes) if tree_bytes else 0
        if page_bytes == 0 or ws_bytes == 0:
            raise ss.SpecStreamError(ss.SS_ERR_INVALID_ARGUMENT, "PagedCache", ss.ss_last_error())
        self.pages = torch.empty(pages, num_kv_heads, page_bytes // num_kv_heads, dtype=torch.uint8, device=device)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        self.table = torch.full((num_requests, width), -1, dtype=torch.int32, device=device)
        self.end = torch.zeros(num_requests, dtype=torch.int32, device=device)
        self.tokens = [0] * num_requests
        self.owned: List[List[int]] = [[] for _ in range(num_requests)]
        self.free = list(range(pages))[::-1]
        self.order = _Order(self.pages.device) if self.pages.is_cuda else None

    def _counts(self, rows: Sequence[int]) -> List[int]:
        rows = [operator.index(n) for n in rows]
        if len(rows) != len(self.tokens) or min(rows) < 0:
            raise ValueError(f"one count of tokens, 0 or more, for each of {len(self.tokens)} requests (got {rows})")
        if self.end.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("grow and release change the host's counts too: they cannot be captured")
        return rows

    def _post(self, rows: List[int], places: List[int], ids: List[int], more: Sequence[int] = (),
              first: Optional[Callable[[torch.Tensor], None]] = None) -> None:
        """``end`` and table entries change on torch's current stream, once ``first`` was called with ``more`` there.
        The numbers travel in one copy from pinned memory, which torch hands out again only once that copy is done, so
        that the host waits for nothing."""
        x = torch.tensor([*more, *rows, *places, *ids], dtype=torch.int32)
        if self.order is not None:
            x = x.pin_memory().to(self.end.device, non_blocking=True)
            self.order.change_begins()
        if first is not None:
            first(x[:len(more)])
        x = x[len(more):]
        n, m = len(rows), len(rows) + len(places)
        if ids:
            self.table.view(-1)[x[n:m]] = x[m:]
        self.end += x[:n]
        if self.order is not None:
            self.order.change_ends()

    def grow(self, rows: Sequence[int]) -> None:
        """Room for rows[b] more tokens of each request; ``end`` then counts them."""
        rows = self._counts(rows)
        need = [-(-(self.tokens[b] + n) // self.desc.page_tokens) for b, n in enumerate(rows)]
        more = [max(0, k - len(self.owned[b])) for b, k in enumerate(need)]
        if max(need) > self.table.shape[1] or sum(more) > len(self.free):
            raise MemoryError("the cache is full")
        places: List[int] = []
        for b, k in enumerate(more):
            at = b * self.table.shape[1] + len(self.owned[b])
            places += range(at, at + k)
        left = len(self.free) - len(places)
        ids = self.free[left:][::-1]
        self._post(rows, places, ids)
        del self.free[left:]
        new = iter(ids)
        for b, n in enumerate(rows):
            self.tokens[b] += n
            self.owned[b] += [next(new) for _ in range(more[b])]

    def release(self, rows: Sequence[int]) -> None:
        """The last rows[b] tokens of each request are rejected: their pages go back."""
        rows = self._counts(rows)
        if any(n > t for n, t in zip(rows, self.tokens)):
            raise ValueError(f"a request holds fewer tokens than it is to release (holds {self.tokens}, releases {rows})")
        self._release(rows)

    def _release(self, rows: List[int], more: Sequence[int] = (), first: Optional[Callable[[torch.Tensor], None]] = None) -> None:
        keep = [-(-(t - n) // self.desc.page_tokens) for n, t in zip(rows, self.tokens)]
        places: List[int] = []
        for b, k in enumerate(keep):
            places += range(b * self.table.shape[1] + k, b * self.table.shape[1] + len(self.owned[b]))
        self._post([-n for n in rows], places, [-1] * len(places), more, first)
        for b, n in enumerate(rows):
            self.tokens[b] -= n
            self.free += self.owned[b][keep[b]:]
            del self.owned[b][keep[b]:]

    def keep(self, kept: Sequence[Sequence[int]], rows: Sequence[int]) -> None:
        """Of request b's last rows[b] tokens, a tree's nodes, those numbered kept[b] stay, in that order, behind the
        history; the others are released.  A change like ``grow`` and ``release``, on torch's current stream."""
        desc = self._tree()
        rows = self._counts(rows)
        paths = [[operator.index(i) for i in path] for path in kept]
        if len(paths) != len(rows):
            raise ValueError(f"one path for each of {len(rows)} requests (got {len(paths)})")
        for path, n, tokens in zip(paths, rows, self.tokens):
            if n > min(tokens, desc.max_rows) or len(path) > n or any(not 0 <= i < n for i in path):
                raise ValueError(f"a path is at most a tree's nodes, a tree at most {desc.max_rows} of a request's tokens "
                                 f"(got {path} of {n} nodes, {tokens} tokens)")
        starts = [0, *itertools.accumulate(rows)]
        total, B = starts[-1], len(rows)
        listed = [i for path, n in zip(paths, rows) for i in path + [-1] * (n - len(path))]

        def move(x: torch.Tensor) -> None:
            ss.ss_cache_keep(desc, self.pages.data_ptr(), self.table.data_ptr(), x[2 * B + 1:].data_ptr(), x.data_ptr(), total,
                             self.end.data_ptr(), x[B:].data_ptr(), torch.cuda.current_stream(self.pages.device).cuda_stream)

        moves = total > 0 and any(path != list(range(len(path))) for path in paths)
        if moves:
            self._on_current_device()
        self._release([n - len(path) for path, n in zip(paths, rows)], [*map(len, paths), *starts, *listed], move if moves else None)

    def _tree(self) -> ss.ss_cache_desc:
        if self.tree_desc is None:
            raise ValueError("a cache made without tree_rows has no trees")
        return self.tree_desc

    def _on_current_device(self) -> None:
        """A call runs on the current device, wherever its addresses lead."""
        device = self.pages.device
        if device.type != "cuda":
            raise ValueError("a cache on the CPU keeps its table only")
        if torch.cuda.current_device() != device.index:
            raise ValueError(f"the cache is on {device}, the current device is {torch.cuda.current_device()}")

    def _begins(self, stream: int, attends: bool) -> Optional["torch.cuda.Stream"]:
        self._on_current_device()
        return None if self.order is None else self.order.call_begins(stream, attends)

    def _counters(self, x: torch.Tensor, n: int, name: str) -> int:
        """Address of an int32 array of n, which the kernels read as it lies."""
        if not isinstance(x, torch.Tensor):
            raise ValueError(f"{name} is a tensor (got {type(x).__name__})")
        if x.dtype != torch.int32 or x.shape != (n,) or not x.is_contiguous() or x.device != self.end.device:
            raise ValueError(f"{name} is a packed int32 [{n}] on {self.end.device} (got {x.dtype} {list(x.shape)} {x.stride()} on {x.device})")
        return x.data_ptr()

    def _starts(self, row_start: Optional[torch.Tensor]) -> Optional[int]:
        return None if row_start is None else self._counters(row_start, len(self.tokens) + 1, "row_start")

    def _row_stride(self, x: torch.Tensor, heads: int) -> int:
        """Elements between the rows [T, heads, 128] of x; 0 (packed) where only one row or none makes it moot."""
        d = self.desc.head_dim
        if x.dtype != torch.bfloat16 or x.dim() != 3 or x.shape[1] != heads or x.shape[2] != d:
            raise ValueError(f"rows are bf16 [T, {heads}, {d}] (got {x.dtype} {list(x.shape)})")
        if x.device != self.pages.device:
            raise ValueError(f"rows are on the cache's device, {self.pages.device} (got {x.device})")
        if x.shape[0] == 0:
            return 0
        if x.stride(2) != 1 or (heads > 1 and x.stride(1) != d):
            raise ValueError(f"a row's {heads} heads of {d} channels lie in one piece (got strides {x.stride()})")
        if x.shape[0] == 1:
            return 0
        if x.stride(0) == 0:
            raise ValueError("rows are not broadcast: an expanded tensor has one row in memory")
        return x.stride(0)

    def write(self, k: torch.Tensor, v: torch.Tensor, stream: int, row_start: Optional[torch.Tensor] = None) -> None:
        """Rows [T, Hkv, 128] of k and v (views of one projection may be strided alike) enter the cache."""
        stride = self._row_stride(k, self.desc.num_kv_heads)
        if v.shape != k.shape or self._row_stride(v, self.desc.num_kv_heads) != stride:
            raise ValueError(f"k and v have one shape and one row stride (got {list(k.shape)} {k.stride()}, {list(v.shape)} {v.stride()})")
        starts = self._starts(row_start)
        on = self._begins(stream, False)
        ss.ss_cache_write(self.desc, self.pages.data_ptr(), self.table.data_ptr(), k.data_ptr(), v.data_ptr(), k.shape[0],
                          self.end.data_ptr(), starts, stride, stream)
        if on is not None:
            self.order.call_ends(on, False)

    def append(self, k: torch.Tensor, v: torch.Tensor, inv_freq: torch.Tensor, stream: int,
               row_start: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, interleaved: int = 0,
               scale: float = 1.0) -> None:
        """Rows enter as in ``write``, K turned by their positions (the tokens' own, or int32 [T]); so do rows q [T, Hq,
        128] into q_out (which may be q).  inv_freq: fp32, one for each of the pairs of channels that turn."""
        stride = self._row_stride(k, self.desc.num_kv_heads)
        if v.shape != k.shape or self._row_stride(v, self.desc.num_kv_heads) != stride:
            raise ValueError(f"k and v have one shape and one row stride (got {list(k.shape)} {k.stride()}, {list(v.shape)} {v.stride()})")
        if (not isinstance(inv_freq, torch.Tensor) or inv_freq.dtype != torch.float32 or inv_freq.dim() != 1
                or not inv_freq.is_contiguous() or inv_freq.device != self.pages.device):
            raise ValueError(f"inv_freq is a packed fp32 tensor on {self.pages.device}")
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out come together")
        q_strides = [0, 0]
        if q is not None:
            q_strides = [self._row_stride(x, self.desc.num_q_heads) for x in (q, q_out)]
            if q.shape != q_out.shape or q.shape[0] != k.shape[0]:
                raise ValueError(f"q and q_out have k's {k.shape[0]} rows (got {list(q.shape)}, {list(q_out.shape)})")
        at = None if positions is None else self._counters(positions, k.shape[0], "positions")
        starts = self._starts(row_start)
        rope = ss.make_rope_desc(2 * inv_freq.numel(), inv_freq.data_ptr(), interleaved, scale)
        on = self._begins(stream, False)
        ss.ss_cache_append(self.desc, self.pages.data_ptr(), self.table.data_ptr(), rope, k.data_ptr(), v.data_ptr(), k.shape[0],
                           self.end.data_ptr(), starts, stride, at, None if q is None else q.data_ptr(),
                           None if q_out is None else q_out.data_ptr(), *q_strides, stream)
        if on is not None:
            self.order.call_ends(on, False)

    def _chunk(self, k: torch.Tensor, v: torch.Tensor, num_rows: int, kv_layout: int) -> None:
        """k and v hold num_rows tokens in the given layout: packed, or the views of one chunk of K and V rows."""
        heads, d = self.desc.num_kv_heads, self.desc.head_dim
        need = num_rows * heads * d
        for x in (k, v):
            if not isinstance(x, torch.Tensor):
                raise ValueError(f"a chunk is a tensor (got {type(x).__name__})")
            if x.dtype != torch.bfloat16 or x.device != self.pages.device:
                raise ValueError(f"a chunk is bf16 on {self.pages.device} (got {x.dtype} on {x.device})")
        if kv_layout != ss.SS_KV_HEAD_MAJOR_KV:
            fits = all(x.is_contiguous() and x.numel() >= need for x in (k, v))
        else:
            packed = zip(k.shape, k.stride(), (2 * d * num_rows, 2 * d, 1))
            rows = k.shape == (heads, num_rows, d) and all(n == 1 or s == want for n, s, want in packed)
            room = k.untyped_storage().nbytes() // BF16_BYTES - k.storage_offset()
            fits = (k.is_contiguous() and k.numel() >= 2 * need or rows and room >= 2 * need) and v.data_ptr() == k.data_ptr() + BF16_BYTES * d
        if not fits:
            raise ValueError(f"a chunk holds {num_rows} rows of {heads} heads in layout {kv_layout} "
                             f"(got {list(k.shape)} {k.stride()}, {list(v.shape)} {v.stride()})")

    def read(self, k: torch.Tensor, v: torch.Tensor, num_rows: int, stream: int, row_start: Optional[torch.Tensor] = None,
             kv_layout: int = ss.SS_KV_TOKEN_MAJOR, end: Optional[torch.Tensor] = None) -> None:
        """The rows that end at ``end`` (the cache's own by default) leave as a bf16 chunk: into k and v, packed tensors of
        num_rows tokens or more, or with SS_KV_HEAD_MAJOR_KV into one [heads, num_rows, 2, 128], v its second rows."""
        self._chunk(k, v, num_rows, kv_layout)
        ends, starts = self._counters(self.end if end is None else end, len(self.tokens), "end"), self._starts(row_start)
        on = self._begins(stream, False)
        ss.ss_cache_read(self.desc, self.pages.data_ptr(), self.table.data_ptr(), k.data_ptr(), v.data_ptr(), num_rows,
                         ends, starts, kv_layout, stream)
        if on is not None:
            self.order.call_ends(on, False)

    def _results(self, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor],
                 prev: Optional[Tuple[torch.Tensor, torch.Tensor]]) -> Tuple[Optional[int], ...]:
        """Addresses of out, lse and prev's, as the attentions take them."""
        for x, shape in ((out, q.shape), (lse, q.shape[:2])) + (((prev[0], q.shape), (prev[1], q.shape[:2])) if prev else ()):
            if x is not None and (x.dtype != torch.float32 or x.shape != shape or not x.is_contiguous() or x.device != q.device):
                raise ValueError(f"out, lse and prev are packed fp32 {list(q.shape)}, {list(q.shape[:2])} on {q.device} "
                                 f"(got {x.dtype} {list(x.shape)} on {x.device})")
        return (out.data_ptr(), None if lse is None else lse.data_ptr(), None if prev is None else prev[0].data_ptr(),
                None if prev is None else prev[1].data_ptr())

    @staticmethod
    def _window(window: int, sinks: int) -> Tuple[int, int]:
        window, sinks = operator.index(window), operator.index(sinks)
        if not 0 <= window < 2 ** 31 or not 0 <= sinks < 2 ** 31 or sinks > 0 and window == 0:
            raise ValueError(f"window and sinks are 0 or more and fit 31 bits, sinks with a window only (got {window}, {sinks})")
        return window, sinks

    def attend(self, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor], stream: int,
               row_start: Optional[torch.Tensor] = None, prev: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
               window: int = 0, sinks: int = 0) -> None:
        """out, lse of rows q [T, Hq, 128], joined with ``prev``'s if given.  window > 0: a row sees the last ``window``
        tokens up to its own, and the request's first ``sinks``."""
        stride = self._row_stride(q, self.desc.num_q_heads)
        to, to_lse, prev_out, prev_lse = self._results(q, out, lse, prev)
        starts = self._starts(row_start)
        window, sinks = self._window(window, sinks)
        on = self._begins(stream, True)
        if window == 0:
            ss.ss_cache_attend(self.desc, self.pages.data_ptr(), self.table.data_ptr(), q.data_ptr(), q.shape[0],
                               self.end.data_ptr(), to, to_lse, starts, prev_out, prev_lse, self.workspace.data_ptr(),
                               self.workspace.numel(), stride, stream)
        else:
            ss.ss_cache_attend_window(self.desc, self.pages.data_ptr(), self.table.data_ptr(), q.data_ptr(), q.shape[0],
                                      self.end.data_ptr(), to, window, sinks, to_lse, starts, prev_out, prev_lse,
                                      self.workspace.data_ptr(), self.workspace.numel(), stride, stream)
        if on is not None:
            self.order.call_ends(on, True)

    def attend_tree(self, q: torch.Tensor, tree: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor], stream: int,
                    row_start: Optional[torch.Tensor] = None, prev: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                    window: int = 0, sinks: int = 0) -> None:
        """out, lse of rows q [T, Hq, 128], each request's last tokens a tree: bit j of tree[row] (int64 or uint64 [T])
        stands for the request's j-th row's token.  The window is one on the tokens before the tree."""
        desc = self._tree()
        stride = self._row_stride(q, self.desc.num_q_heads)
        if (not isinstance(tree, torch.Tensor) or tree.dtype not in (torch.int64, torch.uint64) or tree.shape != q.shape[:1]
                or not tree.is_contiguous() or tree.device != self.pages.device):
            raise ValueError(f"tree is a packed int64 or uint64 [{q.shape[0]}] on {self.pages.device}")
        to, to_lse, prev_out, prev_lse = self._results(q, out, lse, prev)
        starts = self._starts(row_start)
        window, sinks = self._window(window, sinks)
        on = self._begins(stream, True)
        ss.ss_cache_attend_tree(desc, self.pages.data_ptr(), self.table.data_ptr(), q.data_ptr(), q.shape[0], self.end.data_ptr(),
                                tree.data_ptr(), to, to_lse, starts, window, sinks, prev_out, prev_lse,
                                self.workspace.data_ptr(), self.workspace.numel(), stride, stream)
        if on is not None:
            self.order.call_ends(on, True)
