"""What an earlier part of a row brings into the paged cache's attention, and rows whose part is empty or no number.

Only a part whose lse is -inf does not count.  Any other one does, however small its weight: a NaN on either side
reaches the result.  Errors: the text of ``test_gpu_cache``, plus the join's.  Its weights are e^x of a difference
of two lse: a part's is off by 5e-6 at most (what a call without an earlier part is held to), the difference of two
below 16 is rounded by 16 x 2^-24, and expf adds two units of 2^-23, so a weight is off by less than 8e-6 of
itself; times the largest value, 5 among these.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from test_gpu_cache import FORMATS, IDS, Cache, Rows, _normal

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
JOIN = 8e-6 * 5


def _check(r):
    r.check(r._bound() + JOIN)
    again = Rows(r.c, r.hq, r.rows, r.end, causal=r.causal, q=r.q)       # in place
    again.out, again.lse = r.prev[0].clone(), r.prev[1].clone()
    again.prev = (again.out, again.lse)
    again.run()
    torch.cuda.synchronize()
    for a, b in ((again.out, r.out), (again.lse, r.lse)):
        assert np.array_equal(a.cpu().numpy(), b.cpu().numpy(), equal_nan=True)


def _prev(rows, hq, kinds):
    """An earlier part per row: (lse, whether its values are NaN), None for an ordinary one."""
    g = torch.Generator().manual_seed(4)
    out, lse = torch.randn(rows, hq, 128, generator=g), torch.rand(rows, hq, generator=g) * 10 - 2
    for t in range(rows):
        kind = kinds[t % len(kinds)]
        if kind is not None:
            lse[t] = kind[0]
            if kind[1]:
                out[t, :, 5] = NAN
    return out.cuda(), lse.cuda()


# ordinary; nothing came before; no number came before, or in its lse only; a weight that leaves this part's below the
# smallest float, and the other way round
KINDS = (None, (-INF, True), (NAN, True), (NAN, False), (300.0, False), (-300.0, True))


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n,B", ((4, 6, 1), (8, 6, 1), (16, 6, 1), (4, 6, 90)))
def test_no_number_on_either_side(fmt, hq, n, B):
    """Rows of one worker and of several, 12 to 48 per KV head, workgroups and (B copies of the requests) waves alone."""
    end = [300, 290, 0, 64, 64, 3000 if B == 1 else 700, 3000 if B == 1 else 20] * B
    start = np.cumsum([0] + end)
    k, v = _normal(5, int(start[-1]), 2, 128), _normal(6, int(start[-1]), 2, 128)
    for b in range(len(end)):
        if b % 7 in (1, 3):
            k[start[b] + 9, 0, 40] = NAN          # lse NaN, of one head's rows
        if b % 7 in (4, 6):
            v[start[b] + 11, 1, 70] = NAN         # values NaN, lse not
    c = Cache(fmt, 2, 16, end)
    c.fill_tokens(end, 5, k, v)
    rows = [n] * len(end)
    _check(Rows(c, hq, rows, end, causal=0, prev=_prev(sum(rows), hq, KINDS)).run())


@pytest.mark.parametrize("hq,n", ((4, 3), (8, 6), (16, 8)))
@pytest.mark.parametrize("joined", (False, True))
def test_weights_that_are_all_zero(hq, n, joined):
    """Every score of a row is -inf: the row is an empty one, whatever values its tokens have."""
    end = [70, 40, 1500]
    k, v = _normal(5, 1610, 1, 128), _normal(6, 1610, 1, 128)
    k[:, :, 3] = 0.0
    k[70:, :, 3] = -INF
    v[80, 0, 7], v[700, 0, 100], v[1600, 0, 9] = NAN, INF, NAN
    c = Cache(oc.BF16, 1, 16, end)
    c.fill_tokens(end, 5, k, v)
    rows = [n] * 3
    q = _normal(21, 3 * n, hq // 2, 128)
    q[:, :, 3] = 1.0
    r = Rows(c, hq // 2, rows, end, causal=0, q=q, prev=_prev(3 * n, hq // 2, KINDS[:2]) if joined else None).run()
    if joined:
        _check(r)
    else:
        r.check()
        assert (r.out[n:] == 0).all() and (r.lse[n:] == -INF).all()
