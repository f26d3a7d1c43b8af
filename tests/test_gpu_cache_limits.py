"""The paged cache's calls at the border of what they accept."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33184_amd import specstream as ss
from test_cache_limits_cpu import MOST_ROWS
from test_gpu_cache import Cache, _ints

pytestmark = pytest.mark.gpu


def test_a_read_of_the_most_rows():
    """Few of which belong to a request: the others are not touched, so the chunk need not hold them."""
    c = Cache(oc.MXFP8, 2, 16, [40, 30])
    c.fill_tokens([40, 30], 5)
    k, v = torch.full((2, 40, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    e, rs = _ints([40, 30]), _ints([0, 20, 35])
    ss.ss_cache_read(c.desc(), *c.at(), k.data_ptr(), v.data_ptr(), MOST_ROWS, e.data_ptr(), rs.data_ptr())
    torch.cuda.synchronize()
    for got, which in ((k, 0), (v, 1)):
        got = got.float().cpu().numpy()
        for b, (lo, hi) in enumerate(((0, 20), (20, 35))):
            want = oc.tokens(c.pages, oc.MXFP8, 16, c.table, b, [40, 30][b])[which].transpose(1, 0, 2)[lo - hi:]
            assert np.array_equal(got[lo:hi], want.astype(np.float32))
        assert (got[35:] == 7).all()
