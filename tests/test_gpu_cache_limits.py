"""The paged cache's calls at the border of what they accept."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33184_amd import specstream as ss
from test_cache_limits_cpu import MOST_ROWS
from test_gpu_cache import Cache, _bits, _ints

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


@pytest.mark.parametrize("fmt,values", (
    # 1.75 x 2^127 is 448 x 2^119; above it codes are 16 x 2^120 apart, and 248 x 2^120 is half way to 2^128
    (oc.MXFP8, {0x7F60: 0x7F60, 0x7F61: 0x7F60, 0x7F69: 0x7F70, 0x7F77: 0x7F70, 0x7F78: 0x7F80, 0x7F7F: 0x7F80}),
    # 1.5 x 2^127 is 6 x 2^125; above it codes are 2^126 apart, and 3.5 x 2^126 is half way to 2^128
    (oc.MXFP4, {0x7F40: 0x7F40, 0x7F41: 0x7F40, 0x7F5F: 0x7F40, 0x7F60: 0x7F80, 0x7F7F: 0x7F80})), ids=("mxfp8", "mxfp4"))
def test_the_top_of_the_range(fmt, values):
    """The largest bf16 numbers round to 2^128, which reads as an infinity; no other value of the block does."""
    bits = np.zeros((2 * len(values), 1, 128), np.uint16)
    want = bits.copy()
    for t, (x, y) in enumerate(values.items()):
        bits[2 * t, 0, 40], want[2 * t, 0, 40] = x, y
        bits[2 * t, 0, 41], want[2 * t, 0, 41] = 0x7F00, 0x7F00           # 2^127, a code in either step
        bits[2 * t + 1, 0, 127], want[2 * t + 1, 0, 127] = x | 0x8000, y | 0x8000
    k = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    T = len(bits)
    c = Cache(fmt, 1, 16, [T])
    e, rs = _ints([T]), _ints([0, T])
    ss.ss_cache_write(c.desc(), *c.at(), k.data_ptr(), k.data_ptr(), T, e.data_ptr(), rs.data_ptr())
    got = torch.full((2, T, 1, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ss.ss_cache_read(c.desc(), *c.at(), got[0].data_ptr(), got[1].data_ptr(), T, e.data_ptr(), rs.data_ptr())
    torch.cuda.synchronize()
    for x in got:
        assert np.array_equal(_bits(x), want)
    pages = oc.write(c.pages, fmt, 16, c.table, bits, bits, [0, T], [T])
    assert np.array_equal(c.dev.cpu().numpy(), pages)
