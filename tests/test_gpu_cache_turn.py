"""Rotated appends whose angles reach the header's bound, 2^48, on the GPU (tolerances: see test_gpu_cache_tree)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import tree as ot
from paper_2609_33184_amd import specstream as ss
from test_gpu_cache import Cache, _bits, _ints, _normal
from test_gpu_cache_tree import _close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", (0, 1))
def test_append_largest_angles(interleaved):
    """Positions up to the int32's ends times frequencies of up to 2^16.9."""
    rng = np.random.default_rng(3)
    rows, hq, hkv = 200, 4, 2
    positions = rng.integers(-(1 << 31), 1 << 31, rows)
    positions[:4] = (1 << 31) - 1, -(1 << 31), 1, -1
    freq = torch.from_numpy(np.exp2(rng.uniform(-20, 16.9, 64)).astype(np.float32))
    freq[:2] = 2.0 ** 16.9
    assert np.abs(positions).max() * float(freq.max()) < 2.0 ** 48
    c = Cache(oc.BF16, hkv, 32, [rows])
    q, k, v = _normal(1, rows, hq, 128), _normal(2, rows, hkv, 128), _normal(3, rows, hkv, 128)
    before, out = _bits(q), torch.empty_like(q)
    f, at, start, end = freq.cuda(), _ints(positions), _ints([0, rows]), _ints([rows])
    ss.ss_cache_append(c.desc(num_q_heads=hq, max_rows=rows), *c.at(), ss.make_rope_desc(128, f.data_ptr(), interleaved), k.data_ptr(), v.data_ptr(),
                       rows, end.data_ptr(), start.data_ptr(), 0, at.data_ptr(), q.data_ptr(), out.data_ptr(), 0, 0,
                       torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    _close(_bits(out), ot.turned(before, positions, freq.numpy(), interleaved), 128, interleaved)
    K = oc.parts(c.dev.cpu().numpy(), oc.BF16, 32)[0]
    t = np.arange(rows)
    got = np.ascontiguousarray(K[c.table[0][t // 32], :, t % 32]).view(np.uint16)
    _close(got, ot.turned(_bits(k), positions, freq.numpy(), interleaved), 128, interleaved)
