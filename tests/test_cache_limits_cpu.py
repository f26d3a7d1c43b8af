"""Calls of the paged cache beyond what a launch or a number holds are refused by name, before any device is looked at."""
from __future__ import annotations

import pytest

from paper_2609_33184_amd import specstream as ss
from test_cache_cpu import _attend, _desc, _read, _refused, _write, lib  # noqa: F401

MOST_ROWS = (1 << 28) - 16         # 2^24 - 1 workgroups of 256 threads and 16 rows: below 2^32 threads


@pytest.mark.parametrize("call", (_write, _read))
def test_more_rows_than_a_launch_has_threads(call):
    for rows in (MOST_ROWS + 1, 1 << 28, (1 << 31) - 1):
        _refused(ss.SS_ERR_UNSUPPORTED, "num_rows", call, _desc(), num_rows=rows, row_start=0x7F0000000000)


def test_a_scale_that_does_not_fit_in_base_two():
    """Weights are powers of two: softmax_scale x log2(e) is a float too, so the scale stays below FLT_MAX x ln 2."""
    for scale in (2.4e38, 3.4e38):
        d = _desc(softmax_scale=scale)
        assert ss.ss_cache_attend_workspace_bytes(d) == 0 and "softmax_scale" in ss.ss_last_error()
        _refused(ss.SS_ERR_INVALID_ARGUMENT, "softmax_scale", _attend, d)
    assert ss.ss_cache_attend_workspace_bytes(_desc(softmax_scale=2.3e38)) > 0
