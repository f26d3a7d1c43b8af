"""How an attention whose lengths a window bounds is cut (tests/cpp/parts_check.cpp), and what it needs of a workspace, on the CPU.

Parts of a request save a few microseconds over shares of all the work, however long; a part is one workgroup's, which a call
waits for alone where one request fills its window and the others do not.  So parts are short, or there are none.
"""
from __future__ import annotations

import os
import random
import shutil
import subprocess

import pytest

from paper_2609_33184_amd import specstream as ss
from test_cache_cpu import _desc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "cpp", "parts_check.cpp")
LONGEST = {0: 20, 1: 10}             # tiles of a part, in the attentions of few rows and of many


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe = tmp_path_factory.mktemp("parts") / "parts_check"
    subprocess.run([cxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT}/paper_2609_33184_amd/csrc", SRC,
                    "-o", str(exe)], check=True, capture_output=True, text=True)

    def run(cases):
        text = "".join(f"{t} {w} {m} {int(a)} {g}\n" for t, w, m, a, g in cases)
        out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True, timeout=60).stdout
        return [int(x) for x in out.split()]

    return run


def test_parts_are_short_or_none(parts):
    rng = random.Random(1)
    cases = [(rng.choice((rng.randint(1, 40), rng.randint(1, 4000), 1 << 25)), rng.choice((1, 8, 63, 64, 128, 512, 4096, 1 << 21)),
              rng.choice((64, 256, 512)), rng.random() < 0.7, rng.randint(0, 1)) for _ in range(4000)]
    cases += [(34, 512, 256, True, 0), (132, 512, 256, True, 0), (36, 128, 256, True, 0), (66, 128, 256, True, 0), (131, 128, 512, True, 1)]
    for (tiles, wholes, most, alike, group), n in zip(cases, parts(cases)):
        if n == 1 and tiles <= (4 if wholes < 64 else 16):
            continue                                  # few tiles: one workgroup, nothing to join
        assert n == 0 or alike and -(-tiles // n) <= LONGEST[group] and (n == 1 or n * wholes <= most and n <= tiles // 4), (tiles, wholes, most, group, n)


def test_windows_of_common_sizes(parts):
    """16 requests of 8 rows on 8 heads in a window of 1024: two parts; 64 of one row there, or in one of 4096: shares; trees of 128
    rows per KV head in one of 1024: four parts, of 4096: shares."""
    assert parts([(36, 128, 256, True, 0), (34, 512, 256, True, 0), (132, 512, 256, True, 0), (36, 128, 512, True, 1), (132, 128, 512, True, 1)]) == [2, 0, 0, 4, 0]


def test_workspace_of_many_rows():
    """From 128 rows per KV head on the states of a block are held: 512 workers' two, with 128 rows of 130 floats each."""
    most = 2 * 512 * 128 * 130 * 4
    sizes = {n: ss.ss_cache_attend_tree_workspace_bytes(_desc(num_requests=16, num_q_heads=64, num_kv_heads=8, max_rows=n, table_stride=1024)) for n in (12, 16, 17, 32, 64)}
    assert sizes[12] == most // 128 * 96 and all(sizes[n] == most for n in (16, 17, 32, 64)), sizes
