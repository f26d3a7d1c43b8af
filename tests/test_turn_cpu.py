"""Sine and cosine of a row's turn against 113 bits (tests/cpp/turn_check.cpp), on the CPU.

The header promises a turned value within 2^-34 of its pair's length for angles below 2^48: sine and cosine then are off by
less than that together, a few roundings of 2^-53 beside.
"""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "cpp", "turn_check.cpp")
HEADER = os.path.join(ROOT, "include", "specstream.h")


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("needs g++")
    exe = tmp_path_factory.mktemp("turn") / "turn_check"
    subprocess.run([cxx, "-O2", "-std=gnu++17", f"-I{ROOT}/paper_2609_33184_amd/csrc", SRC, "-o", str(exe)], check=True, capture_output=True, text=True)

    def worst(limit):
        out = subprocess.run([str(exe), str(limit)], check=True, capture_output=True, text=True, timeout=120).stdout
        return float(re.search(r"worst 2\^(-[\d.]+)", out)[1])

    return worst


def test_angles_that_the_header_allows(check):
    """Up to the bound that the header gives."""
    limit, bits = re.search(r"Angles are below 2\^(\d+)", open(HEADER).read()), re.search(r"off by 2\^-(\d+) of the pair's length", open(HEADER).read())
    assert limit and bits and check(int(limit[1])) < -int(bits[1])


def test_angles_of_common_positions(check):
    assert check(31) < -36
