"""Rotated heads that would be written over one another are refused, and no others (no GPU: the
calls run in a process that sees no device, where one that is not refused fails to launch)."""
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2608_28099_gb300 as sp
from conftest import ROOT
from paper_2608_28099_gb300 import build_lib

CALLS = """
import sys
sys.path.insert(0, {root!r})
import paper_2608_28099_gb300 as sp
for n, heads, dh, yt, yh in {cases!r}:
    rot = sp.sp_rotary(dh, 2, 0, 1.0, 0x1000)
    try:
        sp.sp_rotate(None, rot, n, 0x2000, 0, sp.SP_F32, heads, 0x10000000, heads * dh, dh, 0x20000000, yt, yh)
        print(0)
    except sp.SpError as e:
        print(e.status)
"""


def answers(cases):
    build_lib.build()
    r = subprocess.run([sys.executable, "-c", CALLS.format(root=ROOT, cases=cases)], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
    assert r.returncode == 0, r.stderr[-500:]
    return [int(x) for x in r.stdout.split()]


def overlap(n, heads, dh, yt, yh):
    at = (np.arange(n)[:, None] * yt + np.arange(heads)[None] * yh).reshape(-1, 1) + np.arange(dh)
    return len(np.unique(at)) < at.size


def test_random_strides():
    rng = np.random.default_rng(1)
    cases = []
    for _ in range(600):
        n, heads, dh = (int(x) for x in rng.integers(1, 8, 3))
        cases.append((n, heads, dh + 1, int(rng.integers(0, 60)), int(rng.integers(0, 60))))
    got = answers(cases)
    assert [g == sp.SP_ERR_INVALID_ARG for g in got] == [overlap(*c) for c in cases]
    assert 100 < sum(overlap(*c) for c in cases) < 500


@pytest.mark.parametrize("case,bad", [
    ((1 << 30, 40, 128, 40 * 128, 128), False), ((1 << 30, 40, 128, 128, 128 << 30), False),  # token- and head-major
    ((2, 2, 128, 128, 128), True), ((1 << 20, 40, 128, 39 * 128, 128), True), ((1 << 20, 40, 128, 128, 127 << 20), True),
    ((1, 1, 128, 0, 0), False), ((5, 1, 128, 128, 0), False), ((1, 5, 128, 0, 128), False)])
def test_layouts(case, bad):
    assert (answers([case])[0] == sp.SP_ERR_INVALID_ARG) == bad
