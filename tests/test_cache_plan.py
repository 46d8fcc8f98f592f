"""The launch plan of attention over the cache (csrc/cache_plan.hpp) on the CPU: compiled into a
small host program and asked what a call takes."""
import os
import shutil
import subprocess
from collections import namedtuple

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
Plan = namedtuple("Plan", "tile row_tiles tile_rows split ranges min_units fits workgroups workspace")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans(calls) -> a Plan for each (B, heads, query heads a head, d, max_q, max_keys)."""
    exe = tmp_path_factory.mktemp("plan") / "cache_plan"
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror",
                          os.path.join(ROOT, "tests", "cache_plan.cpp"), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def ask(calls):
        run = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True,
                             text=True, timeout=60)
        assert run.returncode == 0
        got = [Plan(*map(int, line.split())) for line in run.stdout.splitlines()]
        assert len(got) == len(calls)
        return got
    return ask


def _calls():
    heads = (*range(1, 70), 96, 128, 200, *range(250, 262), 300, *range(380, 390), 450, *range(508, 518), 640, *range(765, 772),
             *range(1020, 1030), 2048, 5000, 65535)
    for H in heads:
        for d in (64, 128):
            for B in (1, 3, 64, 1000):
                for G, max_q in ((1, 1), (7, 1), (16, 1), (8, 3), (1, 64), (8, 64), (4, 513)):
                    for keys in (16, 1024, 1040, 1600, 2064, 8192, 1 << 20):
                        yield B, H, G, d, max_q, keys


def test_tiles_cover_the_rows(plans):
    calls = list(_calls())
    for c, p in zip(calls, plans(calls)):
        B, H, G, d, max_q, keys = c
        rows = max_q * G
        assert p.tile in (16, 32, 128) and (p.tile > 16) == (rows > 16), c
        assert p.row_tiles == -(-rows // p.tile) and p.tile_rows == min(rows, p.tile), c
        assert p.ranges >= 1 and p.workgroups % 8 == 0 and p.workgroups >= p.ranges * H, c
        if not p.split:
            assert p.ranges == B * p.row_tiles and p.workspace == 0, c


def test_cut_calls_have_a_workspace(plans):
    """A call is cut only into ranges that share a key head's row tiles, two at least, and then has room for the
    records and for both ends of every range: the kernels write them whenever a call is cut."""
    calls = list(_calls())
    cut = 0
    for c, p in zip(calls, plans(calls)):
        B, H, G, d, max_q, keys = c
        if p.split:
            cut += 1
            assert p.ranges >= 2, c
            assert p.workspace >= 16 * p.ranges + 2 * p.ranges * H * p.tile_rows * (4 * d + 16), c
    assert cut > len(calls) // 10
