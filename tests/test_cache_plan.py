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
    """plans(calls) -> a Plan for each (B, heads, query heads a head, d, fp8, max_q, max_keys)."""
    exe = tmp_path_factory.mktemp("plan") / "cache_plan"
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror",
                          os.path.join(ROOT, "tests", "cache_plan.cpp"), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def ask(calls):
        run = subprocess.run([str(exe)], input="\n".join(" ".join(str(int(x)) for x in c) for c in calls), capture_output=True,
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
                        yield B, H, G, d, (B + H) % 2 == 0, max_q, keys


def test_tiles_cover_the_rows(plans):
    calls = list(_calls())
    for c, p in zip(calls, plans(calls)):
        B, H, G, d, fp8, max_q, keys = c
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
        B, H, G, d, fp8, max_q, keys = c
        if p.split:
            cut += 1
            assert p.ranges >= 2, c
            assert p.workspace >= 16 * p.ranges + 2 * p.ranges * H * p.tile_rows * (4 * d + 16), c
    assert cut > len(calls) // 10


def test_tile_follows_the_rows_in_use(plans):
    """8 key heads of 8 query heads: the tile measured faster, by 6 % or more, of 32 and 128 rows."""
    points = [(32, 128, False, 4, 1024, 32), (32, 128, False, 4, 4096, 32), (32, 128, False, 8, 1024, 32),
              (32, 128, False, 8, 4096, 32), (32, 128, False, 10, 4096, 32), (32, 128, False, 16, 1024, 128),
              (32, 128, False, 32, 4096, 128), (32, 128, True, 4, 4096, 32), (32, 128, True, 8, 4096, 32),
              (32, 128, True, 16, 4096, 128), (64, 128, False, 3, 4096, 32), (64, 128, False, 4, 4096, 32),
              (64, 128, False, 6, 4096, 32), (64, 128, False, 8, 4096, 32), (64, 128, False, 10, 1024, 128),
              (64, 128, False, 12, 1024, 128), (64, 128, False, 16, 4096, 128), (64, 128, True, 4, 4096, 32),
              (64, 128, True, 8, 4096, 128), (64, 128, True, 12, 4096, 128), (160, 128, False, 4, 2048, 32),
              (160, 128, False, 8, 2048, 32), (160, 128, False, 10, 512, 128), (160, 128, True, 4, 512, 32),
              (160, 128, True, 6, 512, 128), (160, 128, True, 8, 2048, 128), (48, 128, False, 8, 4096, 32),
              (48, 128, True, 8, 1024, 32), (48, 128, True, 12, 4096, 128), (24, 128, False, 16, 8192, 128),
              (16, 128, False, 8, 12288, 32), (16, 128, False, 20, 4096, 32), (64, 64, False, 4, 1024, 32),
              (64, 64, False, 16, 1024, 128), (64, 64, False, 17, 1024, 32), (64, 64, False, 24, 1024, 32),
              (64, 64, False, 32, 1024, 128), (160, 64, False, 8, 512, 32), (160, 64, True, 16, 2048, 128),
              (32, 64, False, 16, 4096, 32), (64, 64, True, 8, 4096, 32), (64, 64, True, 17, 1024, 32)]
    got = plans([(B, 8, 8, d, fp8, tokens, keys) for B, d, fp8, tokens, keys, _ in points])
    for point, p in zip(points, got):
        assert p.tile == point[-1], point


def test_gpu_tables_reach_every_kernel(plans):
    """The batches of the GPU tests that plant hidden values run every kernel of each format, cut and whole."""
    from test_gpu_serving import FULL_TILES, HIDDEN_TOKENS
    for d in (64, 128):
        for fp8 in (False, True):
            seen = set()
            for G, idle in ((2, 0), (5, 0), (20, 0), (20, FULL_TILES)):
                for keys in (256, 6000):
                    p = plans([(1 + -(-idle // 2), 2, G, d, fp8, HIDDEN_TOKENS, keys)])[0]
                    seen.add((p.tile, p.split))
            assert seen == {(t, s) for t in (16, 32, 128) for s in (0, 1)}, (d, fp8)
