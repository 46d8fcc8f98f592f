"""CPU checks of attention over the cache with options: refusals before any HIP call, the workspace, the launch plan of
the shared prefix (csrc/cache_plan.hpp, compiled into a host program), and the oracle's masks and scores by hand."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import serving
from test_serving import PTR, _cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
needs_compiler = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _options(fa, **o):
    opts = fa._lib.AttentionOptions()
    fa.lib.fp4attn_cache_attention_options_init(ctypes.byref(opts))
    assert (opts.struct_size, opts.softcap, opts.slopes, opts.window, opts.prefix, opts.shared) == (40, 0, None, 0, None, 0)
    for k, v in o.items():
        setattr(opts, k, v)
    return ctypes.byref(opts)


def test_refusals(fa):
    f, size = fa.lib.fp4attn_cache_attention_ex, fa.lib.fp4attn_cache_attention_ex_workspace
    c = ctypes.byref(_cache(fa))
    good = dict(c=c, q=PTR[0], n=2, hq=4, qs=256, B=2, table=PTR[1], pages=3, lengths=PTR[2], starts=None, max_q=1, tree=None,
                words=0, scale=0.1, opts=None, out=None, dtype=0, lse=None, work=None, bytes=0, s=None)

    def status(o, **more):
        return f(*dict(good, opts=_options(fa, **o), **more).values())
    for o in (dict(struct_size=12), dict(struct_size=0), dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf),
              dict(softcap=2.0 ** -65), dict(softcap=2.0 ** 65), dict(window=-1), dict(shared=-1), dict(shared=3 * 16 + 1),
              dict(slopes=4098), dict(prefix=4097)):
        assert status(o) == 1 and fa.lib.fp4attn_last_error(), o
        assert size(c, 2, 4, 2, 3, 1, _options(fa, **o)) == -1, o
    assert status(dict(window=(1 << 30) + 1)) == 2
    assert status(dict(softcap=2.0 ** -60), scale=1e30, out=PTR[3]) == 1 and b"finite" in fa.lib.fp4attn_last_error()
    for o in (dict(window=5), dict(slopes=4096), dict(prefix=4096)):
        assert status(o, tree=PTR[4], words=1) == 2, o
    # accepted options come as far as the missing output
    for o in ({}, dict(softcap=2.0 ** -64), dict(softcap=2.0 ** 64), dict(window=1 << 30), dict(shared=48), dict(slopes=4096, prefix=4100)):
        assert status(o) == 1 and b"out" in fa.lib.fp4attn_last_error(), o
    assert f(*dict(good, n=0, opts=_options(fa, softcap=1.0)).values()) == 0


def test_workspace(fa):
    c = ctypes.byref(_cache(fa, heads=8, head_dim=128, page_size=64))
    ex, plain = fa.lib.fp4attn_cache_attention_ex_workspace, fa.lib.fp4attn_cache_attention_workspace
    for B in (1, 7, 64):
        for hq in (8, 32):
            for max_q in (1, 3):
                for pages in (1, 16, 2048):
                    n = B * max_q
                    base = plain(c, hq, B, pages, max_q)
                    assert base == ex(c, n, hq, B, pages, max_q, None) == ex(c, n, hq, B, pages, max_q, _options(fa, softcap=3.0))
                    shared = ex(c, n, hq, B, pages, max_q, _options(fa, shared=64 * pages))
                    # an accumulator and its state for every row of q and each piece of the prefix, where it pays
                    assert shared >= (n * hq * (128 * 4 + 16) if B == 64 and pages == 2048 else 0)
                    if B == 1:
                        assert shared == base
    # a window is a short table
    assert ex(c, 64, 32, 64, 2048, 1, _options(fa, window=200)) < plain(c, 32, 64, 2048, 1)


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "shaped_plan"
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "shaped_plan.cpp"),
                          "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def ask(lines):
        run = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=60)
        assert run.returncode == 0
        return [tuple(map(int, line.split())) for line in run.stdout.splitlines()]
    return ask


@needs_compiler
def test_prefix_plan_covers_rows_and_keys(plans):
    calls = [(H, G, d, n, units * 128) for H in (1, 2, 3, 8, 64, 1000, 65535) for G in (1, 4, 7, 64) for d in (64, 128)
             for n in (1, 2, 5, 16, 64, 300, 4096, 20000) for units in (1, 2, 3, 63, 64, 65, 513, 8192)]
    for c, (tile, row_tiles, pieces, units, ranges, workgroups, rows, fits) in zip(calls, plans(["P %d %d %d %d %d" % c for c in calls])):
        H, G, d, n, keys = c
        assert tile in (16, 32, 128) and (row_tiles - 1) * tile < n * G <= row_tiles * tile, c
        assert 1 <= pieces and (pieces - 1) * units < keys // 128 <= pieces * units, c
        assert rows == n * G * H, c
        if fits:
            assert ranges == row_tiles * pieces and workgroups % 8 == 0 and ranges * H <= workgroups <= 1 << 24, c


@needs_compiler
def test_window_units_cover_every_tile(plans):
    """The units that a row tile's keys touch, from first window's begin to last token's own key, wherever they lie."""
    cases = [(tile, G, window) for tile in (16, 32, 128) for G in (1, 2, 3, 7, 16, 33, 200) for window in (1, 2, 64, 127, 128, 129, 500)]
    got = [u for u, in plans(["W %d %d %d" % c for c in cases])]
    for (tile, G, window), units in zip(cases, got):
        most = 0
        for row0 in range(0, 40 * tile, tile):
            first, last = row0 // G, (row0 + tile - 1) // G
            span = window + last - first   # keys from first + 1 - window to last
            most = max(most, (span + 126) // 128 + 1)
        assert units >= most, (tile, G, window)


def test_oracle_masks_and_scores():
    see = serving.shaped_mask(3, 6, 6, window=2)
    assert see.tolist() == [[j in (p - 1, p) for j in range(6)] for p in (3, 4, 5)]
    see = serving.shaped_mask(3, 6, 6, prefix=5)
    assert see.sum(1).tolist() == [5, 5, 6] and serving.shaped_mask(3, 6, 6, 3, 5).sum(1).tolist() == [4, 3, 3]   # 1-4, 2-4, 3-5
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 2, 8))
    slopes = [0.5, -0.25, 0.0, 1.0]
    see = serving.causal_mask(3, 6, 6)
    out, lse, *_ = serving.shaped_attention(q, k, v, see, 0.5, 2.0, slopes, 6)
    for t in range(3):
        for h in range(4):
            z = np.array([2 * math.tanh(0.25 * float(k[j, h // 2] @ q[t, h])) - slopes[h] * abs(3 + t - j) for j in range(4 + t)])
            w = np.exp(z)
            assert np.allclose(out[t, h], w @ v[:4 + t, h // 2] / w.sum()) and np.isclose(lse[t, h], np.log(w.sum()))
    plain = serving.attention(q, k, v, see, 0.5)
    for x, y in zip(plain, serving.shaped_attention(q, k, v, see, 0.5)):
        assert np.allclose(x, y)


def test_python_refusals_without_a_gpu(fa):
    x, at = torch.zeros(2, 4, 64).bfloat16(), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        fa.cache_attention(x, fa.kv_cache(2, 4, 16, 64, device="cpu"), at.view(2, 1), at, softcap=3.0)
    with pytest.raises(ValueError, match="no gradient"):
        fa.cache_attention(x, None, at, at, slopes=torch.ones(4, requires_grad=True))


# Batches behind a shared prefix with members that end inside it: row tile of the sequences' own pass, head dimensions, new
# tokens, keys, sequences with idle ones, key heads, query heads to each, shared keys (in pages of 16).
INSIDE = [(16, (64, 128), [1] * 16, [2660, 2650, 2400, 1500, 2561, 2600, 0, 200, 2559, 2560, 2570, 5, 2590, 2580, 2660, 2401], 16, 8, 1, 2560),
          (16, (64, 128), [1] * 9, [2690, 2400, 2600, 2560, 3, 2561, 1200, 2650, 2559], 18, 32, 5, 2560),
          (32, (64,), [33, 20, 1, 33, 0, 12, 5], [2660, 2600, 2590, 2500, 0, 1700, 40], 7, 16, 1, 2560),
          (32, (128,), [17, 17, 15, 17, 17, 17, 3, 17, 17, 16], [4180, 4150, 4000, 2050, 4120, 4100, 4099, 4130, 900, 4111], 10, 8, 2, 4096),
          (128, (128,), [33, 30, 33, 9], [2640, 2600, 2500, 2570], 132, 2, 4, 2560),
          (128, (64,), [20, 17, 20, 13], [2640, 2600, 2500, 1000], 88, 8, 5, 2560)]


def _compiled(tmp_path_factory, source):
    exe = tmp_path_factory.mktemp("plan") / "plan"
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", source), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def ask(calls):
        run = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, timeout=60)
        assert run.returncode == 0
        return [tuple(map(int, line.split())) for line in run.stdout.splitlines()]
    return ask


@pytest.fixture(scope="module")
def shared_plans(tmp_path_factory):
    return _compiled(tmp_path_factory, "shared_call_plan.cpp")


@needs_compiler
def test_a_member_inside_a_shared_prefix_is_cut_up(fa, plans):
    """Where a call without the hint cuts sequences up, one with it has room for their pieces beside those of the prefix."""
    c = ctypes.byref(_cache(fa, heads=8, head_dim=128, page_size=64))
    size = fa.lib.fp4attn_cache_attention_ex_workspace
    for B in (8, 16, 24, 48, 96):
        for shared in (16384, 65536):
            for own in (64, 512, 1024):
                pages = (shared + own) // 64
                (_, _, pieces, _, _, _, rows, _), = plans([f"P 8 4 128 {B} {shared}"])
                assert size(c, B, 32, B, pages, 1, None) > 0
                assert size(c, B, 32, B, pages, 1, _options(fa, shared=shared)) > pieces * rows * (128 * 4 + 16), (B, shared, own)


@needs_compiler
def test_shared_call_plans(fa, shared_plans):
    """The own pass: direct ranges for every row tile, others in number and workspace as the kernels take them."""
    rng = np.random.default_rng(5)
    calls = []
    for _ in range(3000):
        B, T, own, shared = (int(np.exp(rng.uniform(0, np.log(m)))) for m in (300, 100, 2500, 100000))
        calls.append((B, int(rng.integers(1, 300)), int(rng.integers(1, 17)), int(rng.choice((64, 128))), int(rng.integers(0, 2)), T,
                      int(rng.integers(1, B * T + 1)), shared + own, shared))
    direct_calls = 0
    for call, (keys, _, pieces, rows, tile, row_tiles, split, ranges, least, fits, direct, units, workgroups, work) in zip(
            calls, shared_plans(calls)):
        B, H, G, d, _, T, n, most, shared = call
        assert keys in (0, shared // 128 * 128) and fits
        assert (row_tiles - 1) * tile < T * G <= row_tiles * tile
        if not direct:
            assert workgroups == -(-ranges * H // 8) * 8 and (split or ranges == B * row_tiles)
            continue
        direct_calls += 1
        others = ranges - direct
        assert keys and not split and direct == B * row_tiles and others >= 2 and units == -(-(most - keys) // 128)
        assert workgroups == -(-direct * H // 8) * 8 + -(-others * H // 8) * 8
        assert work == others * 16 + others * 2 * H * min(tile, T * G) * (d * 4 + 16)
        # a sequence that may end inside the prefix is walked in pieces
        assert least >= 4 and (least - 1) ** 2 * 1.6 < max(-(-most // 128), 16)
    assert direct_calls > 500


@needs_compiler
def test_plans_of_the_batches_with_members_inside(shared_plans):
    for tile, dims, new, keys, B, H, G, shared in INSIDE:
        for d in dims:
            for fp8 in (0, 1):
                most = (-(-max(keys) // 16) + 2) * 16
                (got, _, _, _, own_tile, _, _, _, _, _, direct, _, _, _), = shared_plans([(B, H, G, d, fp8, max(new), sum(new), most, shared)])
                assert (got, own_tile) == (shared, tile) and direct > 0, (tile, d, fp8)


@needs_compiler
def test_a_pass_that_promises_little_is_not_taken(shared_plans):
    """Batches that a pass over their prefix of its own made longer (measured, us with it / without), and ones that it makes shorter."""
    longer = [(7, 2, 2, 128, 0, 1, 7, 16576, 14495), (4, 8, 2, 64, 1, 1, 4, 11840, 10615), (80, 8, 4, 64, 0, 1, 80, 1024, 913),   # 23/14, 21/15, 19/14
              (35, 8, 8, 128, 1, 8, 207, 2368, 1503), (72, 8, 8, 128, 0, 8, 436, 2432, 1700)]                                     # 61/46, 85/67
    shorter = [(64, 8, 4, 128, 0, 1, 64, 9216, 8192), (96, 8, 8, 128, 1, 1, 96, 66048, 65536), (48, 8, 4, 128, 0, 1, 48, 4608, 4096),
               (24, 8, 8, 128, 0, 1, 24, 16896, 16384), (9, 8, 1, 128, 0, 2, 18, 60928, 60843)]                                   # 33/75, 280/1156, 24/36 ..
    assert all(s[0] == 0 for s in shared_plans(longer)) and all(s[0] > 0 for s in shared_plans(shorter))


def test_options_refuse_no_size_that_goes_without_them(fa):
    """A hint and a window choose smaller row tiles for the fewer keys that are left; where tables are huge, more of these than fit."""
    size = fa.lib.fp4attn_cache_attention_ex_workspace
    for B, H, G, T, n, page, pages, shared in ((64, 1, 2, 187, 6797, 128, 1 << 23, (1 << 30) - 639), (50, 1, 2, 326, 3416, 1 << 20, 256, 268432716),
                                               (50, 2, 8, 28, 244, 2048, 1 << 19, (1 << 30) - 586)):
        c = ctypes.byref(_cache(fa, heads=H, head_dim=128, page_size=page))
        plain = size(c, n, H * G, B, pages, T, None)
        assert plain >= 0
        assert size(c, n, H * G, B, pages, T, _options(fa, shared=shared)) == plain
        for window in (1, 300, 1 << 20):
            assert size(c, n, H * G, B, pages, T, _options(fa, window=window)) >= 0, window


# Batches whose own pass takes row tiles of 128 rows behind a pass over their prefix, whole and cut into ranges: new tokens, keys, sequences
# with idle ones, key heads, query heads to each, shared keys, cut (in pages of 16).
WIDE = [([40, 33, 40, 17], [556, 500, 300, 200], 208, 1, 8, 256, False), ([40, 33, 40, 17], [3200, 2600, 1064, 900], 208, 1, 8, 1024, True)]


@needs_compiler
def test_plans_of_wide_row_tiles_behind_a_prefix(shared_plans):
    for new, keys, B, H, G, shared, cut in WIDE:
        for d in (64, 128):
            for fp8 in (0, 1):
                most = (-(-max(keys) // 16) + 2) * 16
                (got, _, _, _, tile, tiles, split, _, _, _, direct, _, _, _), = shared_plans([(B, H, G, d, fp8, max(new), sum(new), most, shared)])
                assert (got, tile, tiles, split, direct) == (shared, 128, 3, int(cut), 0), (d, fp8, cut)


@needs_compiler
def test_a_launch_has_fewer_than_2_to_32_threads(plans, shared_plans):
    """256 to a workgroup; plans at the edge."""
    calls = [(H, 1, 64, (1 << 24) // H * 128 - off, 128) for H in (1, 8, 64, 4096) for off in (0, 1, 127, 128, 300, 128 * 8, 128 * 9)]
    sizes = plans(["P %d %d %d %d %d" % c for c in calls])
    assert all(workgroups < 1 << 24 for *_, workgroups, _, fits in sizes if fits) and any(not s[-1] for s in sizes)
    calls = [(65535, H, 1, 64, 0, 1, 65535, 4096, 4000) for H in (128, 255, 256)]
    assert all(p[12] < 1 << 24 for p in shared_plans(calls) if p[0])
