"""Attention over the cache with capped scores, biases by distance, windows, prefix masks and a shared prefix,
against the fp64 oracle.

Tolerances: those of plain attention over the cache (test_gpu_serving.py: P's rounding to bf16, 2^-8 of the weighted
mean of |v - o|; sums, the exponential, scores), u = 2^-24, and of a score z with |z| <= high after the cap and a bias of
magnitude `bias`:
* the cap: its argument by 4 u relative; tanh by 3 u near zero (2.6 half steps of the fit as it is evaluated), beyond by at most
  11 u (the exponential's argument 5 u, itself 2 u, the reciprocal 2 u, at |x| = 0.8, where they weigh most); two
  products: 20 u high with all of them;
* the bias: slope log2(e), the distance, its product and the sum, and with a shared prefix the step between the two
  places that distances count from: 8 u (bias + high).
Errors of the scores move the output by twice their sum times the weighted mean of |v|.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import serving
from test_gpu_serving import FORMATS, HALF_STEP, U, Batch, _beside_idle, _f64, _tree
from test_shaped import INSIDE, WIDE

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _values(b, i, heads):
    """K and V [n, heads, d] of a sequence, by the cache's documented layout (test_gpu_serving.py checks it key by key)."""
    (p, off), heads = divmod(b.slots[i], b.page), np.array(list(heads))
    if len(p) == 0:
        return np.zeros((2, 0, len(heads), b.d))
    p, off = p[:, None], off[:, None]
    kc, ks, vc, vs = b.cache
    v = vc[p, heads, off // 8, :, off % 8].reshape(len(p), len(heads), -1)
    return serving.values(kc[p, heads, off], ks[p, heads, off], b.fp8), serving.values(v, vs[p, heads, off // 8, :, off % 8], b.fp8)


def _check(b, out, lse=None, tree=None, softcap=None, slopes=None, window=None, prefix=None, only=None):
    """out [n, Hq, d] and lse against the oracle (of many key heads the first, a middle and the last one)."""
    heads = sorted({0, b.H // 2, b.H - 1}) if b.H > 4 else range(b.H)
    hq = [h * b.G + g for h in heads for g in range(b.G)]
    out_dtype, out, lse = out.dtype, _f64(out[:, hq]), None if lse is None else lse[:, hq]
    slopes = None if slopes is None else _f64(slopes)[hq]
    for i, (t, n) in enumerate(zip(b.new, b.keys)):
        if t == 0 or (only is not None and i not in only):
            continue
        rows = slice(b.starts[i], b.starts[i] + t)
        k, v = _values(b, i, heads)
        if tree is not None:
            see = serving.tree_mask(tree[rows].reshape(t, -1).view(np.uint64), t, n, n)
        else:
            see = serving.shaped_mask(t, n, n, window or 0, 0 if prefix is None else int(prefix[i]))
        o, norm, spread, size, reach, high, bias = serving.shaped_attention(
            _f64(b.q[rows])[:, hq], np.nan_to_num(k), np.nan_to_num(v), see, b.scale, softcap or 0.0, slopes, n)
        e = 2 * ((b.d + 4) * U * reach + 20 * U * high + 8 * U * (bias + high) + (n + 64) * 2 * U + 4 * U)
        tol = 2.0 ** -8 * (1 + 2.0 ** -7) * spread + e[..., None] * size
        tol += HALF_STEP[out_dtype] * (np.abs(o) + tol)
        err = np.abs(out[rows] - o)
        assert np.all(err <= tol), f"sequence {i}: {np.max(err / np.maximum(tol, 1e-300)):.3g} of the tolerance"
        if lse is not None:
            got = _f64(lse[rows])
            assert np.array_equal(np.isneginf(got), np.isneginf(norm)), i
            fin = np.isfinite(norm)
            got, norm, e = got[fin], norm[fin], e[fin]
            assert np.all(np.abs(got - norm) <= e + 4 * U * np.abs(norm) + 8 * U), i


def _gpu(x, dtype):
    return None if x is None else torch.tensor(x, dtype=dtype, device="cuda")


def _run(fa, b, tree=None, softcap=None, slopes=None, window=None, prefix=None, check=True, only=None, **o):
    """One call with the normaliser, checked."""
    slopes, lse = _gpu(slopes, torch.float32), torch.empty((b.q.shape[0], b.H * b.G), device="cuda")
    out = b.call(fa, tree=tree, lse=lse, softcap=softcap, slopes=slopes, window=window, prefix=_gpu(prefix, torch.int32), **o)
    if check:
        _check(b, out, lse, tree, softcap, slopes, window, prefix, only)
    return out, lse


def _slopes(H):
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


# batches that reach every row tile, alone and in a chip full of them, cut and whole
TILINGS = [(2, [1, 1, 1, 1], [517, 33, 1, 0], 0, 1), (16, [1, 1], [1300, 95], 0, 6000), (3, [4, 1, 7], [300, 130, 7], 0, 1),
           (8, [30, 3, 0, 17], [400, 1100, 5, 17], 0, 6000), (3, [130, 5], [700, 260], 512, 1), (20, [9, 11], [900, 1500], 512, 6000)]


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS)
@pytest.mark.parametrize("softcap", [0.25, 3.0, 50.0, 1e6])
def test_softcap(fa, softcap, G, new, keys, idle, width, d, fp8):
    b = Batch(keys, new, 2, G, d, fp8, 32, seed=G + d)
    _beside_idle(b, idle, width)
    _run(fa, b, softcap=softcap)
    if softcap == 3.0 and max(new) > 1:
        tree = _tree(b.new, 3, G)
        _run(fa, b, tree=tree, softcap=softcap)


@pytest.mark.parametrize("d,fp8", [(64, True), (128, False)])
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS[2:5])
@pytest.mark.parametrize("softcap", [2.0 ** -64, 1e-6, 1e-3, 170.0, 2000.0, 2.0 ** 64])
def test_caps_far_from_the_scores(fa, softcap, G, new, keys, idle, width, d, fp8):
    """Caps far below and far above the scores, with queries that are zero (all scores are) among them."""
    b = Batch(keys, new, 2, G, d, fp8, 32, seed=G + d)
    b.q[::2] = 0.0
    _beside_idle(b, idle, width)
    out, _ = _run(fa, b, softcap=softcap)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS)
@pytest.mark.parametrize("kind", ["geometric", "both signs", "with softcap"])
def test_slopes(fa, kind, G, new, keys, idle, width, d, fp8):
    b = Batch(keys, new, 2, G, d, fp8, 16, seed=G + d)
    _beside_idle(b, idle, width)
    slopes = _slopes(2 * G)
    if kind == "both signs":
        slopes = [(-1) ** h * 0.01 * h for h in range(2 * G)]
    _run(fa, b, slopes=slopes, softcap=5.0 if kind == "with softcap" else None)


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS)
@pytest.mark.parametrize("window", [1, 31, 33, 128, 250, 1 << 30])
def test_window(fa, window, G, new, keys, idle, width, d, fp8):
    """Keys behind the window: their pages are gone, those on the window's first page are not numbers."""
    b = Batch(keys, new, 2, G, d, fp8, 16, seed=G + d)
    _beside_idle(b, idle, width)
    for i, (t, n) in enumerate(zip(b.new, b.keys)):
        low = n - t + 1 - window
        if t == 0 or low <= 0:
            continue
        b.table[i, : low // 16] = -1
        for j in range(low // 16 * 16, low):
            p, off = divmod(int(b.slots[i][j]), 16)
            for s, at in zip(b.cache, (off, off, (off // 8, slice(None), off % 8), (off // 8, slice(None), off % 8))):
                s[(p, slice(None)) + (at if isinstance(at, tuple) else (at,))] = 0xFF
    out, _ = _run(fa, b, window=window)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS)
def test_prefix_mask(fa, G, new, keys, idle, width, d, fp8):
    b = Batch(keys, new, 2, G, d, fp8, 16, seed=G + d)
    _beside_idle(b, idle, width)
    for share in (0.0, 0.7, 1.0, 2.0):
        prefix = [int(share * n) - (3 if i % 2 else 0) for i, n in enumerate(b.keys)]
        _run(fa, b, prefix=prefix)
    prefix = [n - t // 2 for t, n in zip(b.new, b.keys)]
    _run(fa, b, prefix=prefix, slopes=_slopes(2 * G), softcap=4.0)
    for window in (1, 40, 300):
        _run(fa, b, prefix=prefix, window=window, slopes=_slopes(2 * G))


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("window", [16, 1000])
def test_long_window_calls(fa, window, d, fp8):
    """Sequences far longer than their window, cut into ranges; single tokens and chunks."""
    for new in ([1, 1, 1], [40, 3, 65]):
        b = Batch([5000, 2100, 300], new, 2, 4, d, fp8, 64, seed=d + window)
        _run(fa, b, window=window)
        _run(fa, b, window=window, softcap=6.0, slopes=_slopes(8))
        assert b.call(fa, window=window, out_dtype=torch.bfloat16).dtype == torch.bfloat16


def test_options_that_change_nothing(fa):
    b = Batch([300, 77, 3], [3, 2, 3], 2, 3, 128, False, 32, seed=1)
    for o in ({}, dict(window=301), dict(window=1 << 30), dict(prefix=[0, -5, 0]), dict(slopes=[0.0] * 6), dict(slopes=[-0.0] * 6)):
        out, lse = _run(fa, b, **o)
        _check(b, out, lse)


def test_odd_lengths(fa):
    """Lengths past the table, below zero and shorter than the new tokens, with every option."""
    b = Batch([192, 150, 130], [2, 2, 3], 2, 3, 128, False, 16, seed=4, spare=0)
    real = list(b.keys)
    k, v = serving.key_values(b.cache, b.slots[0], False)
    for more in (0, 50):
        length = 192 + more
        b.keys[0] = length
        for o in (dict(window=70), dict(slopes=_slopes(6)), dict(prefix=[100, 20, 130], softcap=2.0)):
            out, _ = _run(fa, b, only=(1, 2), **o)
            see = serving.shaped_mask(2, 192, length, o.get("window", 0), o.get("prefix", [0])[0])
            want, _, spread, size, *_ = serving.shaped_attention(_f64(b.q[:2]), k, v, see, b.scale, o.get("softcap", 0.0),
                                                                 o.get("slopes"), length)
            assert np.all(np.abs(_f64(out[:2]) - want) <= 2.0 ** -8 * (1 + 2.0 ** -7) * spread + 2.0 ** -14 * size)
    b.keys = [-5, 1, 130]
    for o in (dict(window=70), dict(slopes=_slopes(6)), dict(softcap=2.0), dict(prefix=[100, 0, 0])):
        out, lse = _run(fa, b, check=False, **o)
        assert not out[:3].any() and torch.isneginf(lse[:3]).all() and torch.isfinite(lse[3:]).all()
    b.keys = real
    _run(fa, b, window=9)


@pytest.mark.parametrize("o", [dict(softcap=2.0), dict(slopes=_slopes(4)), dict(window=30), dict(prefix=[47])])
def test_hidden_values_never_reach_a_row(fa, o):
    """NaN keys and value blocks of keys that a row does not see; rows that see one are NaN (values: in its 32 channels)."""
    for d, fp8 in FORMATS:
        b = Batch([50], [6], 2, 2, d, fp8, 16, seed=9)
        clean, _ = _run(fa, b, **o)

        def at(key):
            return divmod(int(b.slots[0][key]), 16)
        # the last key but one: a value block of head 0; the last: a key block of head 1
        p, off = at(48)
        b.cache[3][p, 0, off // 8, 1, off % 8] = 255
        p, off = at(49)
        b.cache[1][p, 1, off, 0] = 255
        out, _ = _run(fa, b, check=False, **o)
        bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        bad[4:, :2, 32:64] = True
        bad[5:, 2:] = True
        assert torch.equal(~torch.isfinite(out), bad) and torch.equal(out[~bad], clean[~bad])
        if "window" in o:   # the first rows see key 16, the later ones do not
            b = Batch([50], [6], 2, 2, d, fp8, 16, seed=9)
            p, off = at(16)
            b.cache[1][p, 1, off, 0] = b.cache[3][p, 0, off // 8, 1, off % 8] = 255
            out, _ = _run(fa, b, check=False, **o)
            bad.zero_()
            bad[:2, :2, 32:64] = True      # tokens at 44, 45: keys from 15, 16
            bad[:2, 2:] = True
            assert torch.equal(~torch.isfinite(out), bad) and torch.equal(out[~bad], clean[~bad])


# ---------------------------------------------------------------- a shared prefix

def _share(b, shared):
    """Gives every sequence the first `shared` keys of the longest: whole pages in common, the rest copied."""
    first = int(np.argmax(b.keys))
    page = b.page
    for i, n in enumerate(b.keys):
        m = min(n, shared)
        if i == first or m == 0:
            continue
        b.table[i, : m // page] = b.table[first, : m // page]
        j = np.arange(n)
        b.slots[i] = b.table[i][j // page].astype(np.int64) * page + j % page
        for key in range(m // page * page, m):
            (p, off), (r, at) = (divmod(int(b.slots[x][key]), page) for x in (i, first))
            for s in b.cache[:2]:
                s[p, :, off] = s[r, :, at]
            for s in b.cache[2:]:
                s[p, :, off // 8, :, off % 8] = s[r, :, at // 8, :, at % 8]
    return b


def _behind(fa, keys, new, G, d, fp8, page, shared, width=1, tile=None, seed=0):
    """Such a batch with as few key heads as make the call pass over the prefix by itself (and in row tiles of 128 rows,
    where `tile` says so: these need more)."""
    need = -(-max(max(keys), width) // page) + 2
    for H in (1, 2, 4, 8, 16, 32, 64, 128, 256, 512, 1024, 2048):
        c = fa._lib.Cache(ctypes.sizeof(fa._lib.Cache), int(fp8), 4, H, page, d, 0, 0, 0, 0)
        size = [fa.lib.fp4attn_cache_attention_ex_workspace(ctypes.byref(c), sum(new), H * G, len(new), need, max(new), ctypes.byref(
            fa._lib.AttentionOptions(ctypes.sizeof(fa._lib.AttentionOptions), shared=s))) for s in (0, shared)]
        # (the time of a pass over the prefix in row tiles of 128 rows falls below that in 32 rows)
        whole = shared // 128 * 128
        wide = 28 + 75e-6 * -(-sum(new) * G // 128) * H * whole < 18.5 + (20e-6 if d == 64 else 25e-6) * -(-sum(new) * G // 32) * H * whole
        if size[1] > size[0] and (tile is None or wide):
            b = Batch(keys, new, H, G, d, fp8, page, seed=seed)
            return _beside_idle(_share(b, shared), 0, width)
    raise AssertionError("no number of heads gains by the pass")


SHARED = [([1] * 5, [300, 260, 257, 400, 290], 256), ([1] * 5, [700, 0, 650, 610, 680], 600), ([1] * 4, [2000, 1400, 1350, 1333], 1331),
          ([3, 1, 5, 0, 2, 1, 2], [400, 300, 270, 500, 310, 267, 300], 265), ([1] * 6, [129, 130, 128, 200, 131, 140], 128),
          ([9, 7, 8, 9, 1], [900, 800, 790, 830, 778], 777), ([2] * 6, [1500, 40, 1501, 1402, 1450, 1499], 1400),
          ([1] * 70, [200 + i for i in range(70)], 190), ([1] * 6, [260, 256, 257, 255, 1, 258], 256)]


@pytest.mark.parametrize("G,page,width,d,fp8", [(1, 16, 1, 64, False), (4, 64, 1, 128, False), (2, 32, 6000, 128, True),
                                                (3, 256, 1, 64, True), (4, 32, 1, 128, True)])
@pytest.mark.parametrize("new,keys,shared", SHARED)
def test_shared_prefix(fa, new, keys, shared, G, page, width, d, fp8):
    """Sequences behind one prefix, of whole pages or not, beside idle ones and ones that end inside the prefix."""
    b = _behind(fa, keys, new, G, d, fp8, page, shared, width, seed=G + len(new))
    _run(fa, b, shared=shared)
    if G in (1, 4):
        _run(fa, b, shared=shared, softcap=3.0, slopes=_slopes(b.H * G))
        tree = _tree(b.new, 1, G)
        _run(fa, b, tree=tree, shared=shared, softcap=8.0)
        _run(fa, b, shared=shared, prefix=[n - t // 2 for t, n in zip(b.new, b.keys)], slopes=_slopes(b.H * G))
        _run(fa, b, shared=shared, window=200)


@pytest.mark.parametrize("d,fp8", FORMATS)
def test_shared_prefix_of_a_large_batch(fa, d, fp8):
    """Row tiles of 128 rows, single tokens without row starts, and a few of several."""
    b = _behind(fa, [1103 + i % 9 for i in range(32)], [1] * 32, 8, d, fp8, 16, 1100, tile=128, seed=3)
    out, lse = _run(fa, b, shared=1100, starts=False, slopes=_slopes(b.H * 8))
    again, norm = _run(fa, b, shared=1100, starts=False, slopes=_slopes(b.H * 8), check=False)
    assert torch.equal(out, again) and torch.equal(lse, norm)
    if d == 128:
        new = [1 + i % 4 for i in range(24)]
        b = _behind(fa, [1104 + i % 7 + t for i, t in enumerate(new)], new, 4, d, fp8, 32, 1100, tile=128, seed=3)
        _run(fa, b, shared=1100, softcap=4.0)


@pytest.mark.parametrize("d,fp8", FORMATS)
def test_few_keys_in_common(fa, d, fp8):
    """Calls that gain nothing by a pass of its own, with any number of shared keys."""
    b = _share(Batch([300, 290, 40], [1, 2, 1], 2, 4, d, fp8, 16, seed=7), 250)
    want, _ = _run(fa, b)
    for shared in (0, 1, 127, 128, 200, 250):
        out, _ = _run(fa, b, shared=shared)
        assert torch.equal(out, want)


def test_shared_prefix_values(fa):
    """A NaN in the prefix reaches every row that sees it; one behind it its own sequence; queries stay apart."""
    for d, fp8 in FORMATS:
        b = _behind(fa, [400, 300, 290, 261, 300], [1] * 5, 4, d, fp8, 16, 256, seed=2)
        assert b.H >= 2
        clean, _ = _run(fa, b, shared=256)
        p, off = divmod(int(b.slots[0][70]), 16)
        real = b.cache[1][p, 1, off, 0], b.cache[3][p, 0, off // 8, 1, off % 8]
        b.cache[3][p, 0, off // 8, 1, off % 8] = 255
        out, _ = _run(fa, b, check=False, shared=256)
        assert torch.isnan(out[:, :4, 32:64]).all()
        out[:, :4, 32:64] = clean[:, :4, 32:64]
        assert torch.equal(out, clean)
        b.cache[3][p, 0, off // 8, 1, off % 8] = real[1]
        b.cache[1][p, 1, off, 0] = 255
        out, _ = _run(fa, b, check=False, shared=256)
        assert torch.isnan(out[:, 4:8]).all()
        out[:, 4:8] = clean[:, 4:8]
        assert torch.equal(out, clean)
        b.cache[1][p, 1, off, 0] = real[0]
        p, off = divmod(int(b.slots[1][270]), 16)
        b.cache[1][p, 1, off, 0] = 255
        out, _ = _run(fa, b, check=False, shared=256)
        assert torch.isnan(out[1, 4:8]).all()
        out[1, 4:8] = clean[1, 4:8]
        assert torch.equal(out, clean)
        b.cache[1][p, 1, off, 0] = 120
        b.q[2, 3, 5] = float("nan")
        out, _ = _run(fa, b, check=False, shared=256)
        assert torch.isnan(out[2, 3]).all() and torch.isfinite(out[2, :3]).all() and torch.isfinite(out[[0, 1, 3, 4]]).all()


def test_shared_prefix_missing_page(fa):
    """A page of the prefix that is not in the cache: its keys do not exist, for any row."""
    b = _behind(fa, [400, 300, 290, 261, 300], [1] * 5, 2, 128, False, 16, 256, seed=2)
    keep = [s.copy() for s in b.slots]
    b.table[:, 5] = 10 ** 6
    out, lse = _run(fa, b, check=False, shared=256)
    for i, n in enumerate(b.keys):   # the oracle's batch without those keys
        b.slots[i] = np.delete(keep[i], range(80, 96))
        b.keys[i] = n - 16
    _check(b, out, lse)


def test_shared_prefix_rows_of_no_sequence_stay(fa):
    b = _behind(fa, [300, 290, 280, 299], [3, 5, 1, 2], 4, 128, True, 32, 256, seed=6)
    n = sum(b.new)
    b.q = torch.cat((b.q[:2], b.q, torch.full_like(b.q[:3], float("nan"))))
    b.starts += 2
    out, lse = torch.full((n + 5, b.H * 4, 128), 7.0, device="cuda"), torch.full((n + 5, b.H * 4), 7.0, device="cuda")
    assert b.call(fa, out=out, lse=lse, shared=256) is out
    _check(b, out, lse)
    want = out.clone()
    rest = [0, 1, n + 2, n + 3, n + 4]
    assert bool((out[rest] == 7).all() and (lse[rest] == 7).all())
    b.new[1] = 4   # max_q of 4 for five tokens: the last row of the second sequence stays
    out.fill_(7)
    b.call(fa, out=out, shared=256)
    assert bool((out[2 + 3 + 4] == 7).all())
    _check(b, out, only=(0, 2, 3))
    # its other rows: two results (a smaller max_q takes other row tiles), each off by 2^-8 (1 + 2^-7) of the mean of |v - o|, which is
    # at most twice the largest |v|
    most = np.abs(_values(b, 1, range(b.H))[1]).max()
    assert (out[5:9] - want[5:9]).abs().max() <= 2 * 2.0 ** -8 * (1 + 2.0 ** -6) * 2 * most


@pytest.mark.parametrize("o", [dict(window=70), dict(window=1200, softcap=4.0), dict(softcap=2.0, slopes=[0.5, 0.01]),
                               dict(prefix=True), dict(prefix=True, window=300, slopes=[0.02, 0.1])])
@pytest.mark.parametrize("B,H,G,T", [(300, 1, 2, 1), (130, 1, 2, 3)])
def test_many_sequences(fa, B, H, G, T, o):
    """More sequences than a wave has lanes, of very different lengths, some idle, cut and whole."""
    rng = np.random.default_rng(B)
    keys = [int(x) for x in rng.integers(T, 90, B)]
    keys[3], keys[70], keys[B - 1] = 2600, 1500, 1100
    new = [T] * B
    if T > 1:
        new[64] = new[10] = 0
    else:
        keys[64] = keys[10] = 0
    o = dict(o)
    if "prefix" in o:
        o["prefix"] = [n - i % 5 for i, n in enumerate(keys)]
    _run(fa, Batch(keys, new, H, G, 64, False, 32, seed=B), **o)


@pytest.mark.parametrize("starts", [False, True])
def test_the_first_sequences_are_idle(fa, starts):
    """The prefix is taken from the first sequence that is behind it, past the first 64; the table's rows of the others hold
    anything."""
    keys = [0] * 66 + [900, 880, 0, 871, 890, 10]
    b = _behind(fa, keys, [1] * len(keys), 2, 128, False, 16, 860, seed=4)
    b.table[:66] = 10 ** 9
    _run(fa, b, shared=860, starts=starts)
    _run(fa, b, shared=860, starts=starts, slopes=_slopes(b.H * 2), softcap=9.0)


@pytest.mark.parametrize("o", [dict(window=300, softcap=5.0), dict(shared=640)])
def test_long_cache_offsets(fa, o):
    """Pages whose bytes lie past 2^32 of the cache: the bits of a small cache's call."""
    page, d = 128, 128
    small = _behind(fa, [700 + i for i in range(40)], [1] * 40, 2, d, False, page, 640, seed=8)   # with a pass over the prefix
    H = small.H
    pages = (1 << 32) // (H * page * d // 2) + 64
    cache = fa.kv_cache(pages, H, page, d)
    n = small.cache[0].shape[0]
    for big, t in zip(cache, small.cache):
        big[pages - n:] = torch.from_numpy(t).cuda()
    table = torch.from_numpy(np.where(small.table < 0, small.table, small.table + pages - n).astype(np.int32)).cuda()
    lengths = torch.tensor(small.keys, dtype=torch.int32, device="cuda")
    got = fa.cache_attention(small.q.cuda(), cache, table, lengths, **o)
    assert torch.equal(got, small.call(fa, starts=False, **o))
    del cache


def test_graph_replays(fa):
    """Captured calls, each with a workspace of its own, replayed with the program's work between."""
    b = _behind(fa, [3000, 2400, 2500, 2900], [1] * 4, 4, 128, False, 64, 2300, seed=8)
    cache = fa.KVCache(*(torch.from_numpy(t).cuda() for t in b.cache))
    table, lengths = torch.from_numpy(b.table).cuda(), torch.tensor(b.keys, dtype=torch.int32, device="cuda")
    q, slopes = b.q.cuda(), torch.tensor(_slopes(b.H * 4), device="cuda")
    calls = [dict(shared=2300), dict(shared=2300, softcap=4.0, slopes=slopes), dict(window=1500, softcap=4.0)]
    want = [fa.cache_attention(q, cache, table, lengths, **o) for o in calls]
    other = [fa.cache_attention(-q, cache, table, lengths - 50, **o) for o in calls]
    side, graphs, outs = torch.cuda.Stream(), [], []
    side.wait_stream(torch.cuda.current_stream())
    for o in calls:
        graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want[0])
        with torch.cuda.graph(graph, stream=side):
            fa.cache_attention(q, cache, table, lengths, out=out, **o)
        graphs.append(graph), outs.append(out)
    for i in range(6):
        q.copy_(b.q.cuda() * (-1 if i % 2 else 1))
        lengths.copy_(torch.tensor(b.keys, dtype=torch.int32) - (50 if i % 2 else 0))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for out, x, y in zip(outs, want, other):
            assert torch.equal(out, y if i % 2 else x), i
        fa.cache_attention(q, cache, table, lengths, shared=2300).sum().item()


def test_two_streams_at_once(fa):
    """Calls behind prefixes on two streams, many in flight: each call's pieces are its own."""
    batches = [_behind(fa, [1500 + 40 * i for i in range(5)], [1] * 5, 4, 128, fp8, 32, 1400, seed=i) for i, fp8 in enumerate((False, True))]
    calls, want = [], []
    for b in batches:
        a = (b.q.cuda(), fa.KVCache(*(torch.from_numpy(t).cuda() for t in b.cache)), torch.from_numpy(b.table).cuda(),
             torch.tensor(b.keys, dtype=torch.int32, device="cuda"))
        calls.append(a)
        want.append(fa.cache_attention(*a, shared=1400))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(20):
        for a, stream, out in zip(calls, streams, outs):
            with torch.cuda.stream(stream):
                out.append(fa.cache_attention(*a, shared=1400))
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        assert all(torch.equal(x, w) for x in out)


def test_refusals_and_the_python_path(fa, monkeypatch):
    b = _share(Batch([300, 290], [2, 2], 2, 2, 64, False, 16, seed=1), 256)
    tree = np.full(4, 3, dtype=np.int64)
    slopes, prefix = torch.tensor(_slopes(4), device="cuda"), torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    for o, error in ((dict(softcap=0.0), ValueError), (dict(softcap=-1.0), ValueError), (dict(softcap=float("nan")), ValueError),
                     (dict(softcap=float("inf")), fa.Fp4AttnError), (dict(window=0), ValueError), (dict(window=-3), ValueError),
                     (dict(window=2.0), TypeError), (dict(window=(1 << 30) + 1), fa.Fp4AttnError), (dict(window=1 << 70), fa.Fp4AttnError),
                     (dict(slopes=slopes[:3]), ValueError), (dict(slopes=slopes.double()), TypeError), (dict(slopes=slopes.cpu()), ValueError),
                     (dict(slopes=slopes.clone().requires_grad_()), ValueError), (dict(prefix=prefix[:1]), ValueError),
                     (dict(prefix=prefix.long()), TypeError), (dict(shared=-1), fa.Fp4AttnError), (dict(shared=1 << 40), fa.Fp4AttnError),
                     (dict(shared=1.0), TypeError), (dict(shared=b.table.shape[1] * 16 + 1), fa.Fp4AttnError),
                     (dict(tree=tree, window=5), fa.Fp4AttnError), (dict(tree=tree, slopes=slopes), fa.Fp4AttnError),
                     (dict(tree=tree, prefix=prefix), fa.Fp4AttnError)):
        with pytest.raises(error):
            b.call(fa, **o)
    with torch.no_grad():
        b.call(fa, slopes=slopes.clone().requires_grad_())
    calls = (dict(softcap=3.0), dict(slopes=slopes), dict(window=77), dict(prefix=prefix), dict(shared=256), dict(shared=3),
             dict(softcap=3, shared=256, slopes=slopes), dict(tree=tree, softcap=2.0, shared=200))
    native = [b.call(fa, **o) for o in calls]
    from paper_2609_04105_amd import api
    monkeypatch.setattr(api, "_binding", api._NoBinding)
    for o, want in zip(calls, native):
        assert torch.equal(b.call(fa, **o), want)


# ---------------------------------------------------------------- capped scores next to what no row sees

NEAR = 50.0   # a cap of which the scores of these batches stay within 0.6, so that they take its polynomial


def _page_zero_unused(b):
    """Page 0, which is read in the place of pages that are not there, becomes one that no sequence holds."""
    used = {int(p) for s in b.slots for p in np.unique(s // b.page)}
    u = next(p for p in range(b.cache[0].shape[0]) if p not in used)
    if 0 not in used:
        return
    b.table[b.table == 0] = u
    b.slots = [np.where(s < b.page, s + u * b.page, s) for s in b.slots]
    for t in b.cache:
        t[[0, u]] = t[[u, 0]]


def _put(b, slots, code, scale):
    """Keys and values of one code and one scale in the given places of the cache."""
    p, off = np.divmod(np.asarray(slots, dtype=np.int64), b.page)
    for t, x in zip(b.cache[:2], (code, scale)):
        t[p, :, off] = x
    for t, x in zip(b.cache[2:], (code, scale)):
        t[p, :, off // 8, :, off % 8] = x


def _bits(x):
    return x.view(torch.int32)


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,new,keys,idle,width", TILINGS)
@pytest.mark.parametrize("window", [None, 33])
def test_capped_scores_ignore_what_no_row_sees(fa, window, G, new, keys, idle, width, d, fp8):
    """Large finite keys behind a sequence's end, behind its window and on pages that are not there leave every bit; those of
    its last token leave the other tokens'."""
    b = Batch(keys, new, 2, G, d, fp8, 16, seed=G + d)
    _page_zero_unused(b)
    _beside_idle(b, idle, width)
    low = [0 if window is None else max(0, n - t + 1 - window) for t, n in zip(b.new, b.keys)]
    for i, n in enumerate(low):
        b.table[i, : n // 32] = -1   # (half of them, the others stay)
    seen = np.unique(np.concatenate([s[n:] for s, n in zip(b.slots, low)]))
    hidden = np.setdiff1d(np.arange(b.cache[0].shape[0] * 16), seen)
    large = (0x7E if fp8 else 0x77, 140)
    for slopes in (None, _slopes(2 * G)):
        o = dict(softcap=NEAR, window=window, slopes=slopes)
        _put(b, hidden, 0, 0)
        want, norm = _run(fa, b, **o)
        _put(b, hidden, *large)
        out, lse = _run(fa, b, check=False, **o)
        assert torch.equal(_bits(out), _bits(want)) and torch.equal(_bits(lse), _bits(norm))
        saved = [t.copy() for t in b.cache]
        last = [i for i, t in enumerate(b.new) if t > 1]
        _put(b, [b.slots[i][-1] for i in last], *large)
        out, lse = _run(fa, b, check=False, **o)
        rest = torch.ones(len(out), dtype=torch.bool, device="cuda")
        rest[[int(b.starts[i + 1]) - 1 for i in last]] = False
        assert torch.equal(_bits(out[rest]), _bits(want[rest])) and torch.equal(_bits(lse[rest]), _bits(norm[rest]))
        b.cache = saved


@pytest.mark.parametrize("d,fp8", FORMATS)
def test_capped_calls_repeat_after_other_work(fa, d, fp8):
    """Row tiles of 128 rows whose keys end inside a step, in turn with calls that leave large and zero codes in the LDS of
    every compute unit."""
    b = Batch([40, 200, 9, 33], [40, 200, 9, 33], 2, 4, d, fp8, 16, seed=d)
    _beside_idle(b, 512, 1)
    other = Batch([256] * 8, [128] * 8, 16, 4, d, fp8, 16, seed=d)
    want, norm = _run(fa, b, softcap=NEAR)
    for i in range(4):
        for code, scale in ((0x7E if fp8 else 0x77, 140), (0, 0)):
            _put(other, np.concatenate(other.slots), code, scale)
            _run(fa, other, softcap=NEAR, check=False)
            out, lse = _run(fa, b, softcap=NEAR, check=False)
            assert torch.equal(_bits(out), _bits(want)) and torch.equal(_bits(lse), _bits(norm)), i


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("tile", [None, 128])
def test_capped_rows_behind_a_prefix_ignore_idle_ones(fa, tile, d, fp8):
    """Queries of idle places hold anything: the rows beside them keep their bits."""
    n = 32 if tile else 6
    keys = [0 if i % 3 == 1 else 1103 + i % 9 for i in range(n)]
    b = _behind(fa, keys, [1] * n, 8 if tile else 3, d, fp8, 16, 1100, tile=tile, seed=3)
    idle = torch.tensor([i % 3 == 1 for i in range(n)])
    b.q[idle] = 0.0
    want, norm = _run(fa, b, shared=1100, starts=False, softcap=NEAR)
    b.q[idle] = 1e4
    out, lse = _run(fa, b, shared=1100, starts=False, softcap=NEAR, check=False)
    assert torch.equal(_bits(out), _bits(want)) and torch.equal(_bits(lse), _bits(norm))


@pytest.mark.parametrize("softcap", [1e-60, 1e-46, 5e-324, 2.0 ** -65])
def test_caps_below_their_range_are_refused(fa, softcap):
    """Also those that fp32 rounds to zero, which would be no cap."""
    b = Batch([300], [2], 2, 2, 64, False, 16, seed=1)
    with pytest.raises((ValueError, fa.Fp4AttnError), match="2\\^-64"):
        b.call(fa, softcap=softcap)


# ---------------------------------------------------------------- members that end inside a shared prefix

def _inside(case, d, fp8):
    _, _, new, keys, B, H, G, shared = case
    b = _share(Batch(keys, new, H, G, d, fp8, 16, seed=d + len(new)), shared)
    return _beside_idle(b, (B - len(new)) * H, 1), shared


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case,d", [(case, d) for case in INSIDE for d in case[1]])
def test_members_inside_a_long_prefix(fa, case, d, fp8):
    """Their keys are cut up beside the other sequences' row tiles (test_shaped.py has these plans), and the pieces joined in one order."""
    b, shared = _inside(case, d, fp8)
    out, lse = _run(fa, b, shared=shared)
    for _ in range(3):
        again, norm = _run(fa, b, shared=shared, check=False)
        assert torch.equal(again, out) and torch.equal(norm, lse)
    _run(fa, b, shared=shared, softcap=3.0, slopes=_slopes(b.H * b.G))
    if max(b.new) > 1:
        _run(fa, b, tree=_tree(b.new, 1, d), shared=shared, softcap=8.0)
        _run(fa, b, tree=_tree(b.new, 2, d), shared=shared)
    _run(fa, b, shared=shared, prefix=[n - t // 2 for t, n in zip(b.new, b.keys)], slopes=_slopes(b.H * b.G))
    _run(fa, b, shared=shared, prefix=[n // 2 for n in b.keys])


@pytest.mark.parametrize("d,fp8", [(64, True), (128, False)])
def test_no_member_behind_the_prefix(fa, d, fp8):
    """All of them are cut up, of a table as long as the prefix; values that are no numbers reach the rows that see them."""
    case = next(c for c in INSIDE if c[0] == 16)
    b, shared = _inside(case, d, fp8)
    b.keys = [min(n, shared - 1) for n in b.keys]
    b.slots = [s[:n] for s, n in zip(b.slots, b.keys)]
    clean, _ = _run(fa, b, shared=shared)
    p, off = divmod(int(b.slots[3][777]), 16)    # (a key of the third sequence and of all behind as long)
    b.cache[3][p, 0, off // 8, 1, off % 8] = 255
    out, _ = _run(fa, b, shared=shared, check=False)
    bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    bad[[i for i, n in enumerate(b.keys) if n > 777 and b.slots[i][777] == b.slots[3][777]], 0, 32:64] = True
    assert bool(bad.any()) and torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], clean[~bad])


def test_members_inside_on_two_streams_and_in_graphs(fa):
    """Calls at once, each with counts of its own, and captured ones whose lengths change from replay to replay."""
    case = next(c for c in INSIDE if c[0] == 16)
    calls, want = [], []
    for d, fp8 in ((64, True), (128, False)):
        b, shared = _inside(case, d, fp8)
        lengths = torch.tensor(b.keys, dtype=torch.int32, device="cuda")
        a = (b.q.cuda(), fa.KVCache(*(torch.from_numpy(t).cuda() for t in b.cache)), torch.from_numpy(b.table).cuda(), lengths)
        calls.append(a)
        want.append([fa.cache_attention(*a[:3], n, shared=shared) for n in (lengths, (lengths - 300).clamp(min=0))])
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(20):
        for a, stream, out in zip(calls, streams, outs):
            with torch.cuda.stream(stream):
                out.append(fa.cache_attention(*a, shared=shared))
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        assert all(torch.equal(x, w[0]) for x in out)
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for a in calls:
        graph, out = torch.cuda.CUDAGraph(), torch.empty_like(a[0], dtype=torch.float32)
        with torch.cuda.graph(graph, stream=side):
            fa.cache_attention(*a, out=out, shared=shared)
        graphs.append((graph, out))
    for i in range(6):
        for a in calls:
            a[3].copy_((torch.tensor(case[3], dtype=torch.int32) - 300 * (i % 2)).clamp(min=0))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            assert torch.equal(out, w[i % 2]), i
        fa.cache_attention(*calls[0], shared=shared).sum().item()


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("new,keys,B,H,G,shared,cut", WIDE)
def test_wide_row_tiles_behind_a_prefix(fa, new, keys, B, H, G, shared, cut, d, fp8):
    """Row tiles of 128 rows that begin with the pieces of the prefix (test_shaped.py has these plans): ragged new tokens, the last row
    tile of a sequence half in use, a member that does not join."""
    b = _beside_idle(_share(Batch(keys, new, H, G, d, fp8, 16, seed=d), shared), (B - len(new)) * H, 1)
    _run(fa, b, shared=shared)
    _run(fa, b, shared=shared, slopes=_slopes(H * G), softcap=3.0)
    _run(fa, b, shared=shared, prefix=[n - t // 2 for t, n in zip(b.new, b.keys)], slopes=_slopes(H * G))
    _run(fa, b, shared=shared, tree=_tree(b.new, 1, d), softcap=8.0)
    _run(fa, b, shared=shared, tree=_tree(b.new, 2, d))
