"""CPU checks of rotary positions, the key/value cache and attention over it: refusals
before any HIP call, the rotation frequencies, and the oracle against plain formulas."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving

PTR = [ctypes.c_void_p(4096 * (i + 1)) for i in range(12)]   # aligned, never dereferenced
ODD = ctypes.c_void_p(4096 + 8)


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def _cache(fa, **o):
    c = dict(struct_size=ctypes.sizeof(fa._lib.Cache), fp8=0, pages=4, heads=2, page_size=16, head_dim=64, k_codes=4096,
             k_scales=8192, v_codes=12288, v_scales=16384)
    c.update(o)
    return fa._lib.Cache(*(c[f] for f, _ in fa._lib.Cache._fields_))


BAD_CACHES = [(dict(struct_size=8), 1), (dict(fp8=2), 1), (dict(pages=0), 1), (dict(heads=0), 1), (dict(page_size=8), 1),
              (dict(page_size=48), 1), (dict(page_size=-16), 1), (dict(head_dim=96), 2), (dict(heads=65536), 2),
              (dict(page_size=1 << 21), 2), (dict(pages=1 << 40), 2), (dict(pages=1 << 62), 2)]
BAD_POINTERS = [dict(k_codes=0), dict(k_scales=4100), dict(v_codes=0), dict(v_scales=4104)]


def test_rotary_refusals(fa):
    f = fa.lib.fp4attn_rotary
    good = dict(x=PTR[0], out=PTR[1], dtype=1, B=1, H=2, N=3, d=64, xs=_strides(0, 64, 128), os=_strides(0, 64, 128),
                pos=PTR[2], ps=0, freq=PTR[3], r=64, m=1.0, i=0, inv=0, stream=None)

    def status(**o):
        return f(*dict(good, **o).values())
    for o in (dict(x=None), dict(out=ODD), dict(dtype=2), dict(B=-1), dict(H=-1), dict(N=-1), dict(d=0), dict(d=72), dict(r=0),
              dict(r=8), dict(r=24), dict(r=80), dict(m=math.inf), dict(m=math.nan), dict(i=2), dict(inv=-1), dict(xs=None),
              dict(xs=_strides(0, 60, 128)), dict(os=_strides(0, 64, -128)), dict(os=_strides(4, 64, 128)), dict(ps=-1),
              dict(pos=ctypes.c_void_p(4100)), dict(freq=None)):
        assert status(**o) == 1, o
    for o in (dict(d=528, r=64), dict(N=(1 << 24) + 1), dict(B=65536), dict(H=65536)):
        assert status(**o) == 2, o
    for o in (dict(B=0), dict(H=0), dict(N=0, x=None)):
        assert status(**o) == 0, o   # no work, no pointer needed


def test_cache_refusals(fa):
    write, read = fa.lib.fp4attn_cache_write, fa.lib.fp4attn_cache_read
    att, size = fa.lib.fp4attn_cache_attention, fa.lib.fp4attn_cache_attention_workspace

    def calls(c):
        return (write(c, PTR[0], PTR[1], 1, 3, 128, 128, PTR[2], None), read(c, PTR[0], 3, PTR[1], PTR[2], 0, None),
                att(c, PTR[0], 2, 4, 256, 2, PTR[1], 3, PTR[2], None, 1, None, 0, 0.1, PTR[3], 0, None, None, 0, None))
    assert calls(None) == (1, 1, 1) and size(None, 4, 2, 3, 1) == -1
    for o, st in BAD_CACHES:
        c = ctypes.byref(_cache(fa, **o))
        assert calls(c) == (st, st, st), o
        assert size(c, 4, 2, 3, 1) == -1, o
    for o in BAD_POINTERS:
        assert calls(ctypes.byref(_cache(fa, **o))) == (1, 1, 1), o
    c = ctypes.byref(_cache(fa))
    for o in ((None, PTR[1], 1, 3, 128, 128, PTR[2]), (PTR[0], ODD, 1, 3, 128, 128, PTR[2]),
              (PTR[0], PTR[1], 2, 3, 128, 128, PTR[2]), (PTR[0], PTR[1], 1, -1, 128, 128, PTR[2]),
              (PTR[0], PTR[1], 1, 3, 132, 128, PTR[2]), (PTR[0], PTR[1], 0, 3, 128, 130, PTR[2]),
              (PTR[0], PTR[1], 1, 3, 128, -128, PTR[2]), (PTR[0], PTR[1], 1, 3, 128, 128, None),
              (PTR[0], PTR[1], 1, 3, 128, 128, ctypes.c_void_p(4100))):
        assert write(c, *o, None) == 1, o
    assert write(c, PTR[0], PTR[1], 1, 1 << 30, 128, 128, PTR[2], None) == 2
    one = ctypes.byref(_cache(fa, heads=1, head_dim=64))
    assert write(one, PTR[0], PTR[1], 1, 1 << 28, 64, 64, PTR[2], None) == 2
    assert write(c, None, None, 1, 0, 128, 128, None, None) == 0
    for o in ((None, 3, PTR[1], PTR[2], 0), (PTR[0], 3, None, PTR[2], 0), (PTR[0], 3, PTR[1], ODD, 0),
              (PTR[0], 3, PTR[1], PTR[2], 5), (PTR[0], -2, PTR[1], PTR[2], 0)):
        assert read(c, *o, None) == 1, o
    assert read(c, None, 0, None, None, 1, None) == 0


def test_cache_attention_refusals(fa):
    f, size = fa.lib.fp4attn_cache_attention, fa.lib.fp4attn_cache_attention_workspace
    good = dict(c=ctypes.byref(_cache(fa)), q=PTR[0], n=2, hq=4, qs=256, B=2, table=PTR[1], pages=3, lengths=PTR[2],
                starts=None, max_q=1, tree=None, words=0, scale=0.1, out=PTR[3], dtype=0, lse=None, work=None, bytes=0, s=None)

    def status(**o):
        return f(*dict(good, **o).values())
    for o in (dict(q=None), dict(q=ODD), dict(n=-1), dict(n=3), dict(hq=0), dict(hq=5), dict(qs=-8), dict(qs=252), dict(B=0),
              dict(table=None), dict(table=ctypes.c_void_p(4098)), dict(pages=0), dict(lengths=None), dict(max_q=0),
              dict(max_q=2), dict(starts=ctypes.c_void_p(4099)), dict(tree=PTR[4], words=0),
              dict(starts=PTR[5], max_q=65, tree=PTR[4], words=1), dict(tree=ctypes.c_void_p(4100), words=1), dict(scale=0.0),
              dict(scale=-1.0), dict(scale=math.nan), dict(out=None), dict(out=ODD), dict(dtype=2),
              dict(lse=ctypes.c_void_p(4097))):
        assert status(**o) == 1, o
    for o in (dict(B=65536, n=65536), dict(pages=(1 << 26) + 1), dict(n=1 << 30, starts=PTR[5], max_q=1),
              dict(starts=PTR[5], max_q=1 << 30)):
        assert status(**o) == 2, o
    assert status(n=0, q=None, out=None) == 0
    # a long table may be cut up, which takes a workspace; the call refuses less than it asks for
    need = size(good["c"], 4, 2, 1000, 1)
    assert need > 0 and size(good["c"], 4, 2, 3, 1) == 0
    assert size(good["c"], 5, 2, 3, 1) == -1 and size(good["c"], 4, 0, 3, 1) == -1
    for o in (dict(work=None, bytes=need), dict(work=PTR[6], bytes=need - 1), dict(work=ODD, bytes=need)):
        assert status(pages=1000, **o) == 1, o


def test_workspace_grows_with_what_it_holds(fa):
    """An accumulator and its state for both ends of at least two ranges of keys."""
    c = ctypes.byref(_cache(fa, heads=8, head_dim=128, page_size=64))
    size = fa.lib.fp4attn_cache_attention_workspace
    for B in (1, 7, 64, 300):
        for hq in (8, 32, 128):
            for max_q in (1, 5, 64):
                for pages in (1, 16, 64, 2048, 1 << 20):
                    n = size(c, hq, B, pages, max_q)
                    assert n >= 0
                    if n:
                        assert 4 * max_q * hq * (128 * 4 + 16) <= n < 1 << 31, (B, hq, max_q, pages, n)


def test_python_refusals_without_a_gpu(fa):
    x, at = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int64)
    cache = fa.kv_cache(2, 4, 16, 64, device="cpu")
    for call in (lambda: fa.rotary(x, at, torch.zeros(32, dtype=torch.float64)), lambda: fa.cache_write(x, x, cache, at),
                 lambda: fa.cache_read(cache, at),
                 lambda: fa.cache_attention(x.bfloat16(), cache, at.int().view(2, 1), at.int())):
        with pytest.raises(ValueError, match="must be a GPU tensor"):
            call()
    for sizes in ((0, 1, 16, 64), (1, 0, 16, 64), (1, 1, 8, 64), (1, 1, 24, 64), (1, 1, 16, 96)):
        with pytest.raises(ValueError):
            fa.kv_cache(*sizes, device="cpu")
    assert [tuple(t.shape) for t in fa.kv_cache(3, 2, 32, 128, fp8=True, device="cpu")] == [
        (3, 2, 32, 128), (3, 2, 32, 4), (3, 2, 4, 16, 8, 8), (3, 2, 4, 4, 8)]


def test_rotary_frequencies(fa):
    def freq(*a, **o):
        f, m = fa.rotary_frequencies(*a, device="cpu", **o)
        assert f.dtype == torch.float64
        return f.numpy(), m
    plain, m = freq(64)
    assert m == 1.0 and np.allclose(plain, [10000.0 ** (-j / 32) for j in range(32)], rtol=1e-15)
    linear, m = freq(64, scaling="linear", factor=8.0)
    assert m == 1.0 and np.allclose(linear, plain / 8, rtol=1e-15)
    ntk, m = freq(64, scaling="ntk", factor=4.0)
    assert m == 1.0 and ntk[0] == 1.0 and math.isclose(ntk[-1], plain[-1] / 4, rel_tol=1e-12)
    assert np.all(np.diff(plain / ntk) > 0)
    yarn, m = freq(128, scaling="yarn", factor=4.0, original_length=4096)
    base = freq(128)[0]
    assert math.isclose(m, 0.1 * math.log(4) + 1)
    turns = 4096 * base / (2 * math.pi)
    ratio = base / yarn
    assert np.all(np.abs(ratio[turns > 40] - 1) < 1e-12) and np.all(np.abs(ratio[turns < 0.8] - 4) < 1e-12)
    assert np.all(np.diff(ratio) >= -1e-12)
    # a factor of 1 mixes f with itself: 1 - m, two products and a sum round, each by 2^-53 of f at most
    same = freq(64, base=5e5, scaling="yarn", factor=1.0, original_length=8192)[0]
    assert np.allclose(same, freq(64, base=5e5)[0], rtol=4 * 2.0 ** -53, atol=0)
    for a, o in (((63,), {}), ((0,), {}), ((64,), dict(base=1.0)), ((64,), dict(scaling="x")), ((64,), dict(factor=0.5)),
                 ((64,), dict(scaling="yarn", factor=2.0)), ((2,), dict(scaling="ntk", factor=2.0)),
                 ((64,), dict(scaling="yarn", original_length=100, fast_turns=1.0, slow_turns=2.0))):
        with pytest.raises(ValueError):
            freq(*a, **o)


def test_oracle_rotation_is_complex_multiplication():
    rng = np.random.default_rng(0)
    x, at, f = rng.standard_normal((2, 3, 5, 40)), rng.integers(0, 1000, (2, 5)), rng.random(8)
    for interleaved in (False, True):
        y = serving.rotary(x, at, f, interleaved, magnitude=0.7)
        z = x[..., 0:16:2] + 1j * x[..., 1:16:2] if interleaved else x[..., :8] + 1j * x[..., 8:16]
        w = 0.7 * z * np.exp(1j * at[:, None, :, None] * f)
        got = y[..., 0:16:2] + 1j * y[..., 1:16:2] if interleaved else y[..., :8] + 1j * y[..., 8:16]
        assert np.allclose(got, w, rtol=1e-13, atol=1e-13) and np.array_equal(y[..., 16:], x[..., 16:])
        back = serving.rotary(y, at, f, interleaved, magnitude=1 / 0.7, inverse=True)
        assert np.allclose(back, x, atol=1e-13)


def test_oracle_attention_and_masks():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 2, 8))
    see = serving.causal_mask(3, 6, 6)
    assert see.sum(1).tolist() == [4, 5, 6] and serving.causal_mask(2, 1, 1).sum(1).tolist() == [0, 1]
    words = np.array([[0b1], [0b10], [0b101]], dtype=np.uint64)
    tree = serving.tree_mask(words, 3, 6, 6)
    assert tree[:, :3].all() and tree[:, 3:].tolist() == [[True, False, False], [False, True, False], [True, False, True]]
    for mask in (see, tree, np.zeros((3, 6), bool)):
        out, lse, spread, size, reach = serving.attention(q, k, v, mask, 0.5)
        for t in range(3):
            for h in range(4):
                z = np.where(mask[t], k[:, h // 2] @ q[t, h] * 0.5, -np.inf)
                if not mask[t].any():
                    assert not out[t, h].any() and lse[t, h] == -np.inf
                    continue
                w = np.exp(z)
                assert np.allclose(out[t, h], w @ v[:, h // 2] / w.sum()) and np.isclose(lse[t, h], np.log(w.sum()))
