"""Rotary positions, the quantized key/value cache and attention over it, against their
fp64 oracle.

Tolerances count roundings.  u = 2^-24 is fp32's half step, 2^-8 bf16's.

Rotary: the angle is off by 2^-26 quarter turns, sine and cosine by 2 ulp, the two products and the
magnitude by one rounding each: (|x_a| + |x_b|) m (2.4e-8 + 6 u) < (|x_a| + |x_b|) m 2^-21,
then the output's half step.

Attention, with w the softmax weights, |q||k| the largest sum of magnitudes of a score:
rounding p to bf16 (relative 2^-8, in numerator and normaliser alike) moves the output by at most
2^-8 sum w |v - o| (1 + 2^-7); scores are off by at most e_z = (d + 4) u |q||k| s, sums over n keys and
their rescalings by (n + 64) 2 u, the exponential by 4 u: relative errors of the weights, hence
twice their sum times sum w |v|; then the output's half step.
"""
import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _f64(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- rotary

def _check_rotary(got, x, positions, freq, dtype, **o):
    want = serving.rotary(x, positions, freq, **o)
    half, m = len(freq), abs(o.get("magnitude", 1.0))
    size = np.abs(x)
    pair = size.copy()
    if o.get("interleaved"):
        s = size[..., 0:2 * half:2] + size[..., 1:2 * half:2]
        pair[..., 0:2 * half:2] = pair[..., 1:2 * half:2] = s
    else:
        s = size[..., :half] + size[..., half:2 * half]
        pair[..., :half] = pair[..., half:2 * half] = s
    tol = pair * m * 2.0 ** -21
    tol[..., 2 * half:] = 0
    tol += (np.abs(want) + tol) * HALF_STEP[dtype]
    err = np.abs(got - want)
    assert np.all(err <= tol), f"worst {np.max(err / np.maximum(tol, 1e-300))} of the tolerance"
    assert np.array_equal(got[..., 2 * half:], x[..., 2 * half:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,H,N,d,r", [(1, 1, 1, 64, 64), (2, 3, 5, 128, 128), (1, 40, 17, 128, 64), (3, 2, 129, 80, 32),
                                       (1, 7, 4, 16, 16), (2, 33, 9, 512, 512), (1, 2, 1030, 96, 48)])
def test_rotary(fa, B, H, N, d, r, interleaved, dtype):
    g = torch.Generator().manual_seed(N + d)
    x = torch.randn((B, H, N, d), generator=g).to(dtype).cuda()
    positions = torch.randint(-5, 1 << 20, (B, N), generator=g)
    freq, _ = fa.rotary_frequencies(r)
    o = dict(interleaved=interleaved, magnitude=1.25)
    got = fa.rotary(x, positions.cuda(), freq, **o)
    _check_rotary(_f64(got), _f64(x), positions.numpy(), _f64(freq), dtype, **o)
    back = fa.rotary(x, positions.cuda(), freq, inverse=True, **o)
    _check_rotary(_f64(back), _f64(x), positions.numpy(), _f64(freq), dtype, inverse=True, **o)
    # one sequence of positions for the whole batch; in place
    shared = fa.rotary(x, positions[0].contiguous().cuda(), freq, **o)
    assert torch.equal(shared[0], got[0])
    y = x.clone()
    assert fa.rotary(y, positions.cuda(), freq, out=y, **o) is y and torch.equal(y, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,H,N,d,r", [(2, 64, 1033, 128, 96), (16, 16, 1030, 64, 32), (1, 40, 835, 512, 512)])
def test_rotary_many_tokens(fa, B, H, N, d, r, dtype):
    """Batches that fill the chip, with the last tokens of a sequence alone; in place, and token-major."""
    g = torch.Generator(device="cuda").manual_seed(N + d)
    x = torch.randn((B, H, N, d), device="cuda", generator=g).to(dtype)
    positions = torch.randint(0, 1 << 20, (B, N), device="cuda", generator=g)
    freq, _ = fa.rotary_frequencies(r)
    for o in (dict(interleaved=False, magnitude=1.25), dict(interleaved=True, magnitude=0.75, inverse=True)):
        got = fa.rotary(x, positions, freq, **o)
        some = slice(0, 2)
        for h in (0, H - 1):
            _check_rotary(_f64(got[some, h:h + 1]), _f64(x[some, h:h + 1]), positions[some].cpu().numpy(), _f64(freq), dtype, **o)
        y = x.clone()
        assert fa.rotary(y, positions, freq, out=y, **o) is y and torch.equal(y, got)
        z = x.transpose(1, 2).contiguous().transpose(1, 2)
        assert torch.equal(fa.rotary(z, positions, freq, **o), got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotary_strides(fa, dtype):
    """Heads of a fused projection, token-major sequences, a head shared by expansion; the
    rest of the output's buffer stays as it was."""
    g = torch.Generator(device="cuda").manual_seed(1)
    freq, _ = fa.rotary_frequencies(128)
    fused = torch.randn((13, 12, 128), device="cuda", generator=g).to(dtype)
    at = torch.arange(100, 113, device="cuda")
    for heads in (slice(0, 8), slice(3, 4), slice(8, 12)):
        x = fused[:, heads]
        want = fa.rotary(x.contiguous(), at, freq)
        assert torch.equal(fa.rotary(x, at, freq), want)
        buf = fused.clone()
        fa.rotary(buf[:, heads], at, freq, out=buf[:, heads])
        assert torch.equal(buf[:, heads], want)
        rest = [i for i in range(12) if i not in range(*heads.indices(12))]
        assert torch.equal(buf[:, rest], fused[:, rest])
    x = torch.randn((2, 9, 5, 128), device="cuda", generator=g).to(dtype).transpose(1, 2)      # [B, H, N, d] of [B, N, H, d]
    at = torch.arange(9, device="cuda")
    assert torch.equal(fa.rotary(x, at, freq), fa.rotary(x.contiguous(), at, freq))
    one = torch.randn((1, 1, 9, 128), device="cuda", generator=g).to(dtype)
    assert torch.equal(fa.rotary(one.expand(2, 5, 9, 128), at, freq), fa.rotary(one, at, freq).expand(2, 5, 9, 128))
    for empty in (torch.empty((0, 4, 128)), torch.empty((2, 0, 3, 128)), torch.empty((2, 3, 0, 128))):
        n = empty.shape[0] if empty.ndim == 3 else empty.shape[2]
        got = fa.rotary(empty.to(dtype).cuda(), torch.zeros(n, dtype=torch.int64, device="cuda"), freq)
        assert got.shape == empty.shape


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient(fa, interleaved):
    """The inverse of a gradient against automatic differentiation of the formula in fp64 and
    against differences of the kernel's own outputs (the map is linear: one step of size 1)."""
    g = torch.Generator().manual_seed(3)
    B, H, N, d, r, m = 2, 2, 7, 64, 48, 0.8
    x, dy = (torch.randn((B, H, N, d), generator=g) for _ in range(2))
    at = torch.randint(0, 100000, (B, N), generator=g)
    freq = fa.rotary_frequencies(r, device="cpu")[0]
    leaf = x.double().requires_grad_()
    t = at.double()[:, None, :, None] * freq
    a, b = (leaf[..., 0:r:2], leaf[..., 1:r:2]) if interleaved else (leaf[..., :r // 2], leaf[..., r // 2:r])
    ya, yb = m * (a * t.cos() - b * t.sin()), m * (a * t.sin() + b * t.cos())
    y = torch.stack((ya, yb), -1).flatten(-2) if interleaved else torch.cat((ya, yb), -1)
    torch.cat((y, leaf[..., r:]), -1).backward(dy.double())
    o = dict(interleaved=interleaved, magnitude=m)
    got = fa.rotary(dy.cuda(), at.cuda(), freq.cuda(), inverse=True, **o)
    _check_rotary(_f64(got), _f64(dy), at.numpy(), freq.numpy(), torch.float32, inverse=True, **o)
    assert np.abs(_f64(got) - leaf.grad.numpy()).max() <= 2.0 ** -20 * 2 * dy.abs().max().item()
    for c in (0, r // 2 - 1, r // 2, r - 1, d - 1):
        step = torch.zeros_like(x)
        step[..., c] = 1.0
        diff = _f64(fa.rotary(step.cuda(), at.cuda(), freq.cuda(), **o))
        want = (diff * _f64(dy)).sum(-1)
        assert np.abs(_f64(got)[..., c] - want).max() <= 2.0 ** -18 * dy.abs().max().item()


def test_rotary_nonfinite_stays_in_its_pair(fa):
    freq, _ = fa.rotary_frequencies(64)
    x = torch.ones((1, 1, 3, 128), device="cuda")
    x[0, 0, 1, 5] = float("nan")
    y = fa.rotary(x, torch.arange(3, device="cuda"), freq)
    bad = torch.isnan(y).nonzero().cpu().tolist()
    assert bad == [[0, 0, 1, 5], [0, 0, 1, 37]]


# ---------------------------------------------------------------- the cache

FORMATS = [(64, False), (64, True), (128, False), (128, True)]


def _numpy(cache):
    return tuple(t.cpu().numpy() for t in cache)


def _special(n, H, d, dtype, g):
    """Normal values with zero, tiny, huge, constant and non-finite blocks among them."""
    x = torch.randn((n, H, d), generator=g)
    x[0, 0, :32] = 0.0
    if n > 5:
        x[1, 0, :32] = -0.0
        x[2, -1, 32:64] = float("inf")
        x[3, 0, :32] = 0.75
        x[3, -1, 5] = float("nan")
        x[4, 0, :32] *= 1e30
        x[5, 0, :32] *= 1e-30
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("n,H,page,pages", [(1, 1, 16, 1), (7, 3, 16, 2), (33, 8, 64, 2), (130, 5, 32, 9), (67, 1, 256, 1)])
def test_cache_write_and_read(fa, n, H, page, pages, d, fp8, dtype):
    """Bytes against the oracle's quantizers (exact), every other byte as it was, and the
    values read back (rounded once)."""
    g = torch.Generator().manual_seed(n * H + d)
    cache = fa.kv_cache(pages, H, page, d, fp8)
    for t in cache:
        t.fill_(0xA5)
    k, v = (_special(n, H, d, dtype, g) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:n]
    slots[::5] = torch.tensor([-1, pages * page, -(1 << 40), 1 << 60])[torch.arange(len(slots[::5])) % 4]   # padding
    if n == 1:
        slots[0] = pages * page - 1
    fa.cache_write(k.cuda(), v.cuda(), cache, slots.cuda())
    got = _numpy(cache)
    want = [np.full(t.shape, 0xA5, dtype=np.uint8) for t in got]
    for x, codes, scales, is_v in ((k, want[0], want[1], False), (v, want[2], want[3], True)):
        c, s = serving.block_quantize(_f64(x), fp8)
        for i, slot in enumerate(slots.tolist()):
            if not 0 <= slot < pages * page:
                continue
            p, off = divmod(slot, page)
            if is_v:
                codes[p, :, off // 8, :, off % 8] = c[i].reshape(H, 16, -1)
                scales[p, :, off // 8, :, off % 8] = s[i]
            else:
                codes[p, :, off], scales[p, :, off] = c[i], s[i]
    for name, a, b in zip(fa.KVCache._fields, got, want):
        assert np.array_equal(a, b), name
    for out_dtype in (torch.float32, torch.bfloat16):
        rk, rv = fa.cache_read(cache, slots.cuda(), out_dtype=out_dtype)
        for r, x in ((rk, k), (rv, v)):
            vals = serving.values(*serving.block_quantize(_f64(x), fp8), fp8)
            vals[[not 0 <= s < pages * page for s in slots.tolist()]] = 0.0
            with np.errstate(over="ignore"):
                want = torch.from_numpy(vals.astype(np.float32)).to(out_dtype)
            same = torch.equal(torch.nan_to_num(r.cpu(), nan=777.0), torch.nan_to_num(want, nan=777.0))
            assert same


def test_cache_write_strides_and_empty(fa):
    g = torch.Generator(device="cuda").manual_seed(2)
    fused = torch.randn((21, 12, 128), device="cuda", generator=g).bfloat16()
    slots = torch.randperm(64, device="cuda", generator=g)[:21]
    a, b = fa.kv_cache(2, 3, 32, 128), fa.kv_cache(2, 3, 32, 128)
    fa.cache_write(fused[:, 6:9], fused[:, 9:], a, slots)
    fa.cache_write(fused[:, 6:9].contiguous(), fused[:, 9:].contiguous(), b, slots)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    fa.cache_write(fused[:0, 6:9], fused[:0, 9:], a, slots[:0])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    k, v = fa.cache_read(a, slots[:0])
    assert k.shape == v.shape == (0, 3, 128)
    # a row of the projection given to every token
    fa.cache_write(fused[:1, 6:9].expand(4, 3, 128), fused[:1, 9:].expand(4, 3, 128), a, slots[:4])
    k, _ = fa.cache_read(a, slots[:4])
    assert all(torch.equal(k[i], k[0]) for i in range(4))


# ---------------------------------------------------------------- attention

class Batch:
    """Sequences over a cache of random bytes in random pages; bytes of places that no sequence holds
    are 0xFF (NaN scales, NaN E4M3 codes)."""

    def __init__(self, keys, new, H, G, d, fp8, page, seed=0, spare=2):
        rng = np.random.default_rng(seed)
        self.keys, self.new, self.H, self.G, self.d, self.fp8, self.page = keys, new, H, G, d, fp8, page
        need = [-(-n // page) for n in keys]
        pages = sum(need) + 2
        order = rng.permutation(pages)
        self.table = np.full((len(keys), max(max(need), 1) + spare), -7, dtype=np.int32)   # unused entries: no page
        self.slots, at = [], 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
            j = np.arange(keys[b])
            self.slots.append(self.table[b][j // page].astype(np.int64) * page + j % page)
        w = d if fp8 else d // 2
        shapes = ((pages, H, page, w), (pages, H, page, d // 32), (pages, H, page // 8, 16, 8, w // 16),
                  (pages, H, page // 8, d // 32, 8))
        self.cache = [np.full(s, 0xFF, dtype=np.uint8) for s in shapes]
        for s in np.concatenate(self.slots) if self.slots else []:
            p, off = divmod(int(s), page)
            kc, vc = (rng.integers(0, 256, (H, w), dtype=np.uint8) for _ in range(2))
            if fp8:   # no NaN, and magnitudes up to 30
                kc, vc = (x & 0xBF for x in (kc, vc))
            self.cache[0][p, :, off] = kc
            self.cache[1][p, :, off] = rng.integers(120, 123, (H, d // 32)) if fp8 else rng.integers(124, 130, (H, d // 32))
            self.cache[2][p, :, off // 8, :, off % 8] = vc.reshape(H, 16, -1)
            self.cache[3][p, :, off // 8, :, off % 8] = rng.integers(122, 128, (H, d // 32))
        n = sum(new)
        self.q = torch.from_numpy(rng.standard_normal((n, H * G, d))).bfloat16()
        self.starts = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        self.scale = d ** -0.5

    def call(self, fa, tree=None, starts=True, **o):
        cache = fa.KVCache(*(torch.from_numpy(t).cuda() for t in self.cache))
        more = dict(q_starts=torch.from_numpy(self.starts).cuda(), max_q=max(self.new)) if starts else {}
        return fa.cache_attention(self.q.cuda(), cache, torch.from_numpy(self.table).cuda(),
                                  torch.tensor(self.keys, dtype=torch.int32).cuda(),
                                  tree=None if tree is None else torch.from_numpy(tree).cuda(), **more, **o)

    def check(self, out, lse=None, tree=None, only=None):
        """out [n, Hq, d] and lse against the oracle (sequences `only`)."""
        out_dtype, out = out.dtype, _f64(out)
        for b, (t, n) in enumerate(zip(self.new, self.keys)):
            if t == 0 or (only is not None and b not in only):
                continue
            rows = slice(self.starts[b], self.starts[b] + t)
            k, v = serving.key_values(self.cache, self.slots[b], self.fp8) if n else np.zeros((2, 0, self.H, self.d))
            see = serving.causal_mask(t, n, n) if tree is None else serving.tree_mask(
                tree[rows].reshape(t, -1).view(np.uint64), t, n, n)
            o, norm, spread, size, reach = serving.attention(_f64(self.q[rows]), k, v, see, self.scale)
            e = 2 * ((self.d + 4) * U * reach + (n + 64) * 2 * U + 4 * U)
            tol = 2.0 ** -8 * (1 + 2.0 ** -7) * spread + e[..., None] * size
            tol += HALF_STEP[out_dtype] * (np.abs(o) + tol)
            err = np.abs(out[rows] - o)
            assert np.all(err <= tol), f"sequence {b}: {np.max(err / np.maximum(tol, 1e-300)):.3g} of the tolerance"
            if lse is not None:
                got = _f64(lse[rows])
                assert np.array_equal(np.isneginf(got), np.isneginf(norm)), b
                fin = np.isfinite(norm)
                got, norm, e = got[fin], norm[fin], e[fin]
                assert np.all(np.abs(got - norm) <= e + 4 * U * np.abs(norm) + 8 * U), b


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,page,keys", [(1, 16, [1, 2, 31, 33, 0]), (4, 64, [517, 64, 32]), (16, 32, [100, 129]),
                                         (7, 16, [47, 48, 49, 17]), (5, 128, [1, 300]), (17, 64, [65, 200]),
                                         (40, 32, [33, 96])])
def test_decode(fa, d, fp8, G, page, keys):
    """Single tokens: sequences that end anywhere in a page and in a tile, an empty one; group
    sizes on either side of the row tiles."""
    b = Batch(keys, [1] * len(keys), 3, G, d, fp8, page, seed=G)
    lse = torch.empty((len(keys), 3 * G), device="cuda")
    out = b.call(fa, starts=False, lse=lse)
    b.check(out, lse)
    b.check(b.call(fa, out_dtype=torch.bfloat16))


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("H,G,keys", [(1, 1, [5000]), (2, 8, [3000, 1, 0, 1025, 1024]), (1, 20, [2500, 64]),
                                      (3, 33, [2100])])
def test_decode_split(fa, d, fp8, H, G, keys):
    """Sequences cut into chunks beside whole and empty ones, every row tiling."""
    b = Batch(keys, [1] * len(keys), H, G, d, fp8, 64, seed=H + G)
    lse = torch.empty((len(keys), H * G), device="cuda")
    out = b.call(fa, lse=lse)
    b.check(out, lse)
    b.check(b.call(fa, out_dtype=torch.bfloat16))


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("new,keys,H,G,page", [([3, 1, 2], [3, 77, 2], 2, 2, 16), ([16, 5, 0, 9], [100, 64, 30, 41], 1, 4, 32),
                                               ([70, 65], [150, 65], 2, 1, 64), ([30], [1600], 1, 8, 128)])
def test_chunks(fa, d, fp8, new, keys, H, G, page):
    """Ragged chunks, causal; a sequence that is all new, one with no new token."""
    b = Batch(keys, new, H, G, d, fp8, page, seed=sum(new))
    lse = torch.empty((sum(new), H * G), device="cuda")
    b.check(b.call(fa, lse=lse), lse)


def _tree(new, words, seed, p_self=0.9):
    """Random ancestors; some tokens see no drafted token at all."""
    rng = np.random.default_rng(seed)
    rows = []
    for t in new:
        seen = []
        for i in range(t):
            up = int(rng.integers(-1, i)) if i else -1
            seen.append(((1 << i) if rng.random() < p_self else 0) | (seen[up] if up >= 0 else 0))
        rows += [[x >> 64 * w & (1 << 64) - 1 for w in range(words)] for x in seen]
    return np.array(rows, dtype=np.uint64).view(np.int64).reshape(len(rows), words)


@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("new,keys,H,G,words", [([8, 3], [200, 3], 2, 4, 1), ([64, 33, 1], [90, 64, 1500], 1, 3, 1),
                                                ([5], [5], 1, 1, 2), ([130, 100], [170, 100], 2, 1, 3)])
def test_trees(fa, d, fp8, new, keys, H, G, words):
    """Trees of drafted tokens, also without a prefix (rows that see no key), of more than
    64 tokens, and shorter than the words given."""
    b = Batch(keys, new, H, G, d, fp8, 32, seed=sum(new))
    tree = _tree(new, words, sum(new))
    lse = torch.empty((sum(new), H * G), device="cuda")
    out = b.call(fa, tree=tree, lse=lse)
    b.check(out, lse, tree=tree)
    if words == 1:
        assert torch.equal(b.call(fa, tree=tree[:, 0].copy()), out)


def test_causal_tree_equals_causal(fa):
    """A chain of drafted tokens sees what causal tokens see: the same bits."""
    b = Batch([300, 90], [20, 11], 2, 4, 128, False, 64, seed=5)
    chain = np.array([(1 << t + 1) - 1 for n in b.new for t in range(n)], dtype=np.uint64).view(np.int64)
    assert torch.equal(b.call(fa, tree=chain), b.call(fa))


@pytest.mark.parametrize("fp8", [False, True])
def test_hidden_values_never_reach_a_row(fa, fp8):
    """NaN keys and NaN and overflowing value blocks of drafted tokens that only some rows see: the
    rows that see them are NaN (value blocks: in their 32 channels), the others exact."""
    b = Batch([50], [6], 2, 2, 128, fp8, 16, seed=9)
    prefix = 44
    # token 1 (child of 0) has a NaN value block 2 of head 0, token 3 (child of the prefix) a NaN key block
    # of head 1, token 4 (child of 0) an overflowing value block 1 of head 1
    tree = np.array([0b1, 0b11, 0b101, 0b1000, 0b10001, 0b100000], dtype=np.int64)

    def at(token):
        return divmod(int(b.slots[0][prefix + token]), 16)

    clean = b.call(fa, tree=tree)
    p, off = at(1)
    b.cache[3][p, 0, off // 8, 2, off % 8] = 255
    p, off = at(3)
    b.cache[1][p, 1, off, 0] = 255
    p, off = at(4)
    b.cache[3][p, 1, off // 8, 1, off % 8] = 254
    out = b.call(fa, tree=tree)
    bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    bad[1, 0:2, 64:96] = True       # head 0: query heads 0, 1
    bad[3, 2:4] = True
    bad[4, 2:4, 32:64] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert torch.equal(out[~bad], clean[~bad])


def test_visible_nonfinite_is_seen(fa):
    """Before the new tokens every row sees a NaN value block (its channels) or key (whole rows)."""
    b = Batch([700, 40], [1, 1], 1, 2, 64, False, 32, seed=2)
    clean = b.call(fa)
    p, off = divmod(int(b.slots[0][70]), 32)
    b.cache[3][p, 0, off // 8, 1, off % 8] = 255
    out = b.call(fa)
    assert torch.isnan(out[0, :, 32:]).all() and torch.equal(out[0, :, :32], clean[0, :, :32])
    assert torch.equal(out[1], clean[1])
    b.cache[1][p, 0, off, 0] = 255
    out = b.call(fa)
    assert torch.isnan(out[0]).all() and torch.equal(out[1], clean[1])
    b.q[1, 1, 3] = float("nan")   # a query: its own row only
    out = b.call(fa)
    assert torch.isnan(out[1, 1]).all() and torch.equal(out[1, 0], clean[1, 0])


@pytest.mark.parametrize("d,fp8", FORMATS)
def test_written_nonfinite_tokens(fa, d, fp8):
    """A token written with a NaN or an infinity: its key block makes every row that sees it NaN, its value
    block their 32 channels; the sequence beside it is untouched."""
    g = torch.Generator(device="cuda").manual_seed(d)
    q = torch.randn((2, 2, d), device="cuda", generator=g).bfloat16()
    k, v = (torch.randn((80, 2, d), device="cuda", generator=g) for _ in range(2))
    table = torch.tensor([[0, 1, 2], [3, 4, 0]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([45, 32], dtype=torch.int32, device="cuda")

    def call(k, v):
        cache = fa.kv_cache(5, 2, 16, d, fp8)
        fa.cache_write(k, v, cache, torch.arange(80, device="cuda"))
        return fa.cache_attention(q, cache, table, lengths)
    clean = call(k, v)
    assert torch.isfinite(clean).all()
    for token in (3, 44):
        for bad in (float("nan"), float("-inf")):
            x = v.clone()
            x[token, 1, 40] = bad
            out = call(k, x)
            assert torch.isnan(out[0, 1, 32:64]).all()
            out[0, 1, 32:64] = clean[0, 1, 32:64]
            assert torch.equal(out, clean)
            x = k.clone()
            x[token, 0, 5] = bad
            out = call(x, v)
            assert torch.isnan(out[0, 0]).all()
            out[0, 0] = clean[0, 0]
            assert torch.equal(out, clean)


@pytest.mark.parametrize("page", [16, 64])
def test_missing_pages_and_odd_lengths(fa, page):
    """Keys in pages outside the cache do not exist; lengths past the table, below zero and shorter
    than the new tokens."""
    b = Batch([192, 150, 130], [2, 2, 3], 2, 3, 128, False, page, seed=4, spare=0)
    keep, real = b.table.copy(), list(b.keys)
    k, v = serving.key_values(b.cache, b.slots[0], False)

    def check_first(out, see):
        o, _, spread, size, _ = serving.attention(_f64(b.q[:2]), k, v, see, b.scale)
        assert np.all(np.abs(_f64(out[:2]) - o) <= 2.0 ** -8 * (1 + 2.0 ** -7) * spread + 2.0 ** -16 * size)
        b.check(out, only=(1, 2))

    for entry in (-1, 10 ** 6, -(1 << 31)):
        b.table = keep.copy()
        b.table[0, 1] = entry
        check_first(b.call(fa), serving.causal_mask(2, 192, 192) & (np.arange(192) // page != 1))
    b.table = keep
    # a length past the table: the new tokens stand behind every key that exists
    assert keep.shape[1] * page == 192
    b.keys[0] = 192 + 1000
    check_first(b.call(fa), np.ones((2, 192), bool))
    b.keys = [-5, 1, 130]
    lse = torch.empty((7, 6), device="cuda")
    out = b.call(fa, lse=lse)
    assert not out[:3].any() and torch.isneginf(lse[:3]).all()      # -5: no key; 1 key for two tokens: the first sees none
    k, v = serving.key_values(b.cache, b.slots[1][:1], False)
    assert np.abs(_f64(out[3]) - np.repeat(v[0], 3, 0)).max() <= 2.0 ** -8 * np.abs(v).max()
    b.keys = real
    b.check(b.call(fa), only=(1, 2))


def test_rows_of_no_sequence_stay(fa):
    """Rows before the first and behind the last sequence, and past max_q."""
    b = Batch([40, 90], [3, 5], 1, 4, 128, True, 32, seed=6)
    want = b.call(fa)
    b.q = torch.cat((b.q[:2], b.q, b.q[:3]))
    b.starts += 2
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((13, 4, 128), 7.0, device="cuda", dtype=dtype)
        lse = torch.full((13, 4), 7.0, device="cuda")
        assert b.call(fa, out=out, lse=lse) is out
        assert torch.equal(out[2:10], want.to(dtype))
        assert bool((out[:2] == 7).all() and (out[10:] == 7).all() and (lse[:2] == 7).all() and (lse[10:] == 7).all())
        assert bool((lse[2:10] != 7).all())
    b.new = [3, 4]   # max_q of 4 for five tokens: the last row stays
    out.fill_(7)
    b.call(fa, out=out)
    assert torch.equal(out[2:9], want[:7].to(dtype)) and bool((out[9] == 7).all())
    b.starts = np.array([2, 5, 1000], dtype=np.int32)   # past the rows: cut at n, and no row outside is written
    b.new = [3, 8]
    out.fill_(7)
    b.call(fa, out=out)
    assert bool((out[:2] == 7).all()) and torch.equal(out[2:5], want[:3].to(dtype))


def _beside_idle(b, tiles, width):
    """The batch with enough idle sequences behind it that `tiles` row tiles are exceeded, and a page table
    for `width` keys."""
    idle = -(-tiles // b.H)
    b.keys, b.new = list(b.keys) + [0] * idle, list(b.new) + [0] * idle
    b.slots += [np.zeros(0, dtype=np.int64)] * idle
    table = np.full((len(b.keys), max(-(-width // b.page), b.table.shape[1])), -7, dtype=np.int32)
    table[:b.table.shape[0], :b.table.shape[1]] = b.table
    b.table = table
    b.starts = np.concatenate((b.starts, np.full(idle, b.starts[-1]))).astype(np.int32)
    return b


@pytest.mark.parametrize("width", [1, 6000])
@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("new,keys,H,G,page", [([1, 1, 1], [77, 0, 1300], 2, 33, 16), ([70, 0, 65], [150, 90, 65], 1, 2, 64),
                                               ([130, 3], [1000, 3], 1, 3, 32), ([16], [1990], 3, 8, 128)])
def test_many_row_tiles(fa, d, fp8, new, keys, H, G, page, width):
    """More than 32 rows in a batch that fills the chip with row tiles, causal and with trees, with
    short page tables and with long ones."""
    b = _beside_idle(Batch(keys, new, H, G, d, fp8, page, seed=sum(new)), 512, width)
    lse = torch.empty((sum(new), H * G), device="cuda")
    b.check(b.call(fa, lse=lse), lse)
    b.check(b.call(fa, out_dtype=torch.bfloat16))
    tree = _tree(b.new, 3, sum(new))
    b.check(b.call(fa, tree=tree, lse=lse), lse, tree=tree)


@pytest.mark.parametrize("width", [1, 6000])
@pytest.mark.parametrize("d,fp8", FORMATS)
@pytest.mark.parametrize("G,idle", [(2, 0), (5, 0), (20, 0), (20, 512)])
def test_hidden_and_missing_in_every_tiling(fa, d, fp8, G, idle, width):
    """NaN keys, NaN and overflowing value blocks that some drafted tokens see, and a page outside the
    cache, in row tiles of every size."""
    b = Batch([190], [6], 2, G, d, fp8, 16, seed=9)
    if idle or width > 1:
        _beside_idle(b, idle, width)
    prefix = 184
    tree = np.array([0b1, 0b11, 0b101, 0b1000, 0b10001, 0b100000], dtype=np.int64)
    clean = b.call(fa, tree=tree)
    b.check(clean, tree=tree)

    def at(token):
        return divmod(int(b.slots[0][prefix + token]), 16)

    p, off = at(1)
    b.cache[3][p, 0, off // 8, 1, off % 8] = 255
    p, off = at(3)
    b.cache[1][p, 1, off, 0] = 255
    p, off = at(4)
    b.cache[3][p, 1, off // 8, 0, off % 8] = 254
    lse = torch.empty((6, 2 * G), device="cuda")
    out = b.call(fa, tree=tree, lse=lse)
    bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    bad[1, :G, 32:64] = True
    bad[3, G:] = True
    bad[4, G:, :32] = True
    assert torch.equal(~torch.isfinite(out), bad)
    nan = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
    nan[3, G:] = True   # (values are not in the normaliser)
    assert torch.equal(torch.isnan(lse), nan) and bool(torch.isfinite(lse[~nan]).all())
    assert torch.equal(out[~bad], clean[~bad])
    # the page of keys 48 .. 63 is missing; the bad tokens are still seen
    real = b.table[0, 3]
    b.table[0, 3] = 10 ** 6
    out = b.call(fa, tree=tree)
    assert torch.equal(~torch.isfinite(out), bad)
    k, v = serving.key_values(b.cache, b.slots[0], fp8)
    see = serving.tree_mask(tree.reshape(6, 1).view(np.uint64), 6, 190, 190) & (np.arange(190) // 16 != 3)
    rows = np.array([0, 2, 5])
    o, _, spread, size, reach = serving.attention(_f64(b.q[rows]), k, np.nan_to_num(v, posinf=0.0, neginf=0.0), see[rows], b.scale)
    e = 2 * ((d + 4) * U * reach + (190 + 64) * 2 * U + 4 * U)
    tol = 2.0 ** -8 * (1 + 2.0 ** -7) * spread + e[..., None] * size + U * np.abs(o)
    assert np.all(np.abs(_f64(out[rows]) - o) <= tol)
    b.table[0, 3] = real
    assert torch.equal(b.call(fa, tree=tree)[~bad], clean[~bad])


@pytest.mark.parametrize("split", [False, True])
def test_long_cache_offsets(fa, split):
    """Pages whose bytes lie past 2^32 of the cache."""
    page, H, d = 128, 8, 128
    pages = (1 << 32) // (H * page * d // 2) + 64
    keys = 4000 if split else 700
    small = Batch([keys], [1], H, 2, d, False, page, seed=8)
    cache = fa.kv_cache(pages, H, page, d)
    n = small.cache[0].shape[0]
    for big, t in zip(cache, small.cache):
        big[pages - n:] = torch.from_numpy(t).cuda()
    table = torch.from_numpy(np.where(small.table < 0, small.table, small.table + pages - n).astype(np.int32)).cuda()
    lengths = torch.tensor([keys], dtype=torch.int32, device="cuda")
    got = fa.cache_attention(small.q.cuda(), cache, table, lengths)
    assert torch.equal(got, small.call(fa))
    slots = torch.from_numpy(small.slots[0] + (pages - n) * page).cuda()
    k, v = fa.cache_read(cache, slots)
    wk, wv = serving.key_values(small.cache, small.slots[0], False)
    assert np.array_equal(_f64(k), wk.astype(np.float32)) and np.array_equal(_f64(v), wv.astype(np.float32))
    fresh = torch.randn((5, H, d), device="cuda")
    fa.cache_write(fresh, fresh, cache, slots[-5:])
    k, v = fa.cache_read(cache, slots[-5:])
    want = serving.values(*serving.block_quantize(_f64(fresh), False), False).astype(np.float32)
    assert np.array_equal(_f64(k), want) and np.array_equal(_f64(v), want)
    del cache


@pytest.mark.parametrize("B,H,G,T", [(300, 1, 2, 1), (130, 2, 1, 3)])
def test_many_sequences(fa, B, H, G, T):
    """More sequences than a wave has lanes, of very different lengths, some idle."""
    rng = np.random.default_rng(B)
    keys = [int(x) for x in rng.integers(T, 90, B)]
    keys[3], keys[70], keys[B - 1] = 2600, 1500, 1100
    new = [T] * B
    if T > 1:
        new[64] = new[10] = 0
    else:
        keys[64] = keys[10] = 0
    b = Batch(keys, new, H, G, 64, False, 32, seed=B)
    lse = torch.empty((sum(new), H * G), device="cuda")
    b.check(b.call(fa, lse=lse), lse)


def test_strided_queries_and_empty(fa):
    b = Batch([100, 60], [2, 2], 2, 3, 128, False, 32, seed=1)
    want = b.call(fa)
    fused = torch.randn((4, 10, 128)).bfloat16()
    fused[:, :6] = b.q
    b.q = fused[:, :6]
    cache = fa.KVCache(*(torch.from_numpy(t).cuda() for t in b.cache))
    args = (torch.from_numpy(b.table).cuda(), torch.tensor(b.keys, dtype=torch.int32).cuda())
    assert torch.equal(fa.cache_attention(fused.cuda()[:, :6], cache, *args), want)
    out = fa.cache_attention(fused.cuda()[:0, :6], cache, *args)
    assert out.shape == (0, 6, 128)
    one = fused.cuda()[:1, :6].expand(4, 6, 128)
    assert torch.equal(fa.cache_attention(one, cache, *args), fa.cache_attention(one.contiguous(), cache, *args))


def _step(fa, s):
    """One decode step: rotary on queries and keys in place, the new keys and values into the
    cache, attention."""
    fa.rotary(s["qkv"][:, :6], s["at"], s["freq"], out=s["turned"][:, :6])
    fa.cache_write(s["turned"][:, 4:6], s["qkv"][:, 6:8], s["cache"], s["slots"])
    return fa.cache_attention(s["turned"][:, :4], s["cache"], s["table"], s["lengths"])


def _decode_state(fa, fp8, seed=0, B=3, page=16, steps=40):
    """Sequences that grow a token at a time: 4 query heads, 2 key heads, d 128, fused projection."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-(steps + 1) // page)
    table = torch.randperm(B * width, device="cuda", generator=g).int().view(B, width)
    return dict(cache=fa.kv_cache(B * width, 2, page, 128, fp8), table=table, freq=fa.rotary_frequencies(128)[0],
                qkv=torch.empty((B, 8, 128), dtype=torch.bfloat16, device="cuda"),
                turned=torch.empty((B, 8, 128), dtype=torch.bfloat16, device="cuda"),
                lengths=torch.zeros(B, dtype=torch.int32, device="cuda"), slots=torch.zeros(B, dtype=torch.int64, device="cuda"),
                at=torch.zeros(B, dtype=torch.int64, device="cuda"), g=g, page=page)


def _next(s, i):
    """New projections and the place of token i of every sequence."""
    s["qkv"].copy_(torch.randn(s["qkv"].shape, device="cuda", generator=s["g"]))
    s["at"].fill_(i)
    s["slots"].copy_(s["table"][:, i // s["page"]].long() * s["page"] + i % s["page"])
    s["lengths"].fill_(i + 1)


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_steps_together(fa, fp8):
    """A cache filled token by token through rotary, cache_write and cache_attention, each step
    against the oracle on the rounded keys that the step stored."""
    s = _decode_state(fa, fp8)
    keys, values = [], []
    for i in range(40):
        _next(s, i)
        out = _step(fa, s)
        x, t = _f64(s["qkv"]), _f64(s["turned"])
        if i in (0, 17, 39):
            _check_rotary(t[:, :6].transpose(1, 0, 2), x[:, :6].transpose(1, 0, 2), np.full(3, i), _f64(s["freq"]),
                          torch.bfloat16)
        keys.append(serving.values(*serving.block_quantize(t[:, 4:6], fp8), fp8))
        values.append(serving.values(*serving.block_quantize(x[:, 6:8], fp8), fp8))
        if i not in (0, 1, 15, 16, 31, 32, 39):
            continue
        for b in range(3):
            k, v = (np.stack([y[b] for y in z]) for z in (keys, values))
            o, _, spread, size, reach = serving.attention(t[b:b + 1, :4], k, v, np.ones((1, i + 1), bool), 128 ** -0.5)
            e = 2 * (132 * U * reach + (i + 65) * 2 * U + 4 * U)
            tol = 2.0 ** -8 * (1 + 2.0 ** -7) * spread + e[..., None] * size + U * np.abs(o)
            assert np.all(np.abs(_f64(out[b:b + 1]) - o) <= tol), (i, b)


def test_graphs_streams_and_repeats(fa):
    """A captured decode step replayed with eager work between, two captured graphs (their
    workspaces are their own) replayed in turn and on two streams at once, and another stream: the eager bits."""
    states = [_decode_state(fa, False, seed=i, B=2, page=64, steps=3000) for i in range(2)]
    for s in states:   # a long prefix, so that sequences are cut and the workspace is used
        n = 2 * s["table"].shape[1] * 64
        x = torch.randn((n, 2, 128), device="cuda", generator=s["g"]).bfloat16()
        fa.cache_write(x, x.flip(0), s["cache"], torch.arange(n, device="cuda"))
    graphs = []
    for s in states:
        _next(s, 2500)
        _step(fa, s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s["out"] = _step(fa, s)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(2501, 2505):
        want = []
        for s in states:
            _next(s, i)
            want.append(_step(fa, s))
            s["out"].fill_(float("nan"))
        torch.cuda.synchronize()
        if i % 2:
            for graph in graphs:
                graph.replay()
        else:
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for s, w in zip(states, want):
            assert torch.equal(s["out"], w), i
        with torch.cuda.stream(streams[0]):
            again = _step(fa, states[0])
        streams[0].synchronize()
        assert torch.equal(again, want[0])


def test_outputs_are_deterministic_and_bounded(fa):
    """Two runs give the same bits, into buffers whose surroundings stay."""
    b = Batch([3000, 700, 1], [5, 1, 1], 2, 3, 128, True, 64, seed=3)
    n, Hq = 7, 6
    first = b.call(fa)
    buf = torch.full((n + 2, Hq, 128), 7.0, device="cuda")
    lse = torch.full((n + 2, Hq), 7.0, device="cuda")
    got = b.call(fa, out=buf[1:-1], lse=lse[1:-1])
    assert torch.equal(got, first)
    assert bool((buf[0] == 7).all() and (buf[-1] == 7).all() and (lse[0] == 7).all() and (lse[-1] == 7).all())


def test_native_calls_equal_the_python_path(fa, monkeypatch):
    """The native call path against the checks in Python: calls that it takes, leaves to them, and refuses."""
    from test_gpu_binding import _outcome, _PythonOnly, _Refused, _same, _Watched
    g = torch.Generator(device="cuda").manual_seed(7)
    B, T, H, G, d = 3, 2, 2, 2, 64
    n, Hq = B * T, H * G
    cache = fa.kv_cache(B * 80, H, 16, d)
    wide = fa.kv_cache(4, H, 16, d, fp8=True)
    fill = torch.randn((B * 1280, H, d), device="cuda", generator=g).bfloat16()
    fa.cache_write(fill, fill, cache, torch.arange(B * 1280, device="cuda"))
    table = torch.arange(B * 80, device="cuda", dtype=torch.int32).view(B, 80)
    lengths = torch.tensor([40, 3, 1200], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device="cuda")
    fused = torch.randn((n, Hq + 2 * H, d), device="cuda", generator=g).bfloat16()
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
    tree = torch.tensor([1, 3] * B, device="cuda")
    slots = torch.arange(n, device="cuda")
    out32, out16 = (torch.empty((n, Hq, d), device="cuda", dtype=t) for t in (torch.float32, torch.bfloat16))
    lse = torch.empty((n, Hq), device="cuda")
    x = torch.randn((2, 3, 5, d), device="cuda", generator=g)
    at, freq = torch.arange(5, device="cuda"), fa.rotary_frequencies(d)[0]
    turned = torch.empty_like(x)

    def wrote(*a):
        c = fa.KVCache(*(t.clone() for t in a[2]))
        return (fa.cache_write(a[0], a[1], c, *a[3:]), *c)[1:]
    att = (q, cache, table, lengths)
    taken = [
        lambda: fa.rotary(x, at, freq), lambda: fa.rotary(x, at, freq, out=turned, inverse=True, magnitude=0.5),
        lambda: fa.rotary(x, at.expand(2, 5).contiguous(), freq, interleaved=True),
        lambda: fa.rotary(x.transpose(1, 2), torch.arange(3, device="cuda"), freq), lambda: fa.rotary(q, slots, freq),
        lambda: fa.rotary(x[:1], at, freq[:8]), lambda: wrote(k, v, cache, slots), lambda: wrote(k.float(), v.float(), wide, slots),
        lambda: wrote(k, v, tuple(cache), slots), lambda: fa.cache_read(cache, slots),
        lambda: fa.cache_read(wide, slots, out_dtype=torch.bfloat16), lambda: fa.cache_attention(*att),
        lambda: fa.cache_attention(*att, q_starts=starts, max_q=2, tree=tree, out=out16, lse=lse),
        lambda: fa.cache_attention(*att, tree=tree.view(n, 1), softmax_scale=0.3, out_dtype=torch.bfloat16),
        lambda: fa.cache_attention(*att, max_q=2, out=out32), lambda: fa.cache_attention(q.contiguous(), *att[1:]),
    ]
    left = [
        lambda: fa.rotary(x, at, freq, magnitude=1), lambda: fa.rotary(x[:0], at, freq),
        lambda: fa.rotary(x, at, freq, interleaved=1), lambda: wrote(k[:0], v[:0], cache, slots[:0]),
        lambda: fa.cache_read(cache, slots[:0]), lambda: fa.cache_attention(*att, softmax_scale=1),
        lambda: fa.cache_attention(q[:0], *att[1:]), lambda: fa.cache_attention(q, list(cache), table, lengths),
    ]
    refused = [
        lambda: fa.rotary(x.double(), at, freq), lambda: fa.rotary(x, at.int(), freq), lambda: fa.rotary(x, at[:3], freq),
        lambda: fa.rotary(x, at, freq.float()), lambda: fa.rotary(x, at, freq[:5]), lambda: fa.rotary(x[..., ::2], at, freq),
        lambda: fa.rotary(x, at, freq, out=turned[:1]), lambda: fa.rotary(x, at, freq, out=turned[:, :, :1].expand(2, 3, 5, d)),
        lambda: fa.rotary(x, at, freq, out=turned.bfloat16()),
        lambda: fa.rotary(x, at, torch.zeros(64, dtype=torch.float64, device="cuda")), lambda: fa.rotary(x, at.cpu(), freq),
        lambda: fa.rotary(x, at, freq, magnitude=float("inf")), lambda: fa.rotary(x[..., 4:], at, freq[:16]),
        lambda: wrote(k, v[:3], cache, slots), lambda: wrote(k, v.float(), cache, slots), lambda: wrote(k, v, cache, slots.int()),
        lambda: wrote(k.half(), v.half(), cache, slots), lambda: wrote(q, q, cache, slots), lambda: wrote(k, v, cache, slots[:2]),
        lambda: wrote(k, v, cache._replace(k_scales=cache.k_scales[:1]), slots),
        lambda: wrote(k, v, cache._replace(v_codes=wide.v_codes), slots), lambda: wrote(k, v, cache[:3], slots),
        lambda: fa.cache_read(cache, slots, out_dtype=torch.float16), lambda: fa.cache_read(cache, slots.view(2, 3)),
        lambda: fa.cache_attention(q.float(), *att[1:]), lambda: fa.cache_attention(q[:, :3], *att[1:]),
        lambda: fa.cache_attention(q[:, :, :32], *att[1:]), lambda: fa.cache_attention(q[:5], *att[1:]),
        lambda: fa.cache_attention(q, cache, table.long(), lengths), lambda: fa.cache_attention(q, cache, table[:2], lengths),
        lambda: fa.cache_attention(q, cache, table[:, ::2], lengths), lambda: fa.cache_attention(q, cache, table, lengths[:2]),
        lambda: fa.cache_attention(*att, q_starts=starts), lambda: fa.cache_attention(*att, q_starts=starts[:3], max_q=2),
        lambda: fa.cache_attention(*att, max_q=3), lambda: fa.cache_attention(*att, tree=tree[:4]),
        lambda: fa.cache_attention(*att, tree=tree.int()), lambda: fa.cache_attention(*att, q_starts=starts, max_q=65, tree=tree),
        lambda: fa.cache_attention(*att, q_starts=starts, max_q=0), lambda: fa.cache_attention(*att, softmax_scale=-0.5),
        lambda: fa.cache_attention(*att, out=out32[:3]), lambda: fa.cache_attention(*att, out=out32.half()),
        lambda: fa.cache_attention(*att, lse=lse[:, :1]), lambda: fa.cache_attention(*att, out_dtype=torch.float16),
        lambda: fa.cache_attention(q.transpose(0, 1), *att[1:]), lambda: fa.cache_attention(q, cache, table.cpu(), lengths),
    ]
    native, buffers = fa.api._binding, (out32, out16, lse, turned)
    for kind, calls in (("taken", taken), ("left", left), ("refused", refused)):
        for i, call in enumerate(calls):
            watched = _Watched(native)
            got = []
            for binding in (watched, _PythonOnly()):
                monkeypatch.setattr(fa.api, "_binding", binding)
                got.append(_outcome(call, buffers))
            a, b = got
            assert _same(a, b), f"{kind} call {i}: {a} through the native path, {b} through Python"
            assert isinstance(a, _Refused) == (kind == "refused"), f"{kind} call {i}: {a}"
            if kind != "refused":
                assert watched.took == (kind == "taken"), f"{kind} call {i}"
    monkeypatch.setattr(fa.api, "_binding", native)


@pytest.mark.parametrize("d,fp8,H,G,new", [(128, False, 390, 2, [1, 1]), (64, False, 520, 1, [1, 1]), (64, True, 390, 1, [20, 3]),
                                           (128, True, 260, 1, [70, 1])])
def test_more_key_heads_than_ranges(fa, d, fp8, H, G, new):
    """So many key heads that a key head's workgroups cannot be two: nothing is cut, and no workspace is asked for,
    in a table of 4096 keys."""
    keys = [200, 130]
    b = Batch(keys, new, H, G, d, fp8, 64, seed=H, spare=60)
    c = fa.api._cache(fa.KVCache(*(torch.from_numpy(t).cuda() for t in b.cache)))
    size = fa.lib.fp4attn_cache_attention_workspace
    assert size(c, H * G, 2, b.table.shape[1], max(new)) == 0 and size(c, H * G, 2, 16, max(new)) == 0
    lse = torch.empty((sum(new), H * G), device="cuda")
    b.check(b.call(fa, lse=lse), lse)


@pytest.mark.parametrize("width", [1, 6000])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,idle", [(2, 0), (5, 0), (20, 0), (20, 512)])
def test_hidden_nan_codes_in_every_tiling(fa, d, G, idle, width):
    """NaN codes of MXFP8 values under ordinary scales: the rows that see them are NaN in their channels, and
    no other row or channel changes; with a tree, causal, and before the new tokens."""
    b = Batch([190], [6], 2, G, d, True, 16, seed=9)
    if idle or width > 1:
        _beside_idle(b, idle, width)
    prefix = 184
    tree = np.array([0b1, 0b11, 0b101, 0b1000, 0b10001, 0b100000], dtype=np.int64)
    clean = {True: b.call(fa, tree=tree), False: b.call(fa)}
    part = d // 16
    codes = [(1, 0, 37, 0x7F), (4, 1, 3, 0xFF), (4, 1, d - 1, 0x7F), (4, 1, d - 2, 0xFF), (0, 1, 20, 0xFF)]
    for token, head, channel, code in codes:
        p, off = divmod(int(b.slots[0][prefix + token]), 16)
        b.cache[2][p, head, off // 8, channel // part, off % 8, channel % part] = code
    for with_tree in (True, False):
        out = b.call(fa, tree=tree if with_tree else None)
        bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for token, head, channel, _ in codes:
            for row in range(6):
                if (int(tree[row]) >> token & 1) if with_tree else token <= row:
                    bad[row, head * G:(head + 1) * G, channel] = True
        assert torch.equal(torch.isnan(out), bad), with_tree
        assert torch.equal(out[~bad], clean[with_tree][~bad]), with_tree
    for token in (0, 100, 183):   # of the prefix: every row sees it
        p, off = divmod(int(b.slots[0][token]), 16)
        b.cache[2][p, 1, off // 8, token % 16, off % 8, 1] = 0x7F
        bad[:, G:, token % 16 * part + 1] = True
    out = b.call(fa)
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad], clean[False][~bad])


HIDDEN_TOKENS = 6    # drafted tokens of the batches with hidden values
FULL_TILES = 1100    # row tiles of idle sequences beside them that fill the chip for every format


@pytest.mark.parametrize("width", [1, 6000])
@pytest.mark.parametrize("d,fp8", FORMATS)
def test_hidden_values_in_a_full_chip(fa, d, fp8, width):
    """The hidden values of the tests above in the kernel of 128 rows, for every format."""
    test_hidden_and_missing_in_every_tiling(fa, d, fp8, 20, FULL_TILES, width)
    if fp8:
        test_hidden_nan_codes_in_every_tiling(fa, d, 20, FULL_TILES, width)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [(2, 3, 5, 64), (7, 4, 64)])
def test_rotary_under_autograd(fa, shape, interleaved, dtype):
    """A leaf's gradient through rotary is the inverse turn of the result's, whatever the strides of the latter;
    against autograd on the formula in fp64; twice differentiated; and without a graph the same values."""
    g = torch.Generator().manual_seed(len(shape))
    x, dy = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    n = shape[0] if len(shape) == 3 else shape[2]
    at = torch.randint(0, 100000, (n,), generator=g)
    freq = fa.rotary_frequencies(48, device="cpu")[0]
    o = dict(interleaved=interleaved, magnitude=0.8)
    args = at.cuda(), freq.cuda()
    leaf = x.cuda().requires_grad_()
    y = fa.rotary(leaf, *args, **o)
    assert y.requires_grad
    with torch.no_grad():
        plain = fa.rotary(leaf, *args, **o)
    assert not plain.requires_grad and torch.equal(plain, y)
    back = fa.rotary(dy.cuda(), *args, inverse=True, **o)
    assert not back.requires_grad
    grad, = torch.autograd.grad(y, leaf, dy.cuda(), retain_graph=True)
    assert torch.equal(grad, back)
    strided = dy.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(torch.autograd.grad(y, leaf, strided, retain_graph=True)[0], back)
    ones = torch.autograd.grad(y.sum(), leaf, retain_graph=True)[0]   # an expanded gradient
    assert torch.equal(ones, fa.rotary(torch.ones_like(leaf, requires_grad=False), *args, inverse=True, **o))
    # the formula: [n, H, d] as [1, H, n, d]
    def heads_first(t):
        return t.transpose(0, 1)[None] if len(shape) == 3 else t
    _check_rotary(_f64(heads_first(grad)), _f64(heads_first(dy)), at.numpy(), freq.numpy(), dtype, inverse=True, **o)
    # linear: the gradient of <grad, w> with respect to dy is rotary of w
    v = dy.cuda().requires_grad_()
    w = torch.randn(shape, generator=g).to(dtype).cuda()
    grad, = torch.autograd.grad(y, leaf, v, create_graph=True)
    assert torch.equal(torch.autograd.grad(grad, v, w)[0], fa.rotary(w, *args, **o))
    turned_back = fa.rotary(leaf, *args, inverse=True, **o)
    assert torch.equal(torch.autograd.grad(turned_back, leaf, dy.cuda())[0], fa.rotary(dy.cuda(), *args, **o))
