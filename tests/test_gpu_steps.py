"""A small server: pages and slots by cache_assign, rotary, cache_write and attention over the cache behind a shared
prefix, step by step; requests join with prompts of any length, draft and take back, end, and wait where pages run out.
Every key and value that a request holds, and every output, against the fp64 oracle (tolerances: test_gpu_shaped.py)."""
import random

import numpy as np
import pytest
import torch

from oracle import serving
from test_gpu_serving import U, _f64

pytestmark = pytest.mark.gpu

B, H, G, D, PAGE, PREFIX = 6, 128, 1, 64, 16, 528   # key heads enough that the prefix gets a pass of its own
HEADS = (0, 31, 127)


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, fa, fp8, pages, seed):
        self.fa, self.fp8, self.rng = fa, fp8, random.Random(seed)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.cache, own = fa.kv_cache(pages, H, PAGE, D, fp8), PREFIX // PAGE
        self.freq, _ = fa.rotary_frequencies(D)
        self.table = _int([list(range(own)) + [-1] * 12] * B)
        self.pool, self.held = fa.cache_pool(pages, first=own), _int([0] * B)
        self.shared = _int([PREFIX] * B)
        k, v = (torch.randn((PREFIX, H, D), device="cuda", generator=self.g).bfloat16() for _ in range(2))
        k = fa.rotary(k, torch.arange(PREFIX, device="cuda"), self.freq)
        fa.cache_write(k, v, self.cache, torch.arange(PREFIX, device="cuda"))
        first = [(x, y) for x, y in zip(self._values(k), self._values(v))]
        self.history = [list(first) for _ in range(B)]   # what each request's keys and values are
        self.prefix, self.keys = first, [0] * B

    def _values(self, x):
        return serving.values(*serving.block_quantize(_f64(x[:, HEADS, :]), self.fp8), self.fp8)

    def step(self, new, back, end, **shape):
        fa, n = self.fa, sum(new) + 3   # three rows of padding
        lengths = [0 if e else max(k, PREFIX) - r + t if t or k else 0 for k, t, r, e in zip(self.keys, new, back, end)]
        step = fa.cache_assign(self.table, self.held, _int(lengths), self.pool, PAGE, n, new=_int(new), shared=self.shared,
                               in_place=True)
        qkv = torch.randn((n, G * H + 2 * H, D), device="cuda", generator=self.g).bfloat16()
        q, k, v = qkv[:, : G * H], qkv[:, G * H:-H], qkv[:, -H:]
        turned = fa.rotary(qkv[:, :-H], step.positions, self.freq)
        fa.cache_write(turned[:, G * H:], v, self.cache, step.slots)
        out = fa.cache_attention(turned[:, : G * H], self.cache, self.table, step.lengths, q_starts=step.q_starts, max_q=max(new + [1]),
                                 shared=PREFIX, **shape)
        assert q.shape == k.shape
        after, starts = step.lengths.tolist(), step.q_starts.tolist()
        ks, vs = self._values(turned[:, G * H:]), self._values(v)
        refused = 0
        for b in range(B):
            if after[b] != lengths[b]:
                assert after[b] == self.keys[b]
                refused += 1
                continue
            if lengths[b] == 0:
                self.history[b] = list(self.prefix)
            else:
                del self.history[b][lengths[b] - new[b]:]
                self.history[b] += [(ks[i], vs[i]) for i in range(starts[b], starts[b + 1])]
                assert len(self.history[b]) == lengths[b]
            self.keys[b] = lengths[b]
            self._check(b, turned, out, starts[b], new[b], **shape)
        return refused

    def _check(self, b, turned, out, first, t, softcap=None, slopes=None, window=None):
        n = self.keys[b]
        if n == 0:
            return
        cache, row = tuple(x.cpu().numpy() for x in self.cache), self.table[b].tolist()
        at = np.array([row[j // PAGE] * PAGE + j % PAGE for j in range(n)])
        p, off = at[:, None] // PAGE, at[:, None] % PAGE
        heads = np.array(HEADS)
        k = serving.values(cache[0][p, heads, off], cache[1][p, heads, off], self.fp8)
        v = serving.values(cache[2][p, heads, off // 8, :, off % 8].reshape(n, len(heads), -1), cache[3][p, heads, off // 8, :, off % 8],
                           self.fp8)
        assert np.array_equal(k, np.stack([x for x, _ in self.history[b]])) and np.array_equal(v, np.stack([y for _, y in self.history[b]]))
        if t == 0:
            return
        q = _f64(turned[first:first + t, HEADS, :])
        slope = None if slopes is None else _f64(slopes)[list(HEADS)]
        o, _, spread, size, reach, high, bias = serving.shaped_attention(
            q, k, v, serving.shaped_mask(t, n, n, window or 0), D ** -0.5, softcap or 0.0, slope, n)
        e = 2 * ((D + 4) * U * reach + 20 * U * high + 8 * U * (bias + high) + (n + 64) * 2 * U + 4 * U)
        tol = 2.0 ** -8 * (1 + 2.0 ** -7) * spread + e[..., None] * size + U * np.abs(o)
        assert np.all(np.abs(_f64(out[first:first + t][:, HEADS, :]) - o) <= tol), b


@pytest.mark.parametrize("fp8", [False, True])
def test_requests_come_and_go(fa, fp8):
    s = Server(fa, fp8, PREFIX // PAGE + 14, seed=3)
    slopes = 2.0 ** (-8.0 * torch.arange(1, H * G + 1, device="cuda") / H)
    shapes = ({}, dict(softcap=20.0), dict(slopes=slopes), dict(window=300), dict(softcap=5.0, slopes=slopes))
    refused = 0
    for i in range(14):
        new = [s.rng.choice((1, 1, 1, s.rng.randint(0, 40))) for _ in range(B)]
        if i % 3 == 0:
            new = [1] * B
        back = [s.rng.randint(0, 2) if k > PREFIX + 4 else 0 for k in s.keys]
        end = [k > 0 and s.rng.random() < 0.12 for k in s.keys]
        new = [0 if e else t for t, e in zip(new, end)]
        refused += s.step(new, back, end, **shapes[i % len(shapes)])
    assert refused   # the pool is smaller than what they ask for
    # all end: every page of their own is free again
    s.step([0] * B, [0] * B, [True] * B)
    free, (taken, returned) = s.pool.free.tolist(), s.pool.counts.tolist()
    assert sorted(free[i % len(free)] for i in range(taken, returned)) == list(range(PREFIX // PAGE, PREFIX // PAGE + 14))


def test_captured_step(fa):
    """A decode step captured once, lengths and pool moved on by each replay: the bits of eager steps of a second server."""
    servers = [Server(fa, False, PREFIX // PAGE + 40, seed=7) for _ in range(2)]
    one, qkv = _int([1] * B), torch.empty((B, G * H + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    for s in servers:
        s.held.fill_(PREFIX)

    def step(s):
        st = fa.cache_assign(s.table, s.held, s.held + one, s.pool, PAGE, B, shared=s.shared, in_place=True)
        turned = fa.rotary(qkv[:, :-H], st.positions, s.freq)
        fa.cache_write(turned[:, G * H:], qkv[:, -H:], s.cache, st.slots)
        return fa.cache_attention(turned[:, : G * H], s.cache, s.table, st.lengths, shared=PREFIX, softcap=30.0)

    qkv.normal_(generator=servers[0].g)
    for s in servers:
        warm = step(s)
    assert torch.isfinite(warm).all()
    graph = torch.cuda.CUDAGraph()
    state = [t.clone() for t in (servers[0].table, servers[0].held, *servers[0].pool, *servers[0].cache)]
    with torch.cuda.graph(graph):
        out = step(servers[0])
    for t, x in zip((servers[0].table, servers[0].held, *servers[0].pool, *servers[0].cache), state):
        assert torch.equal(t, x)   # capturing runs nothing
    for i in range(40):
        qkv.normal_(generator=servers[0].g)
        graph.replay()
        want = step(servers[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    assert servers[0].held.tolist() == [PREFIX + 41] * B
    assert all(torch.equal(x, y) for x, y in zip((servers[0].table, *servers[0].pool, *servers[0].cache),
                                                 (servers[1].table, *servers[1].pool, *servers[1].cache)))
