"""Pages, slots and positions of a step against the oracle, which goes sequence by sequence: whole
numbers, equal everywhere."""
import random

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def _scenario(rng, B, width, page, spread, uniform=None, shared=False, scarce=False, wild=False):
    """Rows with the pages that their sequences hold, a ring that has turned, and a step's wishes."""
    def pages(keys, s):
        return max(-(-keys // page), s // page)
    capacity = width * page
    held, lengths, new, common = [], [], [], []
    for _ in range(B):
        s = rng.choice((0, rng.randint(0, capacity // 2))) if shared else 0
        h = rng.randint(s, capacity) if rng.random() < 0.8 else 0
        what = rng.random()
        if what < 0.1:
            n, t = 0, 0
        elif what < 0.3:
            n, t = h, rng.randint(0, min(h, spread))
        else:
            t = rng.randint(0, spread)
            n = min(max(h, s) - rng.randint(0, min(20, max(h, s) - s)) + t, capacity)
            t = min(t, n)
        if uniform is not None:
            t, n = uniform, 0 if n == 0 else min(max(h, s) + uniform, capacity)
        if wild and rng.random() < 0.2:
            n, t, h, s = rng.choice(((capacity + 1, 3, h, s), ((1 << 31) - 1, 1, h, s), (-(1 << 31), 2, h, s), (n, -5, h, s),
                                     (n, t, h, -9), (n, t, -4, 0), (2, 5, h, s)))
        held.append(h), lengths.append(n), new.append(t), common.append(s)
    had = [pages(min(max(h, 0), capacity), max(s, 0)) for h, s in zip(held, common)]
    need = sum(max(0, min(pages(n, s), width) - h) for n, s, h in zip(lengths, common, had))
    free = max(1, need // 3 if scarce else need + 3)
    order = list(range(sum(had) + free))
    rng.shuffle(order)
    table, at = [], 0
    for h in had:
        table.append(order[at:at + h] + [-1] * (width - h))
        at += h
    ring, taken = [-1] * len(order), rng.choice((0, 12345678901))
    for i in range(free):
        ring[(taken + i) % len(ring)] = order[at + i]
    return table, held, lengths, ring, [taken, taken + free], new, common


def _run(fa, scenario, page, tokens, new, shared, in_place=False):
    def put(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")
    table, held, lengths, ring, counts = scenario[:5]
    table, held, lengths, pool = put(table), put(held), put(lengths), fa.KVPool(put(ring), put(counts, torch.int64))
    step = fa.cache_assign(table, held, lengths, pool, page, tokens, new=None if new is None else put(new),
                           shared=None if shared is None else put(shared), in_place=in_place)
    assert step.pool.free is pool.free
    if in_place:
        assert step.lengths is held and step.pool.counts is pool.counts
    return (step.slots.tolist(), step.positions.tolist(), step.q_starts.tolist(), step.lengths.tolist(),
            step.pool.counts.tolist()), table.tolist(), pool.free.tolist()


def _check(fa, scenario, page, tokens, new, shared, in_place=False):
    table, ring = [list(r) for r in scenario[0]], list(scenario[3])
    want = serving.assign(table, scenario[1], scenario[2], ring, scenario[4], page, tokens, new, shared)
    got = _run(fa, scenario, page, tokens, new, shared, in_place)
    for name, x, y in zip(("slots", "positions", "starts", "lengths", "counts"), got[0], want):
        assert x == y, name
    assert got[1] == table and got[2] == ring


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("B,width,page,spread", [(1, 1, 16, 5), (1, 300, 16, 4000), (3, 7, 64, 40), (64, 33, 16, 100), (65, 9, 128, 3),
                                                 (1000, 5, 16, 30), (1024, 3, 32, 9), (1025, 3, 32, 9), (2500, 4, 16, 20)])
def test_steps(fa, B, width, page, spread, seed, in_place):
    rng = random.Random(B * 10 + seed)
    scenario = _scenario(rng, B, width, page, spread, shared=seed % 2 == 1, scarce=seed >= 2, wild=seed == 3)
    new, shared = scenario[5], scenario[6]
    total = sum(max(0, n) for n in new)
    tokens = (total, total + 13, max(0, total - 4), total + 1)[seed]   # padding, too few
    _check(fa, scenario, page, tokens, new, shared if seed % 2 else None, in_place)


@pytest.mark.parametrize("B,each", [(1, 1), (64, 1), (5, 17), (300, 4), (1500, 2), (7, 0)])
def test_equal_numbers_of_tokens(fa, B, each):
    scenario = _scenario(random.Random(B), B, 6, 16, 1, uniform=each)
    _check(fa, scenario, 16, B * each, None, None)


def test_most_sequences(fa):
    """65535 sequences, and a table with more pages than a launch has threads."""
    B = 65535
    held = [16 * (b % 3) + b % 5 for b in range(B)]
    lengths = [(0 if b % 11 == 0 else h + b % 19) for b, h in enumerate(held)]
    new = [0 if b % 11 == 0 else b % 19 for b in range(B)]
    had = [-(-h // 16) for h in held]
    first = np.cumsum([0] + had)
    table = [list(range(first[b], first[b] + had[b])) + [-1] * (5 - had[b]) for b in range(B)]
    free = list(range(first[-1], first[-1] + 50000))
    ring = free + [-1] * int(first[-1])
    _check(fa, (table, held, lengths, ring, [0, len(free)]), 16, sum(new) + 5, new, None)
    width = 1 << 19
    for held, lengths in (([5, 0], [5 + 16 * 300000, 16 * 90000]), ([16 * 300001, 16 * 90000], [3, 0])):
        had = [-(-h // 16) for h in held]
        table = [list(range(had[0])) + [-1] * (width - had[0]), list(range(had[0], sum(had))) + [-1] * (width - had[1])]
        ring = list(range(sum(had), 400000)) + [-1] * sum(had)
        _check(fa, (table, held, lengths, ring, [400000 * 7, 400000 * 7 + 400000 - sum(had)]), 16, 3, [2, 1], None)


def test_nothing_to_do(fa):
    table = [[3, -1], [4, 5]]
    _check(fa, (table, [10, 20], [10, 20], [0, 1, 2], [4, 6]), 16, 0, [0, 0], None)
    _check(fa, (table, [10, 20], [0, 0], [0, 1, 2, 6, 7, 8], [4, 6]), 16, 0, None, None)


def test_captured_steps(fa):
    """A decode step captured once: each replay moves every sequence on, across pages, until the pool is empty."""
    B, width, page = 5, 4, 16
    g = random.Random(1)
    held = [g.randint(1, 30) for _ in range(B)]
    had = [-(-h // page) for h in held]
    first = np.cumsum([0] + had)
    table = [[int(x) for x in range(first[b], first[b] + had[b])] + [-1] * (width - had[b]) for b in range(B)]
    ring = list(range(int(first[-1]), 16)) + [-1] * int(first[-1])
    counts = [0, 16 - int(first[-1])]
    d_table, d_held = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (table, held))
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    pool = fa.KVPool(torch.tensor(ring, dtype=torch.int32, device="cuda"), torch.tensor(counts, device="cuda"))
    before = [t.clone() for t in (d_table, d_held, *pool)]
    graph = torch.cuda.CUDAGraph()
    fa.cache_assign(d_table, d_held, d_held + one, pool, page, B, in_place=True)   # warm
    with torch.cuda.graph(graph):
        step = fa.cache_assign(d_table, d_held, d_held + one, pool, page, B, in_place=True)
    for t, x in zip((d_table, d_held, *pool), before):
        t.copy_(x)
    refused = 0
    for i in range(40):
        graph.replay()
        torch.cuda.synchronize()
        slots, positions, starts, after, counts = serving.assign(table, held, [h + 1 for h in held], ring, counts, page, B)
        assert step.slots.tolist() == slots and step.positions.tolist() == positions, i
        assert step.q_starts.tolist() == starts and d_held.tolist() == after and pool.counts.tolist() == counts, i
        assert d_table.tolist() == table and pool.free.tolist() == ring, i
        refused += after == held
        held = after
        (one * 3).sum().item()   # the program's own work between the replays
    assert refused


def test_streams(fa):
    """Two streams, each with its own tables; the work is ordered by the stream it is called on."""
    rng = random.Random(8)
    cases = [_scenario(rng, 200, 9, 16, 30) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    for scenario, stream in zip(cases, streams):
        with torch.cuda.stream(stream):
            _check(fa, scenario, 16, sum(scenario[5]), scenario[5], None)


def test_refusals_and_the_python_path(fa, monkeypatch):
    def put(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")
    table, held, pool = put([[0, -1], [1, -1]]), put([3, 4]), fa.cache_pool(4, first=2)
    good = dict(page_table=table, held=held, lengths=held + 1, pool=pool, page_size=16, tokens=2)
    for o, error in ((dict(page_table=table.long()), TypeError), (dict(page_table=table[0]), ValueError),
                     (dict(page_table=table.t()), ValueError), (dict(held=put([3])), ValueError), (dict(held=held.long()), TypeError),
                     (dict(lengths=put([3, 4, 5])), ValueError), (dict(new=put([1])), ValueError), (dict(new=put([1., 1.], torch.float32)),
                     TypeError), (dict(shared=put([1, 2, 3])), ValueError), (dict(pool=(pool.free,)), ValueError),
                     (dict(pool=(pool.free, pool.counts[:1])), ValueError), (dict(pool=(pool.free.long(), pool.counts)), TypeError),
                     (dict(pool=(pool.free[:0], pool.counts)), fa.Fp4AttnError), (dict(page_size=24), fa.Fp4AttnError),
                     (dict(page_size=16.0), TypeError), (dict(tokens=3), fa.Fp4AttnError), (dict(tokens=-2), fa.Fp4AttnError),
                     (dict(tokens=1 << 25), fa.Fp4AttnError), (dict(lengths=held.cpu()), ValueError),
                     (dict(lengths=held, in_place=True), fa.Fp4AttnError), (dict(new=held, in_place=True), fa.Fp4AttnError),
                     (dict(shared=held, in_place=True), fa.Fp4AttnError)):
        with pytest.raises(error):
            fa.cache_assign(**dict(good, **o))
    assert table.tolist() == [[0, -1], [1, -1]] and pool.counts.tolist() == [0, 2]   # refused calls change nothing
    from paper_2609_04105_amd import api
    scenario = _scenario(random.Random(3), 20, 5, 16, 30, shared=True)
    native = _run(fa, scenario, 16, sum(scenario[5]), scenario[5], scenario[6])
    monkeypatch.setattr(api, "_binding", api._NoBinding)
    for in_place in (False, True):
        assert _run(fa, scenario, 16, sum(scenario[5]), scenario[5], scenario[6], in_place) == native
