"""CPU checks of page assignment: refusals before any HIP call, and the oracle's own invariants."""
import ctypes
import random

import pytest
import torch

from oracle import serving

PTR = [ctypes.c_void_p(4096 * (i + 1)) for i in range(16)]   # aligned, never dereferenced


@pytest.fixture(scope="module")
def fa():
    import paper_2609_04105_amd as fa
    return fa


def test_refusals(fa):
    f, size = fa.lib.fp4attn_cache_assign, fa.lib.fp4attn_cache_assign_workspace
    need = size(3, 5000)
    good = dict(table=PTR[0], B=3, pages=4, page=16, held=PTR[1], lengths=PTR[2], new=PTR[3], shared=PTR[4], ring=PTR[5],
                ring_size=9, counts=PTR[6], tokens=5000, slots=PTR[7], positions=PTR[8], starts=PTR[9], after=PTR[10],
                counts_out=PTR[11], work=PTR[12], bytes=need, stream=None)

    def status(**o):
        return f(*dict(good, **o).values())
    odd4, odd8 = ctypes.c_void_p(4098), ctypes.c_void_p(4100)
    for o in (dict(B=0), dict(B=-1), dict(pages=0), dict(ring_size=0), dict(tokens=-1), dict(page=8), dict(page=48),
              dict(page=0), dict(page=-16), dict(new=None), dict(after=PTR[2]), dict(after=PTR[3]), dict(after=PTR[4]), dict(work=None), dict(work=odd8), dict(bytes=need - 1),
              *(dict([(name, bad)]) for name in ("table", "held", "lengths", "ring", "starts", "after") for bad in (None, odd4)),
              *(dict([(name, bad)]) for name in ("counts", "slots", "positions", "counts_out") for bad in (None, odd8)),
              dict(new=odd4), dict(shared=odd4)):
        assert status(**o) == 1, o
    for o in (dict(B=65536, bytes=1 << 30), dict(tokens=(1 << 24) + 1), dict(ring_size=1 << 31), dict(page=1 << 21),
              dict(pages=(1 << 26) + 1), dict(pages=1 << 30, page=16), dict(B=65535, pages=32769, bytes=1 << 30),
              dict(pages=1 << 62)):
        assert status(**o) == 2, o
    assert size(0, 1) == size(65536, 1) == size(1, -1) == size(1, (1 << 24) + 1) == -1
    assert size(1, 1) == size(1024, 4096) == 0 and 0 < size(1, 4097) <= size(65535, 1) < 1 << 21


def test_python_refusals_without_a_gpu(fa):
    pool = fa.cache_pool(8, device="cpu")
    assert pool.free.tolist() == list(range(8)) and pool.counts.tolist() == [0, 8]
    some = fa.cache_pool(8, first=3, device="cpu")
    assert some.free.tolist() == [3, 4, 5, 6, 7, -1, -1, -1] and some.counts.tolist() == [0, 5]
    for bad in ((0,), (4, 4), (4, -1)):
        with pytest.raises(ValueError):
            fa.cache_pool(*bad, device="cpu")
    table, lengths = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        fa.cache_assign(table, lengths, lengths, pool, 16, 2)


def test_oracle_keeps_every_page():
    """Through many steps every page is in one row's used places or in the ring's free part, once."""
    rng = random.Random(5)
    B, width, page, pages = 7, 9, 16, 40
    table, ring, counts = [[-1] * width for _ in range(B)], list(range(pages)), [0, pages]
    held = [0] * B
    refused = 0
    for _ in range(300):
        new = [rng.choice((0, 1, 1, rng.randint(0, 60))) for _ in range(B)]
        lengths = [0 if rng.random() < 0.1 else max(0, h - rng.randint(0, 3)) + n for h, n in zip(held, new)]
        new = [min(n, length) for n, length in zip(new, lengths)]
        slots, positions, starts, after, counts = serving.assign(table, held, lengths, ring, counts, page, sum(new), new)
        refused += sum(a != n for a, n in zip(after, lengths))
        rows = [table[b][j] for b in range(B) for j in range(-(-after[b] // page))]
        free = [ring[i % pages] for i in range(counts[0], counts[1])]
        assert sorted(rows + free) == list(range(pages))
        for b in range(B):
            mine = slice(starts[b], starts[b + 1])
            assert positions[mine] == list(range(lengths[b] - new[b], lengths[b]))
            want = [table[b][p // page] * page + p % page for p in positions[mine]] if after[b] == lengths[b] else [-1] * new[b]
            assert slots[mine] == want
        held = after
    assert refused > 20


def test_oracle_by_hand():
    table, ring = [[4, 5, -1], [7, -1, -1], [9, 2, 3]], [10, 11, 12, 13]
    # the first grows by two tokens into a new page, the second asks for two pages that are not there, the third takes
    # back seventeen keys and a page
    got = serving.assign(table, [31, 5, 40], [33, 40, 23], ring, [5, 7], 16, 8, [2, 3, 1])
    assert got == ([95, 11 * 16, -1, -1, -1, 2 * 16 + 6, -1, -1], [31, 32, 37, 38, 39, 22, 0, 0], [0, 2, 5, 6], [33, 5, 23], [6, 8])
    assert table == [[4, 5, 11], [7, -1, -1], [9, 2, 3]] and ring == [10, 11, 12, 3]
    # shared pages are neither taken nor written nor returned
    table, ring = [[1, 2, -1], [1, 2, 6]], [3, 4]
    got = serving.assign(table, [0, 35], [34, 0], ring, [0, 1], 16, 3, [3, 0], [32, 40])
    assert got == ([-1, 48, 49], [31, 32, 33], [0, 3, 3], [34, 0], [1, 2]) and table[0] == [1, 2, 3] and ring == [3, 6]
