"""Pins of the pages oracle: small states worked out by hand, what always holds, and attention against a slab without pages."""
import random

import pytest
import torch

from oracle import pages_oracle as P


def pool(n_pages, size, table, lens, refs=None, hk=2, d=4):
    gen = torch.Generator().manual_seed(n_pages)
    k, v = (torch.randn(n_pages, hk, size, d, generator=gen).bfloat16() for _ in range(2))
    if refs is None:
        refs = [sum(row.count(p) for row in table) for p in range(n_pages)]
    return P.Pool(k, v, refs, table, lens)


def test_reserve_by_hand():
    # two sequences on the same two pages of 4 rows, 6 rows each; a third alone on page 5 with 4 rows
    s = pool(8, 4, [[3, 1, -1], [3, 1, -1], [5, -1, -1]], [6, 6, 4])
    before = s.k.clone()
    assert s.reserve(3) == 0
    # rows 6..8 of the first two are on pages 1 and 2 of the table: the first sequence gets a copy of page 1, the second keeps it
    assert s.table == [[3, 0, 2], [3, 1, 4], [5, 6, -1]]
    assert s.refs == [1, 1, 1, 2, 1, 1, 1, 0]
    assert torch.equal(s.k[0], before[1]) and torch.equal(s.k[1:], before[1:])
    assert s.reserve(3) == 0 and s.table == [[3, 0, 2], [3, 1, 4], [5, 6, -1]]           # once is enough
    assert s.reserve(8, count=[0, 9, 0], first=[0, 0, 0]) == 0 and s.table[1] == [7, 1, 4] and s.refs[3] == 1
    assert s.reserve(5, count=[0, 0, 5]) == P.SHORT                                      # rows 4..8: one more page, none free
    assert s.reserve(13) == P.MISSING and s.table[2] == [5, 6, -1]


def test_sequences_not_in_use():
    s = pool(6, 4, [[0, 1], [2, -1], [-1, -1]], [5, -1, -3])
    before = s.k.clone()
    assert s.reserve(2) == 0 and s.table == [[0, 1], [2, -1], [-1, -1]]
    assert s.append(*[torch.ones(3, 1, 2, 4, dtype=torch.bfloat16)] * 2) == 0
    assert torch.equal(s.k[2:], before[2:]) and bool((s.k[1, :, 1] == 1).all())
    assert s.fork([1], [2]) == P.MISSING
    assert s.free([5, 3, 0]) == 0 and s.len == [5, -1, -3] and s.table == [[0, 1], [-1, -1], [-1, -1]] and s.refs == [1, 1, 0, 0, 0, 0]


def test_fork_and_free_by_hand():
    s = pool(6, 4, [[0, 1, 2], [3, -1, -1], [-1, -1, -1]], [5, 2, 0])                    # page 2 is reserved ahead
    assert s.fork([0, 1], [1, 2]) == 0                                                   # the second takes what the first pair overwrites
    assert s.table == [[0, 1, 2], [0, 1, -1], [3, -1, -1]] and s.len == [5, 5, 2] and s.refs == [2, 2, 1, 1, 0, 0]
    assert s.fork([0, 2, 7], [2, 2, 0]) == P.MISSING and s.table[2] == [3, -1, -1]       # the last pair of a child counts: its own parent
    assert s.free([5, 4, -1]) == 0
    assert s.table == [[0, 1, -1], [0, -1, -1], [3, -1, -1]] and s.len == [5, 4, 2] and s.refs == [2, 1, 0, 1, 0, 0]
    assert s.free([0, 0, 0]) == 0 and s.refs == [0] * 6 and s.len == [0, 0, 0]


def test_compact_by_hand():
    s = pool(7, 2, [[6, 1, -1], [6, 4, 2]], [3, 5])
    before = s.k.clone()
    assert s.compact() == 4                                                              # held: 1, 2, 4, 6 -> 0 and 3 are filled from 4 and 6
    assert s.table == [[3, 1, -1], [3, 0, 2]] and s.refs == [1, 1, 1, 2, 0, 0, 0]
    assert torch.equal(s.k[0], before[4]) and torch.equal(s.k[3], before[6])


def test_what_always_holds():
    rng = random.Random(3)
    s = pool(40, 3, [[-1] * 6 for _ in range(7)], [0] * 7)
    for _ in range(400):
        kept = [s.rows(b, s.len[b]) for b in range(7)]
        do = rng.choice(["reserve", "fork", "free", "compact"])
        if do == "reserve":
            n = rng.randint(1, 5)
            ok = s.reserve(n) == 0
            if ok:
                for b in range(7):
                    m = rng.randint(0, n)
                    for r in range(s.len[b], s.len[b] + m):
                        page, at = s.place(b, r)
                        assert s.refs[page] == 1
                        s.k[page, :, at] = s.v[page, :, at] = rng.random()
                    assert torch.equal(s.rows(b, s.len[b]), kept[b])
                    s.len[b] += m
        elif do == "fork":
            pairs = [(rng.randrange(7), rng.randrange(7)) for _ in range(rng.randint(1, 4))]
            assert s.fork(*zip(*pairs)) == 0
            for c, p in dict((c, p) for p, c in pairs).items():
                assert torch.equal(s.rows(c, s.len[c]), kept[p])
        elif do == "free":
            s.free([rng.randint(-3, 12) for _ in range(7)])
        else:
            used = s.compact()
            assert all(r > 0 for r in s.refs[:used]) and not any(s.refs[used:])
            for b in range(7):
                assert torch.equal(s.rows(b, s.len[b]), kept[b])
        assert s.refs == [sum(row.count(p) for row in s.table) for p in range(40)]


@pytest.mark.parametrize("n", [0, 1, 5, 11])
def test_attention_is_that_over_a_slab(n):
    s = pool(9, 4, [[7, 0, 3]], [n])
    k, v = s.rows(0, n)
    slab_k = torch.cat([s.k[p] for p in (7, 0, 3)], 1)[:, :n].double()
    assert torch.equal(k, slab_k)
    q = torch.randn(4, 4, generator=torch.Generator().manual_seed(n)).bfloat16()
    o, lse, p = P.attention(q, k, v, 2)
    if n == 0:
        assert not o.any() and torch.isinf(lse).all()
        return
    for i in range(4):
        e = torch.tensor([float(torch.exp((q[i].double() * slab_k[i // 2, r]).sum() / 2)) for r in range(n)], dtype=torch.float64)
        assert torch.allclose(lse[i], e.sum().log(), atol=1e-12)
        assert torch.allclose(o[i], (e[:, None] * v[i // 2]).sum(0) / e.sum(), atol=1e-12)
