"""The cache in pages on the GPU against its oracle: rows in and out, pages reserved, forked, freed and compacted.  Everything here is whole
numbers and rows that are moved as they are: results are equal, bit for bit."""
import random

import pytest
import torch

from oracle import pages_oracle as P

pytestmark = pytest.mark.gpu


def make(hk=2, dh=64, hq=None, **kw):
    from paper_2510_04476_b200.binding import CCA
    hq = hq or hk
    return CCA(d_model=hq * dh, n_q_heads=hq, n_kv_heads=hk, head_dim=dh, **kw)


def ints(*x):
    return torch.tensor(x[0] if len(x) == 1 and isinstance(x[0], (list, tuple)) else x, dtype=torch.int32, device="cuda")


def filled(cca, n_pages, size, B, wide, seed=0):
    """A pool whose pages all hold numbers, free ones too."""
    pages = cca.new_pages(n_pages, size, B, wide)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for n in ("k", "v"):
        pages[n].normal_(generator=gen)
    return pages


def same(pages, pool):
    torch.cuda.synchronize()
    for n in ("refs", "table", "len"):
        assert pages[n].tolist() == getattr(pool, n), n
    for n in ("k", "v"):
        assert torch.equal(pages[n].cpu().view(torch.int16), getattr(pool, n).view(torch.int16)), n


def bits(t):
    return t.cpu().view(torch.int16)


# ------------------------------------------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("hk,dh", [(2, 32), (1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("size", [1, 3, 16, 40])
@pytest.mark.parametrize("n", [1, 17, 50])
def test_append_and_read(hk, dh, size, n):
    cca = make(hk, dh)
    B, room = 3, 90
    wide = -(-room // size)
    pages = filled(cca, B * wide + 2, size, B, wide)
    ws = cca.alloc_pages_workspace(B * wide + 2, B, wide)
    cca.pages_reserve(pages, room, ws)
    pages["table"].copy_(pages["table"].flatten()[torch.randperm(B * wide, device="cuda")].view(B, wide))
    pages["len"].copy_(ints(0, 5, room - n))
    pool = P.Pool.of(pages)
    gen = torch.Generator().manual_seed(n)
    k, v = (torch.randn(B, n, hk, dh, generator=gen).bfloat16() for _ in range(2))
    k[0, 0, 0, 0], v[1, 0, 0, 1] = float("nan"), float("inf")
    cca.paged_append(pages, k.cuda(), v.cuda())
    assert pool.append(k, v) == 0
    same(pages, pool)
    for got, want in zip(cca.paged_read(pages, n), (k, v)):
        assert torch.equal(bits(got), bits(want))
    first = [room - 3, -2, 4]
    for got, want in zip(cca.paged_read(pages, 9, ints(first)), pool.read(9, first)):
        assert torch.equal(bits(got), bits(want))
    assert cca.last_status() == 0
    cca.close()


@pytest.mark.parametrize("size", [50001, 65536, 4097, 3])
def test_rows_far_into_a_sequence(size):
    """Up to the last of 2^24 rows: which page a row lies in, and where."""
    cca = make(1, 32)
    wide = (1 << 24) // size
    at = [0, wide // 2, wide - 2, wide - 1]
    n_pages = min(len(at) + 1, (1 << 31) // size - 1)
    pages = filled(cca, n_pages, size, 4, wide)
    for b, i in enumerate(at):
        pages["table"][:, i] = b
    pages["refs"].copy_(ints([1] * 4 + [0]))
    k, v = (torch.randn(4, 5, 1, 32).bfloat16() for _ in range(2))
    lens = [at[0] * size, at[1] * size + 1, at[2] * size + size - 3, at[3] * size + size - 5]       # the third runs on from one page to the next
    if size == 3:
        lens = [0, at[1] * size, at[2] * size + 1, at[3] * size - 2]
    pages["len"].copy_(ints(lens))
    pool = P.Pool.of({n: t if n != "table" else t[:1] for n, t in pages.items()})
    pool.table = pool.table * 4
    for b in range(4):                                         # one after the other, the sequences share their pages here
        one = {**pages, "table": pages["table"][b:b + 1], "len": pages["len"][b:b + 1]}
        cca.paged_append(one, k[b:b + 1].cuda(), v[b:b + 1].cuda())
        for i in range(5):
            place = pool.place(b, lens[b] + i)
            if place is not None:
                pool.k[place[0], :, place[1]], pool.v[place[0], :, place[1]] = k[b, i], v[b, i]
    torch.cuda.synchronize()
    for n in ("k", "v"):
        assert torch.equal(bits(pages[n]), getattr(pool, n).view(torch.int16))
    for got, want in zip(cca.paged_read(pages, 7, ints([n - 1 for n in lens])), pool.read(7, [n - 1 for n in lens])):
        assert torch.equal(bits(got), bits(want))
    cca.close()


def test_append_leaves_out_what_it_may_not_write():
    """Counts of a padded batch; rows on shared pages, without a page, on a page that is none of the pool's, behind the table, behind a
    negative length."""
    cca = make()
    pages = filled(cca, 12, 4, 8, 3)
    pages["table"].copy_(torch.tensor([[0, 1, 2], [3, 4, -1], [5, 4, -1], [6, 12, 7], [8, -7, 9], [10, 2147483647, -1], [11, -1, -1], [-1, -1, -1]]))
    pages["refs"].copy_(ints(1, 1, 1, 1, 2, 1, 1, 1, 1, 1, 1, 1))
    pages["len"].copy_(ints(9, 2, 3, 3, 3, 3, -1, 0))
    pool = P.Pool.of(pages)
    k, v = (torch.randn(8, 5, 2, 64).bfloat16() for _ in range(2))
    for count, status in (([3, 0, 1, 1, 1, 1, -4, 0], 0), ([9, 9, 9, 9, 9, 9, 9, 9], 122), (None, 122)):
        cca.paged_append(pages, k.cuda(), v.cuda(), None if count is None else ints(count))
        assert pool.append(k, v, count) == status
        same(pages, pool)
        assert cca.last_status() == status and cca.last_status() == 0
        k, v = v, k
    got = cca.paged_read(pages, 13, ints(0, 0, 0, 0, 0, 0, -1, 0))
    for g, w in zip(got, pool.read(13, [0, 0, 0, 0, 0, 0, -1, 0])):
        assert torch.equal(bits(g), bits(w))
    assert cca.last_status() == 0
    cca.close()


# ------------------------------------------------------------------------------------------------ reserve, fork, free, compact
@pytest.mark.parametrize("n_pages,size,B,wide,seed", [(1, 4, 1, 1, 0), (9, 1, 3, 5, 1), (60, 7, 6, 9, 2), (300, 16, 40, 12, 3), (5000, 3, 70, 100, 4),
                                                      (20000, 2, 9, 3000, 5)])
def test_a_life_of_calls(n_pages, size, B, wide, seed):
    """Calls in any order, some of them asking for more than there is, each compared with the oracle."""
    cca = make(1, 32)
    rng = random.Random(seed)
    pages = filled(cca, n_pages, size, B, wide, seed)
    ws = cca.alloc_pages_workspace(n_pages, B, wide)
    ws.fill_(255)
    pool = P.Pool.of(pages)
    most = wide * size
    for step in range(40):
        do = rng.choice(["reserve", "reserve", "fork", "free", "compact", "grow"])
        status = 0
        if do == "reserve":
            n = rng.choice([1, 2, size, rng.randint(1, most)])
            count = [rng.randint(-2, n + 2) for _ in range(B)] if rng.random() < 0.7 else None
            first = [rng.randint(-1 if rng.random() < 0.1 else 0, max(0, most - n)) for _ in range(B)] if rng.random() < 0.3 else None
            cca.pages_reserve(pages, n, ws, None if count is None else ints(count), None if first is None else ints(first))
            status = pool.reserve(n, count, first)
        elif do == "fork":
            m = rng.randint(1, B)
            parent = [rng.randrange(B) if rng.random() > 0.02 else rng.choice([-1, B]) for _ in range(m)]
            child = [rng.randrange(B) if rng.random() > 0.02 else rng.choice([-1, B]) for _ in range(m)]
            cca.pages_fork(pages, ints(parent), ints(child), ws)
            status = pool.fork(parent, child)
        elif do == "free":
            keep = [rng.choice([-1, -1, 0, rng.randint(0, most)]) for _ in range(B)]
            cca.pages_free(pages, ints(keep))
            status = pool.free(keep)
        elif do == "compact":
            used = cca.pages_compact(pages, ws)
            assert used.tolist() == [pool.compact()]
        else:                                                  # tokens come in: as far as there are pages
            for b in range(B):
                n = 0
                while pool.place(b, pool.len[b] + n) and n < 3 * size:
                    n += 1
                pool.len[b] += rng.randint(0, n)
            pages["len"].copy_(ints(pool.len))
        same(pages, pool)
        got = cca.last_status()
        assert got == status or {got, status} <= {122, 123}, (step, do)      # of two reasons either may be told
        assert pool.refs == [sum(r.count(p) for r in pool.table) for p in range(n_pages)] if n_pages < 400 else True
    cca.close()


def test_reserve_copies_shared_pages_and_gives_the_last_its_own():
    cca = make(2, 128)
    pages = filled(cca, 40, 16, 8, 4)
    ws = cca.alloc_pages_workspace(40, 8, 4)
    cca.pages_reserve(pages, 37, ws, ints(37, 0, 0, 0, 0, 0, 0, 0))
    pages["len"].copy_(ints(37, 0, 0, 0, 0, 0, 0, 0))
    cca.pages_fork(pages, ints([0] * 7), ints([1, 2, 3, 4, 5, 6, 7]), ws)
    pool = P.Pool.of(pages)
    assert pool.refs[:3] == [8, 8, 8] and pool.len == [37] * 8
    cca.pages_reserve(pages, 1, ws, ints(1, 1, 1, 0, 1, 1, 1, 1))            # one of them does not go on: nobody keeps the page
    assert pool.reserve(1, [1, 1, 1, 0, 1, 1, 1, 1]) == 0
    same(pages, pool)
    assert pool.refs[2] == 1 and pool.table[3][2] == 2
    cca.pages_reserve(pages, 37, ws, first=ints([0] * 8))                    # everything of its own: the last keeps the rest
    assert pool.reserve(37, first=[0] * 8) == 0
    same(pages, pool)
    assert pool.table[7][:2] == [0, 1] and max(pool.refs) == 1
    assert cca.last_status() == 0
    cca.close()


def test_reserve_takes_all_or_nothing():
    cca = make()
    pages = filled(cca, 6, 4, 3, 4)
    ws = cca.alloc_pages_workspace(6, 3, 4)
    pool = P.Pool.of(pages)
    cca.pages_reserve(pages, 9, ws)                            # 9 pages of 6
    torch.cuda.synchronize()
    assert cca.last_status() == 123
    same(pages, pool)
    cca.pages_reserve(pages, 8, ws)                            # exactly all
    assert pool.reserve(8) == 0
    same(pages, pool)
    assert cca.last_status() == 0 and pool.refs == [1] * 6
    cca.pages_reserve(pages, 17, ws)                           # behind the table's end
    torch.cuda.synchronize()
    assert cca.last_status() == 122
    same(pages, pool)
    cca.close()


def test_sequences_not_in_use():
    """A negative length: skipped by every call that goes by it, without a word."""
    cca = make(1, 32)
    pages = filled(cca, 9, 2, 4, 3)
    ws = cca.alloc_pages_workspace(9, 4, 3)
    cca.pages_reserve(pages, 5, ws, ints(5, 3, 0, 5))
    pages["len"].copy_(ints(3, -1, -5, 2))
    pool = P.Pool.of(pages)
    k, v = (torch.randn(4, 2, 1, 32).bfloat16() for _ in range(2))
    cca.pages_reserve(pages, 2, ws)
    cca.paged_append(pages, k.cuda(), v.cuda())
    cca.pages_free(pages, ints(9, 1, 0, -1))
    assert pool.reserve(2) == 0 and pool.append(k, v) == 0 and pool.free([9, 1, 0, -1]) == 0
    same(pages, pool)
    assert cca.last_status() == 0 and pages["len"].tolist() == [3, -1, -5, 2]
    cca.pages_fork(pages, ints(1), ints(0), ws)
    cca.pages_reserve(pages, 1, ws, first=ints(0, -1, 0, 0))
    assert pool.fork([1], [0]) == 122 and pool.reserve(1, first=[0, -1, 0, 0]) == 122
    same(pages, pool)
    assert cca.last_status() == 122
    cca.close()


def test_tables_that_name_no_page_of_the_pool():
    """Entries outside the pool, counts that do not agree with the table: no access outside, and what is held stays in order."""
    cca = make(1, 32)
    pages = filled(cca, 9, 2, 3, 4)
    pages["table"].copy_(torch.tensor([[0, 9, -5, 2147483647], [1, -2147483648, 2, -1], [3, 3, -1, -1]]))
    pages["refs"].copy_(ints(1, 1, 1, 1, 0, 0, 0, 0, -3))
    pages["len"].copy_(ints(8, 5, 4))
    ws = cca.alloc_pages_workspace(9, 3, 4)
    pool = P.Pool.of(pages)
    cca.pages_fork(pages, ints(0, 9, 1), ints(1, 1, -1), ws)
    assert pool.fork([0, 9, 1], [1, 1, -1]) == 122
    same(pages, pool)
    assert cca.last_status() == 122
    cca.pages_free(pages, ints(-1, -1, 0))                     # page 3 twice, held once
    assert pool.free([-1, -1, 0]) == 122
    same(pages, pool)
    assert cca.last_status() == 122
    cca.pages_reserve(pages, 8, ws, first=ints(0, 0, 0), count=ints(8, 0, 0))
    assert pool.reserve(8, [8, 0, 0], [0, 0, 0]) == 0
    same(pages, pool)
    assert cca.last_status() == 0
    cca.close()


@pytest.mark.parametrize("n_pages,B,wide,every", [(70000, 3, 30000, 3), (1 << 20, 2, 600000, 2), (1025, 5, 1000, 1)])
def test_large_pools(n_pages, B, wide, every):
    """Pools that take many rounds of a cluster: a compaction and a reservation, checked with torch."""
    cca = make(1, 32)
    pages = cca.new_pages(n_pages, 1, B, wide)
    ws = cca.alloc_pages_workspace(n_pages, B, wide)
    gen = torch.Generator(device="cuda").manual_seed(wide)
    held = torch.arange(0, n_pages, every, device="cuda")
    held = held[torch.randperm(len(held), generator=gen, device="cuda")][:B * wide]
    flat = torch.full((B * wide,), -1, dtype=torch.int32, device="cuda")
    flat[:len(held)] = held.int()
    pages["table"].copy_(flat.view(B, wide))
    pages["refs"][held] = 1
    mark = torch.arange(n_pages, device="cuda")
    for n, x in (("k", 0), ("v", 10)):
        pages[n].view(torch.int32)[:, 0, 0, :] = ((mark << 1) + x)[:, None].int()
    used = cca.pages_compact(pages, ws)
    torch.cuda.synchronize()
    U = len(held)
    assert used.tolist() == [U] and int(pages["refs"][:U].min()) == 1 and not pages["refs"][U:].any()
    stay = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    stay[held] = True
    to = torch.arange(n_pages, device="cuda")
    to[(stay & (mark >= U)).nonzero().flatten()] = (~stay & (mark < U)).nonzero().flatten()
    assert torch.equal(pages["table"].flatten()[:U].long(), to[held])
    for n, x in (("k", 0), ("v", 10)):
        assert torch.equal(pages[n].view(torch.int32)[to[held], 0, 0, 5].long(), (held << 1) + x)
    # all of the first sequence's rows once more: only what it has no page for
    missing = int((pages["table"][0] < 0).sum())
    pages["len"].zero_()
    fits = missing <= n_pages - U
    cca.pages_reserve(pages, wide, ws, ints([wide] + [0] * (B - 1)))
    torch.cuda.synchronize()
    assert cca.last_status() == (0 if fits else 123)
    if fits:
        assert torch.equal(pages["table"][0].long().sort().values, torch.arange(wide, device="cuda")) or missing == 0 or U > wide
        assert int(pages["refs"].sum()) == U + missing and int(pages["refs"].max()) == 1
    cca.close()


def test_large_pages_and_many_copies():
    """Pages of several blocks' copies, not a whole number of them."""
    cca = make(3, 64)
    pages = filled(cca, 30, 123, 5, 4)
    ws = cca.alloc_pages_workspace(30, 5, 4)
    cca.pages_reserve(pages, 400, ws, ints(400, 0, 0, 0, 0))
    pages["len"].copy_(ints(400, 0, 0, 0, 0))
    cca.pages_fork(pages, ints(0, 0, 0), ints(1, 3, 4), ws)
    pool = P.Pool.of(pages)
    cca.pages_reserve(pages, 400, ws, first=ints([0] * 5), count=ints(400, 400, 0, 130, 400))
    assert pool.reserve(400, [400, 400, 0, 130, 400], [0] * 5) == 0
    same(pages, pool)
    cca.pages_free(pages, ints(0, -1, -1, -1, 124))
    pool.free([0, -1, -1, -1, 124])
    assert cca.pages_compact(pages, ws).tolist() == [pool.compact()]
    same(pages, pool)
    assert cca.last_status() == 0
    cca.close()


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    from paper_2510_04476_b200.binding import CcaError
    cca = make()
    pages = cca.new_pages(8, 4, 2, 3)
    ws = cca.alloc_pages_workspace(8, 2, 3)
    k = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    keep = ints(0, 0)
    for match, call in [
        ("invalid", lambda: cca.pages_reserve(pages, 0, ws)),
        ("unsupported", lambda: cca.pages_reserve(pages, (1 << 24) + 1, ws)),
        ("workspace too small", lambda: cca.pages_reserve(pages, 1, ws[:300])),
        ("count", lambda: cca.pages_reserve(pages, 1, ws, ints(1))),
        ("first", lambda: cca.pages_reserve(pages, 1, ws, first=torch.zeros(2, dtype=torch.int64, device="cuda"))),
        ("workspace too small", lambda: cca.pages_compact(pages, ws[:300])),
        ("used", lambda: cca.pages_compact(pages, ws, ints(1, 2))),
        ("invalid", lambda: cca.pages_fork(pages, ints([]), ints([]), ws)),
        ("invalid", lambda: cca.pages_fork(pages, ints(0, 0, 0), ints(1, 1, 1), ws)),
        ("parent", lambda: cca.pages_fork(pages, ints(0), ints(1, 1), ws)),
        ("workspace", lambda: cca.pages_fork(pages, ints(0), ints(1), ws.cpu())),
        ("keep", lambda: cca.pages_free(pages, ints(0))),
        ("k: wants", lambda: cca.paged_append(pages, k.float(), k)),
        ("v: wants", lambda: cca.paged_append(pages, k, k[:1])),
        ("invalid", lambda: cca.paged_append(pages, k[:, :0], k[:, :0])),
        ("invalid", lambda: cca.paged_append(pages, *[torch.zeros(2, 13, 2, 64, dtype=torch.bfloat16, device="cuda")] * 2)),
        ("invalid", lambda: cca.paged_read(pages, 0)),
        ("invalid", lambda: cca.paged_read(pages, -1)),
        ("contiguous", lambda: cca.paged_read({**pages, "k": pages["k"][:, :, ::2]}, 1)),
        ("refs", lambda: cca.pages_free({**pages, "refs": pages["refs"][:7]}, keep)),
        ("len", lambda: cca.pages_free({**pages, "len": pages["len"][:1]}, keep)),
        ("v: wants", lambda: cca.pages_free({n: t for n, t in pages.items() if n != "v"}, keep)),
    ]:
        with pytest.raises(CcaError, match=match):
            call()
    before = cca.launch_count()
    n = torch.zeros(1 << 20, dtype=torch.bfloat16, device="cuda")
    off = {**pages, "k": n[4:4 + pages["k"].numel()].view_as(pages["k"])}          # not on a 16-byte boundary
    with pytest.raises(CcaError, match="align"):
        cca.pages_free(off, keep)
    assert cca.launch_count() == before and cca.last_status() == 0
    cca.close()


# ------------------------------------------------------------------------------------------------ streams, graphs, a part of the sequences
def test_on_another_stream_in_a_graph_and_again():
    """Captured once, replayed over states that change in between; two graphs share one workspace."""
    cca = make(2, 32)
    pages = filled(cca, 64, 4, 6, 8)
    ws = cca.alloc_pages_workspace(64, 6, 8)
    side = torch.cuda.Stream()
    parent, child, keep = ints(0, 1, 2), ints(3, 4, 5), ints(-1, 5, -1, 0, 3, -1)
    used = ints(0)
    cca.pages_reserve(pages, 9, ws)                            # (kernels are loaded before the capture)
    cca.pages_fork(pages, parent, child, ws)
    cca.pages_free(pages, keep)
    cca.pages_compact(pages, ws, used)
    torch.cuda.synchronize()
    graphs = []
    for calls in ((lambda: (cca.pages_reserve(pages, 3, ws), cca.pages_fork(pages, parent, child, ws))),
                  (lambda: (cca.pages_free(pages, keep), cca.pages_compact(pages, ws, used)))):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            calls()
        graphs.append(g)
    pool = P.Pool.of(pages)
    for turn in range(4):
        pool.len = [min(27, 2 + 3 * turn + b) if turn < 2 else n for b, n in enumerate(pool.len)]
        pages["len"].copy_(ints(pool.len))
        torch.cuda.synchronize()
        graphs[0].replay()
        status = pool.reserve(3) or 0
        pool.fork([0, 1, 2], [3, 4, 5])
        same(pages, pool)
        graphs[1].replay()
        pool.free(keep.tolist())
        want = pool.compact()
        same(pages, pool)
        assert used.tolist() == [want] and cca.last_status() == status
    cca.close()


def test_some_sequences_on_their_own():
    cca = make(2, 32)
    pages = filled(cca, 20, 4, 5, 4)
    ws = cca.alloc_pages_workspace(20, 5, 4)
    part = {**pages, "table": pages["table"][2:4], "len": pages["len"][2:4]}
    cca.pages_reserve(part, 6, ws)
    k, v = (torch.randn(2, 6, 2, 32, device="cuda").bfloat16() for _ in range(2))
    cca.paged_append(part, k, v)
    part["len"].fill_(6)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    assert pages["table"].tolist() == [[-1] * 4, [-1] * 4, [0, 1, -1, -1], [2, 3, -1, -1], [-1] * 4] and pages["len"].tolist() == [0, 0, 6, 6, 0]
    cca.pages_fork(pages, ints(3), ints(0), ws)
    got, _ = cca.paged_read({**pages, "table": pages["table"][:1], "len": pages["len"][:1]}, 6, ints(0))
    assert torch.equal(got, k[1:])
    cca.close()
