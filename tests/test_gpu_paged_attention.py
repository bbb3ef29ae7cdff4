"""Attention of one token per sequence over pages, on the GPU, against the fp64 oracle.

Tolerances (derived, u = 2^-24 for fp32; a bf16 rounding is off by at most 2^-8 of the value):
* logits (in log2 units): products are exact, d of them and a factor are added in fp32 with adds that may truncate: |err| <= e with
  e = 2 u (d + 16) A, A = max_r sum |q k| log2(e) / sqrt(d), plus 4 u (A + 64) where they are taken from the running maximum.
* a weight: relative error ln 2 times that of its logit, plus 2^-20 (the hardware's exp2 and the factors of a join), plus 2^-16 for
  its two bf16 parts.  The sum has the same; and n weighted rows are added in fp32, by truncating adds: n u.
* o: twice the weights' relative error times sum p |v|, plus the output's rounding, 2^-8 |o|.
* lse: ln 2 times the logits' error, plus 2^-20 for the sum's relative error, plus 4 u (|lse| + 64), plus n u.
"""
import math

import pytest
import torch

from oracle import pages_oracle as P
from tests.test_gpu_pages import ints, make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def cached(cca, size, lens, seed, spare=3, scale=1.0, wide=None, junk=True):
    """Sequences of `lens` rows on pages in any order; what no row lies in holds NaN."""
    gen = torch.Generator().manual_seed(seed)
    hk, dh = cca.cfg.n_kv_heads, cca.cfg.head_dim
    counts = [-(-n // size) for n in lens]
    n_pages = sum(counts) + spare
    pages = cca.new_pages(n_pages, size, len(lens), wide or max(1, max(counts)))
    for x in ("k", "v"):
        pages[x].copy_(((scale if x == "k" else 1.0) * torch.randn(n_pages, hk, size, dh, generator=gen)).bfloat16())
    order = torch.randperm(n_pages, generator=gen).int()
    used = torch.zeros(n_pages, size, dtype=torch.bool)
    table = torch.full(pages["table"].shape, -1, dtype=torch.int32)
    at = 0
    for b, (n, c) in enumerate(zip(lens, counts)):
        table[b, :c] = order[at:at + c]
        for i in range(c):
            used[order[at + i], :min(size, n - i * size)] = True
        at += c
    if junk:
        for x in ("k", "v"):
            pages[x].masked_fill_(~used.cuda()[:, None, :, None], float("nan"))
    pages["table"].copy_(table)
    pages["refs"].copy_(used.any(1).int())
    pages["len"].copy_(torch.tensor(lens, dtype=torch.int32))
    return pages


def check(cca, pages, q, lens, o, lse, only=None):
    pool, g = P.Pool.of(pages), cca.cfg.n_q_heads // cca.cfg.n_kv_heads
    dh = cca.cfg.head_dim
    o, lse = o.cpu().double(), None if lse is None else lse.cpu().double()
    for b, n in enumerate(lens):
        if only is not None and b not in only:
            continue
        k, v = pool.rows(b, n)
        want, want_lse, p = P.attention(q[b], k, v, g)
        if k.shape[1] == 0:
            assert not o[b].any() and (lse is None or bool((lse[b] == -math.inf).all())), b
            continue
        for i in range(q.shape[1]):
            A = float((k[i // g].abs() @ q[b, i].double().abs()).max()) * math.log2(math.e) / math.sqrt(dh)
            e = 2 * U * (dh + 16) * A + 4 * U * (A + 64)
            rel = math.log(2) * e + 2.0 ** -20 + 2.0 ** -16 + n * U
            tol = 2 * rel * (p[i] @ v[i // g].abs()) + 2.0 ** -8 * want[i].abs() + 1e-30
            err = (o[b, i] - want[i]).abs()
            assert bool((err <= tol).all()), (b, i, n, float((err / tol).max()))
            if lse is not None:
                tol = math.log(2) * e + 2.0 ** -20 + 4 * U * (abs(float(want_lse[i])) + 64) + n * U
                assert abs(float(lse[b, i] - want_lse[i])) <= tol, (b, i, n, float(lse[b, i]), float(want_lse[i]))


def attend(cca, size, lens, seed, max_len=None, scale=1.0, qscale=1.0, wide=None, status=0, pages=None):
    pages = pages or cached(cca, size, lens, seed, scale=scale, wide=wide)
    B, hq, dh = len(lens), cca.cfg.n_q_heads, cca.cfg.head_dim
    q = (qscale * torch.randn(B, hq, dh, generator=torch.Generator().manual_seed(seed + 1))).bfloat16()
    max_len = max_len or max(1, max(lens))
    ws = cca.alloc_paged_workspace(B, max_len)
    ws.fill_(255)                                              # NaN wherever a kernel reads what nobody wrote
    lse = torch.full((B, hq), 7.0, device="cuda")
    o = cca.paged_attention(q.cuda(), pages, max_len, ws, lse=lse)
    torch.cuda.synchronize()
    assert cca.last_status() == status
    check(cca, pages, q, lens, o, lse)
    return pages, q, ws, o, lse


LENGTHS = [1, 2, 7, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 256, 257, 0]


@pytest.mark.parametrize("hq,hk,dh", [(4, 4, 32), (8, 2, 64), (8, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("size", [1, 5, 16, 64, 300])
def test_every_kind_of_length_and_page(hq, hk, dh, size):
    cca = make(hk, dh, hq)
    attend(cca, size, LENGTHS, dh + size)
    cca.close()


@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 7, 8, 9, 11, 16, 17, 33, 64])
@pytest.mark.parametrize("dh", [32, 64, 128, 256])
def test_any_number_of_heads_per_group(g, dh):
    hk = 2 if g <= 32 else 1
    cca = make(hk, dh, g * hk)
    attend(cca, 16, [150, 83], g * 1000 + dh)
    cca.close()


@pytest.mark.parametrize("hq,hk,dh,size,lens,max_len", [
    (8, 2, 128, 64, [4999], 5000),
    (8, 2, 64, 16, [3001, 1, 1777], 3001),
    (4, 1, 256, 40, [1999, 1000], 2000),
    (4, 2, 32, 128, [29989], 29990),
    (8, 2, 128, 32, [50, 3], 64),                              # short sequences in a long table, a tight bound
    (8, 2, 128, 64, [1 + b for b in range(40)], 70),
    (2, 1, 64, 16, [(37 * b) % 91 for b in range(700)], 91),   # more sequences than a CTA has threads, empty ones among them
    (8, 1, 128, 48, [5000, 0, 0, 0, 0, 64, 3000], 5000),
    (8, 2, 128, 64, [16384], 16384),
    (4, 1, 128, 64, [9000 if b == 7 else (53 * b) % 200 for b in range(150)], 16384),      # a bound far above most lengths: units shared out
    (2, 1, 128, 32, [9000 if b == 290 else (53 * b) % 70 for b in range(300)], 16384),     # and more sequences than CTAs
    (12, 2, 64, 16, [3000] * 70, 16384),
])
def test_long_and_ragged(hq, hk, dh, size, lens, max_len):
    cca = make(hk, dh, hq)
    attend(cca, size, lens, len(lens) + dh, max_len, wide=-(-max_len // size) + 2)
    cca.close()


@pytest.mark.parametrize("qscale,scale", [(30.0, 30.0), (1e-3, 1e-3), (1e4, 1.0), (0.0, 1.0)])
def test_sharp_and_flat_softmax(qscale, scale):
    """Logits far beyond what exp can hold (one row takes all), and all but equal ones."""
    cca = make(2, 64, 8)
    attend(cca, 16, [300, 1000], 5, scale=scale, qscale=qscale)
    cca.close()


def test_rising_and_falling_logits():
    """The running maximum moves at every step, or never after the first row."""
    cca = make(1, 128, 2)
    for turn in (1, -1):
        pages = cached(cca, 16, [900], 1)
        q = torch.zeros(1, 2, 128)
        q[..., 0], q[..., 1] = 1.0, -1.0
        pool = pages["table"][0, :-(-900 // 16)].long()
        ramp = torch.arange(57 * 16, device="cuda").view(57, 16).float() * turn
        pages["k"][pool, 0, :, 0] = ramp.bfloat16()
        pages["k"][pool, 0, :, 1] = 0
        ws = cca.alloc_paged_workspace(1, 900)
        o = cca.paged_attention(q.bfloat16().cuda(), pages, 900, ws)
        torch.cuda.synchronize()
        check(cca, pages, q.bfloat16(), [900], o, None)
    cca.close()


def test_values_near_the_end_of_the_range():
    """A value of 2^127 in a row that a few later ones outweigh by a little: nothing overflows on the way."""
    cca = make(1, 64, 4)
    pages = cached(cca, 16, [200], 1)
    pool = pages["table"][0].long()
    pages["v"][pool[1], 0, 3, 5] = 2.0 ** 127
    q = torch.zeros(1, 4, 64)
    q[..., 0] = 1.0
    pages["k"][pool, 0, :, 0] = (torch.arange(13 * 16, device="cuda").view(13, 16) // 8).bfloat16()      # logits rise by 1/8 every 8 rows
    o = cca.paged_attention(q.bfloat16().cuda(), pages, 200, cca.alloc_paged_workspace(1, 200))
    assert bool(torch.isfinite(o).all()) and float(o[0, 0, 5]) > 2.0 ** 110
    check(cca, pages, q.bfloat16(), [200], o, None)
    cca.close()


def test_shared_pages():
    cca = make(2, 64, 8)
    pages = cached(cca, 16, [100, 40], 3, junk=False)
    pages["table"] = torch.cat([pages["table"], pages["table"][:1]])
    pages["len"] = ints(100, 40, 77)
    attend(cca, 16, [100, 40, 77], 4, pages=pages)
    cca.close()


def test_rows_without_a_page_are_left_out():
    """Entries outside the pool within a sequence; one sequence has nothing but them."""
    cca = make(2, 64, 8)
    pages = cached(cca, 16, [400, 90, 64, 33], 6)
    n = pages["refs"].numel()
    pages["table"][0, 2], pages["table"][0, 24], pages["table"][1, 0] = -1, n, -2147483648
    pages["table"][2, :4] = ints(-1, n + 5, 2147483647, -1)
    attend(cca, 16, [400, 90, 64, 33], 6, pages=pages, status=122)
    cca.close()


def test_lengths_outside_the_bound_are_skipped():
    cca = make(1, 64, 4)
    pages = cached(cca, 16, [50, 60, 70, 20], 2)
    pages["len"].copy_(ints(50, 61, -1, 20))
    q = torch.randn(4, 4, 64).bfloat16()
    ws = cca.alloc_paged_workspace(4, 60)
    out = torch.full((4, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, 4), 7.0, device="cuda")
    cca.paged_attention(q.cuda(), pages, 60, ws, out=out, lse=lse)
    torch.cuda.synchronize()
    assert cca.last_status() == 122
    assert bool((out[1:3] == 7).all()) and bool((lse[1:3] == 7).all())
    check(cca, pages, q, [50, 61, 0, 20], out, lse, only=(0, 3))
    # one that is not in use is no error, whichever way the rows are shared out
    for lens, max_len in (([50, 60, -1, 20], 60), ([50, 60, -7, 20], 64)):
        pages["len"].copy_(ints(lens))
        out.fill_(7)
        ws = cca.alloc_paged_workspace(4, max_len)
        cca.paged_attention(q.cuda(), pages, max_len, ws, out=out, lse=lse)
        torch.cuda.synchronize()
        assert cca.last_status() == 0 and bool((out[2] == 7).all())
        check(cca, pages, q, [50, 60, 0, 20], out, lse, only=(0, 1, 3))
    cca.close()


def test_sequences_not_in_use_among_long_ones():
    cca = make(1, 128, 4)
    lens = [9000 if b == 7 else (53 * b) % 200 for b in range(150)]
    pages = cached(cca, 64, lens, 5, wide=256)
    for b in range(0, 150, 3):
        pages["len"][b] = -1 - b
    q = torch.randn(150, 4, 128, generator=torch.Generator().manual_seed(1)).bfloat16()
    out = torch.full((150, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    cca.paged_attention(q.cuda(), pages, 16384, cca.alloc_paged_workspace(150, 16384), out=out)
    torch.cuda.synchronize()
    assert cca.last_status() == 0 and bool((out[::3] == 7).all())
    check(cca, pages, q, lens, out, None, only=[b for b in range(150) if b % 3])
    cca.close()


def test_numbers_that_are_none():
    """A NaN in a key spoils its kv head's queries alone, in a value its channel alone; an infinite key gives no number there."""
    cca = make(2, 64, 8)
    pages = cached(cca, 16, [200, 200, 200], 8)
    pages["k"][pages["table"][0, 1], 1, 3, 5] = float("nan")
    pages["v"][pages["table"][1, 1], 0, 3, 5] = float("nan")
    pages["k"][pages["table"][2, 0], 0, 0, 0] = float("inf")
    q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(1)).abs().bfloat16()
    ws = cca.alloc_paged_workspace(3, 200)
    o = cca.paged_attention(q.cuda(), pages, 200, ws).cpu()
    bad = torch.isnan(o)
    want = torch.zeros_like(bad)
    want[0, 4:] = True
    want[1, :4, 5] = True
    want[2, :4] = True
    assert torch.equal(bad, want)
    cca.close()


def test_the_same_every_time_on_any_stream_and_in_a_graph():
    cca = make(2, 128, 8)
    lens = [5000, 77, 0, 2300]
    pages, q, ws, o, lse = attend(cca, 64, lens, 11)
    qd = q.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = cca.paged_attention(qd, pages, 5000, ws)
    torch.cuda.synchronize()
    assert torch.equal(again, o)
    out, l2 = torch.empty_like(o), torch.empty_like(lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cca.paged_attention(qd, pages, 5000, ws, out=out, lse=l2)
    ws.fill_(255)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, o) and torch.equal(l2, lse)
    pages["len"].copy_(ints(4000, 70, 5, 0))                   # the next replay goes by what is there then
    pages["table"][2, 0] = pages["table"][0, 70]
    g.replay()
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    check(cca, pages, q, [4000, 70, 5, 0], out, l2)
    cca.close()


def test_a_longer_bound_and_a_larger_workspace_change_nothing():
    cca = make(2, 64, 8)
    lens = [700, 12, 333]
    pages, q, _, o, lse = attend(cca, 16, lens, 12, wide=200)
    for max_len in (701, 3000):
        l2 = torch.empty_like(lse)
        ws = cca.alloc_paged_workspace(9, 3200)
        ws.fill_(255)
        o2 = cca.paged_attention(q.cuda(), pages, max_len, ws, lse=l2)
        torch.cuda.synchronize()
        check(cca, pages, q, lens, o2, l2)
    cca.close()


def test_a_pool_of_more_than_2_to_the_32_elements():
    """Pages at the far end of pools of 8.7 GB each: offsets of elements and bytes pass 32 bits."""
    cca = make(2, 256, 4)
    size, n_pages = 64, 131500
    pages = {n: torch.empty(n_pages, 2, size, 256, dtype=torch.bfloat16, device="cuda") for n in ("k", "v")}
    pages.update(refs=torch.zeros(n_pages, dtype=torch.int32, device="cuda"), len=ints(0, 0),
                 table=torch.tensor([[n_pages - 1, 0, n_pages - 2], [65536, n_pages - 3, -1]], dtype=torch.int32, device="cuda"))
    pages["refs"][pages["table"][pages["table"] >= 0].long()] = 1
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn(2, 150, 2, 256, generator=gen).bfloat16() for _ in range(2))
    cca.paged_append(pages, k.cuda(), v.cuda(), ints(150, 128))
    for got, want in zip(cca.paged_read(pages, 150), (k, v)):
        assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1, :128].cpu(), want[1, :128])
    pages["len"].copy_(ints(150, 128))
    q = torch.randn(2, 4, 256, generator=gen).bfloat16()
    o = cca.paged_attention(q.cuda(), pages, 192, cca.alloc_paged_workspace(2, 192)).cpu().double()
    assert cca.last_status() == 0
    for b, n in enumerate((150, 128)):
        want, _, p = P.attention(q[b], *(x[b, :n].transpose(0, 1).double() for x in (k, v)), 2)
        assert bool(((o[b] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -12).all())
    ws = cca.alloc_pages_workspace(n_pages, 2, 3)
    assert cca.pages_compact(pages, ws).tolist() == [5]
    got, _ = cca.paged_read(pages, 150, ints(0, 0))
    assert torch.equal(got[0].cpu(), k[0]) and torch.equal(got[1, :128].cpu(), k[1, :128])
    cca.close()


def test_the_largest_batch():
    """65535 sequences, most of them short or empty."""
    cca = make(1, 32, 2)
    B = 65535
    lens = torch.arange(B) * 7919 % 23
    lens[::5] = 0
    pages = {n: torch.randn(4096, 1, 8, 32, device="cuda").bfloat16() for n in ("k", "v")}
    gen = torch.Generator().manual_seed(3)
    pages.update(refs=torch.ones(4096, dtype=torch.int32, device="cuda"), len=lens.int().cuda(),
                 table=torch.randint(0, 4096, (B, 3), generator=gen).int().cuda())
    q = torch.randn(B, 2, 32, generator=gen).bfloat16()
    for max_len in (22, 24):
        lse = torch.full((B, 2), 7.0, device="cuda")
        o = cca.paged_attention(q.cuda(), pages, max_len, cca.alloc_paged_workspace(B, max_len), lse=lse)
        torch.cuda.synchronize()
        assert cca.last_status() == 0
        for b in [*range(40), *range(30000, 30040), *range(B - 40, B)]:
            one = {**pages, "table": pages["table"][b:b + 1], "len": pages["len"][b:b + 1]}
            check(cca, one, q[b:b + 1], [int(lens[b])], o[b:b + 1], lse[b:b + 1])
        assert not o[(lens == 0).cuda()].any() and bool(torch.isinf(lse[(lens == 0).cuda()]).all())
    cca.close()


def test_two_streams_at_once():
    """Calls of one handle side by side, each stream with its own pages and workspace: the same as one after the other."""
    cca = make(2, 128, 8)
    sides = []
    for seed, lens in ((1, [5000, 300]), (2, [700, 16, 2200])):
        pages = cached(cca, 16, lens, seed)
        q = torch.randn(len(lens), 8, 128, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
        ws = cca.alloc_paged_workspace(len(lens), 5000)
        sides.append((torch.cuda.Stream(), pages, q, ws, max(lens), cca.paged_attention(q, pages, max(lens), ws)))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, (stream, pages, q, ws, n, _) in enumerate(sides):
            with torch.cuda.stream(stream):
                outs[i].append(cca.paged_attention(q, pages, n, ws))
    torch.cuda.synchronize()
    for got, side in zip(outs, sides):
        assert all(torch.equal(o, side[5]) for o in got)
    cca.close()


def test_refusals():
    from paper_2510_04476_b200.binding import CcaError
    cca = make(2, 64, 8)
    pages = cached(cca, 16, [30, 4], 1)
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    ws = cca.alloc_paged_workspace(2, 32)
    for match, call in [
        ("invalid", lambda: cca.paged_attention(q, pages, 0, ws)),
        ("invalid", lambda: cca.paged_attention(q, pages, 33, ws)),
        ("unsupported", lambda: cca.alloc_paged_workspace(1025, 1 << 20)),
        ("align", lambda: cca.paged_attention(torch.zeros(2 * 8 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 8, 64), pages, 32, ws)),
        ("workspace too small", lambda: cca.paged_attention(q, pages, 32, ws[:1000])),
        ("workspace", lambda: cca.paged_attention(q, pages, 32, ws.float())),
        ("q: wants", lambda: cca.paged_attention(q[:1], pages, 32, ws)),
        ("q: wants", lambda: cca.paged_attention(q.half(), pages, 32, ws)),
        ("out: wants", lambda: cca.paged_attention(q, pages, 32, ws, out=q.float())),
        ("lse: wants", lambda: cca.paged_attention(q, pages, 32, ws, lse=torch.zeros(2, 4, device="cuda"))),
        ("q: wants", lambda: cca.paged_attention(q.transpose(0, 1).contiguous().transpose(0, 1), pages, 32, ws)),
    ]:
        with pytest.raises(CcaError, match=match):
            call()
    assert cca.last_status() == 0
    cca.close()
    with pytest.raises(CcaError):
        cca.paged_attention(q, pages, 32, ws)
