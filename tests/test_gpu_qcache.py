"""The 4-bit cache on the GPU against its fp64 oracle: rows in and out, attention with gathered weights, eviction, and what is refused.

Tolerances (derived, u = 2^-24 for fp32, a bf16 rounding is off by at most 2^-8 of the value):
* codes, scales, positions, moved rows: equal.
* o: each probability times its row's scale is rounded to fp16 once, and the output to bf16 once: |err| <= 2^-11 sum_r p |v| + 2^-8 |o|,
  plus the fp32 part below, plus what fp16 cannot resolve: the operands are scaled so that the largest p times the largest scale is
  2^7 or more, and below 2^-14 they are off by 2^-25 at most, codes are 7 at most: n 7 2^-32 max p max s for n rows.
* logits (in log2 units): sums of d products and d / 32 scalings in fp32 whose adds may truncate: |err| <= 2 u (d + 16) A with
  A = max_r sum |q k| log2(e) / sqrt(d); the maximum and the logarithm of the sum bring the same again plus 4 u (|logit| + 64) (the
  largest value scale's logarithm, -30 or more, and 2^7 are part of the maximum).  p: relative error ln 2 times that, plus 2^-21 (exp2, log2 of the hardware).
* weight: the relative error of p on every head's part, plus the rounding of the sum with what was there, 4 u |weight|.
"""
import math

import pytest
import torch

from oracle import q_oracle as Q

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _cca(hq, hk, dh):
    from paper_2510_04476_b200.binding import CCA
    return CCA(d_model=hq * dh, n_q_heads=hq, n_kv_heads=hk, head_dim=dh)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _filled(cca, B, S, lens, seed, scale=1.0, junk=True):
    """A cache with `lens` rows put in by the append call; behind them every byte is junk (NaN scales among it)."""
    gen = _gen(seed)
    hk, dh = cca.cfg.n_kv_heads, cca.cfg.head_dim
    n = max(max(lens), 1)
    k = (scale * torch.randn(B, n, hk, dh, generator=gen)).bfloat16()
    v = torch.randn(B, n, hk, dh, generator=gen).bfloat16()
    cache = cca.new_qcache(B, S)
    if junk:
        for name in ("k", "v"):
            cache[name + "_codes"].fill_(0xAB)
            cache[name + "_scales"].fill_(float("nan"))
        cache["weight"].fill_(float("nan"))
    cca.qcache_append(cache, k.cuda(), v.cuda(), count=torch.tensor(lens, dtype=torch.int32).cuda())
    cache["len"].copy_(torch.tensor(lens, dtype=torch.int32))
    return cache, k, v


def _stored(cache, name):
    """[B, hk, S, d] values of every row, decoded by the oracle from the cache's bytes."""
    return Q.values(Q.unpack(cache[name + "_codes"]), cache[name + "_scales"].cpu())


# ------------------------------------------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("hk,dh", [(2, 32), (1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("B,n,S", [(1, 1, 1), (3, 5, 17), (2, 130, 131)])
def test_append_and_read(hk, dh, B, n, S):
    cca = _cca(hk, hk, dh)
    gen = _gen(B * 100 + n + dh)
    k = (torch.randn(B, n, hk, dh, generator=gen) * torch.exp(2 * torch.randn(B, n, hk, 1, generator=gen))).bfloat16()
    v = torch.randn(B, n, hk, dh, generator=gen).bfloat16()
    k[0, 0, 0, 1] = float("inf")
    v[0, 0, 0, :32] = 0
    v[B - 1, n - 1, hk - 1, dh - 1] = float("nan")
    first = torch.tensor([(S - n) * b // max(1, B - 1) if B > 1 else 0 for b in range(B)], dtype=torch.int32)
    cache = cca.new_qcache(B, S)
    for t in cache.values():
        if t.dtype is not torch.int32:
            t.fill_(3)
    before = {name: t.clone() for name, t in cache.items()}
    cache["len"].copy_(first)
    pos0 = torch.arange(B, dtype=torch.int32) * 7 + 2
    cca.qcache_append(cache, k.cuda(), v.cuda(), pos0.cuda())
    got_k, got_v = cca.qcache_read(cache, n)
    torch.cuda.synchronize()
    assert cca.last_status() == 0 and torch.equal(cache["len"].cpu(), first)
    for name, x, got in (("k", k, got_k), ("v", v, got_v)):
        c, s = Q.quantise(x)
        ref = Q.values(c, s).float()
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=1e30), torch.nan_to_num(ref, nan=1e30))
        for b in range(B):
            f = int(first[b])
            rows = slice(f, f + n)
            assert torch.equal(cache[name + "_codes"][b, :, rows].cpu(), Q.pack(c[b].transpose(0, 1)))
            others = [r for r in range(S) if not f <= r < f + n]
            for t in ("_codes", "_scales"):
                assert torch.equal(cache[name + t][b, :, others], before[name + t][b, :, others])
    for b in range(B):
        f = int(first[b])
        assert not cache["weight"][b, :, f:f + n].any()
        assert torch.equal(cache["position"][b, :, f:f + n].cpu(), (pos0[b] + torch.arange(n, dtype=torch.int32)).expand(hk, n))
    cca.close()


def test_append_of_every_quotient():
    """Every pair of an 8-bit significand over an 8-bit scale that a group can hold: 128 largest values (each with another scale)
    against all numbers up to them, halves between two codes among them; and the same far down and far up in the range."""
    cca = _cca(1, 1, 64)
    mant = torch.arange(128, 256, dtype=torch.float64)
    top = mant.repeat_interleave(128 * 8)                            # the largest of a group
    x = mant.repeat(128)[:, None] * 2.0 ** -torch.arange(8, dtype=torch.float64)
    x = torch.minimum(x.reshape(-1), top)                            # 1024 numbers for each of 128 scales
    g = x.view(-1, 16)
    rows = torch.zeros(g.shape[0], 32, dtype=torch.float64)
    rows[:, :16] = g
    rows[:, 16:31] = -g[:, :15]
    rows[:, 31] = top.view(-1, 16)[:, 0]
    for scale in (1.0, 2.0 ** -90, 2.0 ** -104, 2.0 ** -130, 2.0 ** 52, 2.0 ** 119):
        k = (rows * scale).bfloat16().view(1, -1, 1, 64)
        cache = cca.new_qcache(1, k.shape[1])
        cca.qcache_append(cache, k.cuda(), k.cuda())
        c, s = Q.quantise(k)
        assert torch.equal(cache["k_scales"][0, 0].cpu().double(), s[0, :, 0]), scale
        assert torch.equal(cache["k_codes"][0, 0].cpu(), Q.pack(c[0, :, 0])), scale
    cca.close()


def test_append_of_a_padded_batch_and_rows_that_do_not_fit():
    cca = _cca(2, 2, 64)
    B, n, S = 5, 4, 10
    gen = _gen(1)
    k, v = (torch.randn(B, n, 2, 64, generator=gen).bfloat16().cuda() for _ in range(2))
    cache = cca.new_qcache(B, S)
    cache["len"].copy_(torch.tensor([0, 3, 7, -1, 8], dtype=torch.int32))
    count = torch.tensor([0, 2, 4, 1, 9], dtype=torch.int32).cuda()          # 9 is cut to n = 4; 7 + 4 and 8 + 4 pass the capacity
    cca.qcache_append(cache, k, v, count=count)
    torch.cuda.synchronize()
    assert cca.last_status() == 121 and cca.last_status() == 0
    written = (cache["k_codes"] != 0).any(-1)[:, 0].cpu()
    want = torch.zeros(B, S, dtype=torch.bool)
    want[1, 3:5] = True
    assert torch.equal(written, want)
    # without a count, and with an exact fit
    cache["len"].copy_(torch.tensor([6, 6, 6, 6, 6], dtype=torch.int32))
    cca.qcache_append(cache, k, v)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    assert torch.equal(cache["position"][2, 1, 6:].cpu(), torch.arange(6, 10, dtype=torch.int32))
    # a cache without weights and positions
    bare = {name: t for name, t in cache.items() if name not in ("weight", "position")}
    cca.qcache_append(bare, k, v, torch.zeros(B, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    # a negative position: that sequence is left as it is
    before = cache["k_codes"].clone()
    cca.qcache_append(cache, v, k, torch.tensor([0, 1, -5, 3, 4], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert cca.last_status() == 121
    assert torch.equal(cache["k_codes"][2], before[2]) and not torch.equal(cache["k_codes"][1], before[1])
    # positions up to the last that 32 bits hold, and one further
    before = cache["k_codes"].clone()
    top = (1 << 31) - 1
    cca.qcache_append(cache, k, v, torch.tensor([0, top - 3, top - 2, 3, 4], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert cca.last_status() == 121
    assert torch.equal(cache["k_codes"][2], before[2]) and not torch.equal(cache["k_codes"][1], before[1])
    assert cache["position"][1, 0, 6:].tolist() == [top - 3, top - 2, top - 1, top]
    cca.close()


def test_read_of_given_rows():
    cca = _cca(2, 2, 32)
    cache, k, _ = _filled(cca, 2, 9, [9, 4], 3)
    got, _ = cca.qcache_read(cache, 5, torch.tensor([6, -2], dtype=torch.int32).cuda())
    ref = _stored(cache, "k").transpose(1, 2).float()
    assert torch.equal(got[0, :3].cpu(), ref[0, 6:9]) and not got[0, 3:].any()
    assert not got[1, :2].any() and torch.equal(got[1, 2:].cpu(), ref[1, :3])
    cca.close()


# ------------------------------------------------------------------------------------------------ attention
def _check_attention(cca, cache, q, lens, o, weight_before, weight_after):
    hq, hk, dh = cca.cfg.n_q_heads, cca.cfg.n_kv_heads, cca.cfg.head_dim
    g = hq // hk
    n = max(max(lens), 1)
    k, v = _stored(cache, "k")[:, :, :n], _stored(cache, "v")[:, :, :n]
    o, wb, wa = o.cpu().double(), weight_before.cpu().double(), weight_after.cpu().double()
    ref, p = Q.attention(q, k, v, lens, g)
    for b, m in enumerate(lens):
        if m == 0:
            assert not o[b].any()
            assert torch.equal(torch.nan_to_num(wa[b], nan=7.0), torch.nan_to_num(wb[b], nan=7.0))
            continue
        grow = torch.zeros(hk, m, dtype=torch.float64)
        slack = torch.zeros(hk, m, dtype=torch.float64)
        for i in range(hq):
            j = i // g
            qi = q[b, i].double()
            A = float((qi.abs() * k[b, j, :m].abs()).sum(-1).max()) * math.log2(math.e) / math.sqrt(dh)
            rel = math.log(2) * (4 * U * (dh + 16) * A + 4 * U * (A + 64)) + 2.0 ** -21
            pv = p[b, i, :m] @ v[b, j, :m].abs()
            coarse = m * 7 * 2.0 ** -32 * float(p[b, i, :m].max()) * float(cache["v_scales"][b, j, :m].float().max())
            tol = (2.0 ** -11 + rel) * pv + 2.0 ** -8 * ref[b, i].abs() + coarse + 1e-30
            err = (o[b, i] - ref[b, i]).abs()
            assert (err <= tol).all(), (b, i, float((err / tol).max()))
            grow[j] += p[b, i, :m]
            slack[j] += rel * p[b, i, :m]
        err = (wa[b, :, :m] - (wb[b, :, :m] + grow)).abs()
        tol = slack + 4 * U * wa[b, :, :m].abs() + 2.0 ** -120        # what lies below the smallest normal number is dropped
        assert (err <= tol).all(), (b, float((err / tol).max()))
        rest = slice(m, None)
        assert torch.equal(torch.nan_to_num(wa[b, :, rest], nan=7.0), torch.nan_to_num(wb[b, :, rest], nan=7.0))


def _attend(cca, B, S, lens, seed, max_len=None, scale=1.0, qscale=1.0):
    cache, _, _ = _filled(cca, B, S, lens, seed, scale)
    gen = _gen(seed + 1)
    q = (qscale * torch.randn(B, cca.cfg.n_q_heads, cca.cfg.head_dim, generator=gen)).bfloat16()
    for b, n in enumerate(lens):
        cache["weight"][b, :, :n] = torch.rand(cca.cfg.n_kv_heads, n, generator=gen).cuda()
    before = cache["weight"].clone()
    max_len = max_len or S
    ws = cca.alloc_qcache_workspace(B, max_len)
    ws.fill_(255)                                  # NaN wherever a kernel reads what nobody wrote
    o = cca.qcache_attention(q.cuda(), cache, max_len, ws)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    _check_attention(cca, cache, q, lens, o, before, cache["weight"])
    return cache, q, ws, o


LENGTHS = [1, 2, 7, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200]


@pytest.mark.parametrize("hq,hk,dh", [(4, 4, 32), (8, 2, 64), (8, 2, 128), (4, 1, 256)])
def test_attention_at_every_kind_of_length(hq, hk, dh):
    cca = _cca(hq, hk, dh)
    lens = LENGTHS + [0]
    _attend(cca, len(lens), 201, lens, dh)
    cca.close()


@pytest.mark.parametrize("g", [1, 2, 3, 5, 7, 8, 9, 12, 16, 17, 33, 64])
@pytest.mark.parametrize("dh", [32, 64, 128, 256])
def test_attention_with_any_number_of_heads_per_group(g, dh):
    hk = 2 if g <= 32 else 1
    cca = _cca(g * hk, hk, dh)
    _attend(cca, 2, 150, [150, 83], g * 1000 + dh)
    cca.close()


@pytest.mark.parametrize("hq,hk,dh,B,S,lens,max_len", [
    (8, 2, 128, 1, 5000, [4999], 5000),
    (8, 2, 64, 3, 3001, [3001, 1, 1777], 3001),
    (4, 1, 256, 2, 2000, [1999, 1000], 2000),
    (4, 2, 32, 1, 30000, [29989], 29990),
    (8, 2, 128, 2, 4000, [50, 3], 64),               # short sequences in a large cache, a tight bound
    (8, 2, 128, 40, 70, [1 + b for b in range(40)], 70),
])
def test_attention_long_and_ragged(hq, hk, dh, B, S, lens, max_len):
    cca = _cca(hq, hk, dh)
    _attend(cca, B, S, lens, S, max_len)
    cca.close()


@pytest.mark.parametrize("qscale,scale", [(30.0, 30.0), (1e-3, 1e-3), (1e4, 1.0), (0.0, 1.0)])
def test_attention_with_sharp_and_flat_softmax(qscale, scale):
    """Logits far beyond what exp can hold (one row takes all), and all but equal ones."""
    cca = _cca(8, 2, 64)
    _attend(cca, 2, 700, [700, 333], 11, scale=scale, qscale=qscale)
    cca.close()


def test_attention_when_the_maximum_keeps_rising():
    """Keys ordered so that every row's logit passes the one before: the running maximum moves all the way."""
    cca = _cca(8, 2, 64)
    S = 900
    gen = _gen(2)
    q = torch.randn(1, 8, 64, generator=gen).abs().bfloat16()
    k = (torch.linspace(0, 40, S)[:, None, None] * torch.ones(S, 2, 64)).bfloat16()[None]
    v = torch.randn(1, S, 2, 64, generator=gen).bfloat16()
    cache = cca.new_qcache(1, S)
    cca.qcache_append(cache, k.cuda(), v.cuda())
    cache["len"].fill_(S)
    before = cache["weight"].clone()
    o = cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(1, S))
    _check_attention(cca, cache, q, [S], o, before, cache["weight"])
    cca.close()


@pytest.mark.parametrize("hq,hk,dh", [(4, 2, 32), (8, 2, 64), (8, 2, 128), (4, 1, 256), (24, 2, 64)])
@pytest.mark.parametrize("low,high", [(-12, 12), (-40, -30), (30, 45), (-25, 0)])
def test_attention_over_values_of_very_different_size(hq, hk, dh, low, high):
    """Every group of 32 channels of every row has a size of its own, within a row and from row to row."""
    cca = _cca(hq, hk, dh)
    B, S = 2, 333
    gen = _gen(dh + high)
    k, v = (torch.randn(B, S, hk, dh, generator=gen).bfloat16() for _ in range(2))
    v = v * torch.exp2(torch.randint(low, high + 1, (B, S, hk, dh // 32), generator=gen).float()).repeat_interleave(32, -1).bfloat16()
    v[:, 100:140] = 0
    cache = cca.new_qcache(B, S)
    cca.qcache_append(cache, k.cuda(), v.cuda())
    for lens in ([S, 140], [40, S]):
        cache["len"].copy_(torch.tensor(lens, dtype=torch.int32))
        q = torch.randn(B, hq, dh, generator=gen).bfloat16()
        before = cache["weight"].clone()
        o = cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(B, S))
        torch.cuda.synchronize()
        _check_attention(cca, cache, q, lens, o, before, cache["weight"])
    cca.close()


@pytest.mark.parametrize("dh", [64, 128, 256])
def test_attention_with_a_nan_value_touches_its_own_group_alone(dh):
    cca = _cca(4, 2, dh)
    cache, _, _ = _filled(cca, 2, 40, [40, 40], 5, junk=False)
    q = torch.randn(2, 4, dh, generator=_gen(6)).bfloat16().cuda()
    ws = cca.alloc_qcache_workspace(2, 40)
    want = cca.qcache_attention(q, cache, 40, ws)
    cache["v_scales"][0, 1, 7, 1] = float("nan")
    o = cca.qcache_attention(q, cache, 40, ws)
    assert torch.isnan(o[0, 2:, 32:64]).all()
    o[0, 2:, 32:64] = want[0, 2:, 32:64]
    # the NaN is no part of the maximum that the operands are scaled by, so that they may be rounded at another place: 2^-11 of the sum of
    # p |v| (below 7 max s = 4.5 here) and a rounding of the output that may fall to the other side
    assert ((o - want).abs() <= 2.0 ** -10 * 4.5 + 2.0 ** -7 * want.abs()).all()
    cca.close()


def test_attention_with_an_infinite_key_touches_its_own_head_alone():
    cca = _cca(4, 2, 64)
    cache, _, _ = _filled(cca, 2, 40, [40, 40], 5, junk=False)
    cache["k_scales"][0, 1, 7] = float("nan")
    q = torch.randn(2, 4, 64, generator=_gen(6)).bfloat16().cuda()
    o = cca.qcache_attention(q, cache, 40, cca.alloc_qcache_workspace(2, 40))
    assert torch.isnan(o[0, 2:]).all() and torch.isfinite(o[0, :2]).all() and torch.isfinite(o[1]).all()
    assert torch.isnan(cache["weight"][0, 1, :40]).all() and torch.isfinite(cache["weight"][0, 0]).all()
    cca.close()


def test_attention_without_weights_gives_the_same_output():
    cca = _cca(8, 2, 128)
    cache, q, ws, o = _attend(cca, 2, 300, [300, 123], 9)
    weight = cache["weight"].clone()
    o2 = cca.qcache_attention(q.cuda(), cache, 300, ws, accumulate=False)
    bare = {n: t for n, t in cache.items() if n not in ("weight", "position")}
    o3 = cca.qcache_attention(q.cuda(), bare, 300, ws)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(o, o3)
    assert torch.equal(torch.nan_to_num(weight, nan=7.0), torch.nan_to_num(cache["weight"], nan=7.0))
    cca.close()


def test_attention_is_the_same_every_time():
    cca = _cca(8, 2, 128)
    B, S = 3, 2049
    cache, q, ws, o = _attend(cca, B, S, [2049, 800, 2], 21)
    w0 = torch.zeros_like(cache["weight"])
    seen = []
    for _ in range(3):
        cache["weight"].copy_(w0)
        seen.append((cca.qcache_attention(q.cuda(), cache, S, ws), cache["weight"].clone()))
    for a, b in seen[1:]:
        assert torch.equal(a, seen[0][0]) and torch.equal(b, seen[0][1])
    assert torch.equal(seen[0][0], o)
    cca.close()


def test_attention_skips_a_length_outside_its_cache():
    cca = _cca(4, 2, 64)
    cache, _, _ = _filled(cca, 3, 20, [20, 5, 20], 4, junk=False)
    cache["len"].copy_(torch.tensor([17, -1, 16], dtype=torch.int32))
    q = torch.randn(3, 4, 64, generator=_gen(6)).bfloat16().cuda()
    out = torch.full((3, 4, 64), 3.0, dtype=torch.bfloat16).cuda()
    cca.qcache_attention(q, cache, 16, cca.alloc_qcache_workspace(3, 16), out=out)      # 17 and -1 are outside 0 .. 16
    torch.cuda.synchronize()
    assert cca.last_status() == 121 and cca.last_status() == 0
    assert (out[:2] == 3).all() and not (out[2] == 3).all()
    assert not cache["weight"][:2].any() and cache["weight"][2].any()
    cca.close()


def test_attention_far_into_a_large_cache():
    """The last sequence's rows lie beyond 2^32 bytes of codes."""
    cca = _cca(8, 4, 256)
    B, S = 2, 1 << 23
    dev = "cuda"
    cache = {"len": torch.zeros(B, dtype=torch.int32, device=dev),
             "weight": torch.empty(B, 4, S, dtype=torch.float32, device=dev), "position": torch.empty(B, 4, S, dtype=torch.int32, device=dev)}
    for n in ("k", "v"):
        cache[n + "_codes"] = torch.empty(B, 4, S, 128, dtype=torch.uint8, device=dev)
        cache[n + "_scales"] = torch.empty(B, 4, S, 8, dtype=torch.bfloat16, device=dev)
    assert cache["k_codes"][1, 3].data_ptr() - cache["k_codes"].data_ptr() > 1 << 32
    gen = _gen(8)
    k, v = (torch.randn(B, 40, 4, 256, generator=gen).bfloat16() for _ in range(2))
    cca.qcache_append(cache, k.cuda(), v.cuda())
    cache["len"].fill_(40)
    q = torch.randn(B, 8, 256, generator=gen).bfloat16()
    o = cca.qcache_attention(q.cuda(), cache, 64, cca.alloc_qcache_workspace(B, 64))
    small = {n: t[:, :, :40].contiguous() if t.dim() > 1 else t for n, t in cache.items()}
    _check_attention(cca, small, q, [40, 40], o, torch.zeros(B, 4, 40), small["weight"])
    # and rows at the far end of a head: put in, read back, moved by an eviction
    cache["len"].fill_(S - 40)
    cca.qcache_append(cache, v.cuda(), k.cuda())
    got, _ = cca.qcache_read(cache, 40)
    c, s = Q.quantise(v)
    assert torch.equal(got.cpu(), Q.values(c, s).float())
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    cca.close()


# ------------------------------------------------------------------------------------------------ eviction
def _random_cache(cca, B, S, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cache = cca.new_qcache(B, S)
    for n in ("k", "v"):
        cache[n + "_codes"].copy_(torch.randint(0, 256, cache[n + "_codes"].shape, generator=gen, device="cuda", dtype=torch.uint8))
        cache[n + "_scales"].copy_(torch.randn(cache[n + "_scales"].shape, generator=gen, device="cuda"))
    hk = cca.cfg.n_kv_heads
    cache["position"].copy_(torch.rand(B, hk, S, generator=gen, device="cuda").argsort(-1))
    cache["weight"].copy_(torch.randn(B, hk, S, generator=gen, device="cuda").exp())
    return cache


def _check_evict(cca, cache, lens, keep, recent, nxt, max_len=None):
    B, hk, S = cache["weight"].shape
    cache["len"].copy_(torch.tensor(lens, dtype=torch.int32))
    before = {n: t.clone().cpu() for n, t in cache.items()}
    max_len = max_len or S
    ws = cca.alloc_qcache_workspace(B, max_len)
    ws.fill_(255)
    cca.qcache_evict(cache, keep, recent, torch.tensor(nxt, dtype=torch.int32).cuda(), max_len, ws)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    want = {n: t.clone() for n, t in before.items()}
    moves = 0
    for b in range(B):
        for j in range(hk):
            for src, dst in Q.evict(before["weight"][b, j].tolist(), before["position"][b, j].tolist(), lens[b], keep, recent, nxt[b]):
                moves += 1
                for n in want:
                    if n != "len":
                        want[n][b, j, dst] = before[n][b, j, src]
        want["len"][b] = min(lens[b], keep)
    for n in want:
        got = cache[n].cpu()
        if n == "len":
            assert torch.equal(got, want[n])
        else:
            bits = {torch.float32: torch.int32, torch.bfloat16: torch.int16}.get(got.dtype)
            assert torch.equal(got.view(bits) if bits else got, want[n].view(bits) if bits else want[n]), n
    return moves


@pytest.mark.parametrize("dh", [32, 64, 128, 256])
@pytest.mark.parametrize("keep,recent", [(0, 0), (1, 0), (1, 1), (7, 3), (64, 64), (99, 10), (100, 0), (101, 50), (200, 9)])
def test_evict(dh, keep, recent):
    cca = _cca(4, 2, dh)
    cache = _random_cache(cca, 4, 101, keep * 10 + dh)
    _check_evict(cca, cache, [101, 100, 0, 33], keep, recent, [101, 100, 5, 60])
    cca.close()


@pytest.mark.parametrize("S,keep,recent", [(4097, 4096, 256), (5000, 1234, 100), (33000, 20000, 5000)])
def test_evict_long(S, keep, recent):
    cca = _cca(4, 2, 64)
    cache = _random_cache(cca, 2, S, S)
    assert _check_evict(cca, cache, [S, S - 3], keep, recent, [S, S + 10]) > 0
    cca.close()


def test_evict_of_a_cache_beyond_the_shared_memory():
    cca = _cca(2, 1, 32)
    S = 70001
    cache = _random_cache(cca, 1, S, 3)
    assert _check_evict(cca, cache, [S], 40000, 1000, [S]) > 0
    cca.close()


def test_evict_of_long_caches_of_a_full_batch():
    """More heads than the chip has room for clusters, and more rows than a CTA has shared memory for keys."""
    cca = _cca(1, 1, 32)
    B, S = 150, 50011
    cache = _random_cache(cca, B, S, 9)
    cache["weight"][7] = cache["weight"][7].round()          # many equal ones
    lens = [10 + b for b in range(B)]
    lens[7], lens[149], lens[60] = S, S - 1, 48000          # CTAs' warps take more than 1024 rows each
    assert _check_evict(cca, cache, lens, 30000, 700, [S] * B) > 0
    cca.close()


def test_evict_odd_weights():
    """Equal weights (the lower row stays), zeros of both signs, NaN, infinities, negative ones."""
    cca = _cca(2, 2, 64)
    S = 300
    cache = _random_cache(cca, 3, S, 3)
    odd = torch.tensor([0.0, -0.0, float("nan"), float("inf"), -float("inf"), -1.0, 1.0, 1e-45, -1e-45, 3e38])
    cache["weight"].copy_(odd[torch.randint(0, 10, cache["weight"].shape, generator=_gen(4))])
    cache["weight"][1] = 2.5
    cache["weight"][2] = float("nan")
    for keep, recent in ((150, 0), (150, 40), (299, 100), (10, 10)):
        _check_evict(cca, {n: t.clone() for n, t in cache.items()}, [S, S - 1, S], keep, recent, [S, S, S])
    cca.close()


def test_evict_when_more_rows_are_recent_than_are_kept():
    cca = _cca(2, 2, 32)
    cache = _random_cache(cca, 1, 64, 5)
    cache["position"].fill_(9)
    _check_evict(cca, cache, [64], 20, 20, [9])
    # positions at the ends of 32 bits: the border is computed in more
    cache = _random_cache(cca, 2, 64, 6)
    cache["position"][0] = -(1 << 31)
    _check_evict(cca, cache, [64, 64], 20, 20, [-(1 << 31) + 5, (1 << 31) - 1])
    cca.close()


def test_evict_again_and_again_then_attend():
    """As decoding does it: a row in, attention, one row out; the rows that remain give the oracle's attention."""
    cca = _cca(4, 2, 64)
    B, S, keep = 2, 41, 40
    cache, _, _ = _filled(cca, B, S, [keep, keep], 31, junk=False)
    gen = _gen(32)
    ws = cca.alloc_qcache_workspace(B, S)
    pos = torch.full((B,), keep, dtype=torch.int32).cuda()
    for step in range(30):
        k, v = (torch.randn(B, 1, 2, 64, generator=gen).bfloat16().cuda() for _ in range(2))
        cca.qcache_append(cache, k, v, pos)
        pos += 1
        cache["len"] += 1
        q = (2 * torch.randn(B, 4, 64, generator=gen)).bfloat16()
        before = cache["weight"].clone()
        o = cca.qcache_attention(q.cuda(), cache, S, ws)
        _check_attention(cca, cache, q, [S, S], o, before, cache["weight"])
        cca.qcache_evict(cache, keep, 8, pos, S, ws)
    assert torch.equal(cache["len"].cpu(), torch.full((B,), keep, dtype=torch.int32))
    recent = cache["position"][:, :, :keep].sort(-1).values[..., -8:]
    assert torch.equal(recent.cpu(), torch.arange(62, 70, dtype=torch.int32).expand(B, 2, 8))
    assert cca.last_status() == 0
    cca.close()


def test_evict_skips_a_length_outside_its_cache():
    cca = _cca(2, 2, 32)
    cache = _random_cache(cca, 3, 30, 7)
    cache["len"].copy_(torch.tensor([30, -4, 20], dtype=torch.int32))
    before = cache["k_codes"].clone()
    cca.qcache_evict(cache, 10, 0, torch.full((3,), 30, dtype=torch.int32).cuda(), 25, cca.alloc_qcache_workspace(3, 25))
    torch.cuda.synchronize()
    assert cca.last_status() == 121
    assert cache["len"].tolist() == [30, -4, 10]
    assert torch.equal(cache["k_codes"][:2], before[:2])
    cca.close()


# ------------------------------------------------------------------------------------------------ streams, graphs, refusals
def test_on_another_stream_and_in_graphs_that_share_a_workspace():
    cca = _cca(8, 2, 128)
    B, S = 2, 500
    a, q, ws, o_ref = _attend(cca, B, S, [500, 77], 51)
    b = {n: t.clone() for n, t in a.items()}
    nxt = torch.full((B,), S, dtype=torch.int32).cuda()
    q = q.cuda()
    k, v = (torch.randn(B, 1, 2, 128, generator=_gen(52)).bfloat16().cuda() for _ in range(2))

    def step(cache, out):
        cca.qcache_attention(q, cache, S, ws, out=out)
        cca.qcache_evict(cache, 60, 10, nxt, S, ws)
        cca.qcache_append(cache, k, v, nxt)

    outs = [torch.empty(B, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ref = {n: t.clone() for n, t in a.items()}
    want = torch.empty_like(outs[0])
    step(ref, want)
    side = torch.cuda.Stream()
    start = {n: t.clone() for n, t in a.items()}
    torch.cuda.synchronize()
    graphs = []
    for cache, out in ((a, outs[0]), (b, outs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(cache, out)
        graphs.append(g)
    for rep in range(2):                       # the second replay starts from the same cache
        for cache in (a, b):
            for n in cache:
                cache[n].copy_(start[n])
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for cache, out in ((a, outs[0]), (b, outs[1])):
            assert torch.equal(out, want)
            for n in cache:
                assert torch.equal(torch.nan_to_num(cache[n].float(), nan=7.0), torch.nan_to_num(ref[n].float(), nan=7.0)), n
    assert torch.equal(want, o_ref)
    with torch.cuda.stream(side):
        other = {n: t.clone() for n, t in start.items()}
        out = cca.qcache_attention(q, other, S, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and cca.last_status() == 0
    cca.close()


def test_refusals():
    from paper_2510_04476_b200.binding import CcaError
    cca = _cca(4, 2, 64)
    B, S = 2, 16
    cache = cca.new_qcache(B, S)
    ws = cca.alloc_qcache_workspace(B, S)
    q = torch.zeros(B, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(B, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    nxt = torch.zeros(B, dtype=torch.int32, device="cuda")
    bare = {n: t for n, t in cache.items() if n not in ("weight", "position")}

    def no(fn, *args, match=None, **kw):
        with pytest.raises(CcaError, match=match):
            fn(*args, **kw)

    no(cca.qcache_attention, q, cache, S + 1, ws, match="invalid")
    no(cca.qcache_attention, q, cache, 0, ws, match="invalid")
    no(cca.qcache_attention, q, cache, S, ws[:300], match="workspace")
    no(cca.qcache_attention, q.float(), cache, S, ws, match="q:")
    no(cca.qcache_attention, q[:1], cache, S, ws, match="q:")
    no(cca.qcache_attention, q.transpose(1, 2).contiguous().transpose(1, 2), cache, S, ws, match="contiguous")
    no(cca.qcache_attention, q.cpu(), cache, S, ws, match="cuda")
    no(cca.qcache_attention, q, cache, S, ws.cpu(), match="workspace")
    no(cca.qcache_attention, q, bare, S, ws, accumulate=True, match="invalid")
    no(cca.qcache_attention, q, {**cache, "v_scales": cache["v_scales"].half()}, S, ws, match="v_scales")
    no(cca.qcache_attention, q, {**cache, "len": cache["len"].long()}, S, ws, match="len")
    no(cca.qcache_evict, bare, 4, 1, nxt, S, ws, match="invalid")
    no(cca.qcache_evict, cache, -1, 0, nxt, S, ws, match="invalid")
    no(cca.qcache_evict, cache, 4, 5, nxt, S, ws, match="invalid")
    no(cca.qcache_evict, cache, 4, -1, nxt, S, ws, match="invalid")
    no(cca.qcache_evict, cache, 4, 1, nxt, S + 1, ws, match="invalid")
    no(cca.qcache_evict, cache, 4, 1, nxt[:1], S, ws, match="next_position")
    no(cca.qcache_append, cache, kv, kv[:, :, :1], match="v:")
    no(cca.qcache_append, cache, kv[:, :0], kv[:, :0], match="invalid")
    no(cca.qcache_append, cache, kv.expand(B, S + 1, 2, 64).contiguous(), kv.expand(B, S + 1, 2, 64).contiguous(), match="invalid")
    no(cca.qcache_append, cache, kv, kv, count=nxt.long(), match="count")
    no(cca.qcache_read, cache, 0, match="invalid")
    odd = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device="cuda")[1:1 + q.numel()].view_as(q)
    no(cca.qcache_attention, odd, cache, S, ws, match="aligned")
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    cca.close()
