"""Attention over the 4-bit cache where numbers are far apart: large logits beside large or small values, values of any size side by
side.  Bounds are derived (u = 2^-24 for fp32), against 64 bits:

* an output is rounded to bf16 once: half a step of the larger of the two numbers;
* a probability times a value's scale reaches the tensor cores in two bf16 parts, the second of which is rounded: 2^-15 of it at most
  (8 significant bits are cut off, what is left is below 2^-7 and rounded to 2^-8 of itself);
* the adds of the output's sums may truncate: 2 for every 16 rows of a warp and 8 + 128 in the joins, 2^-23 of sum p |v| each;
* probabilities are off by ln 2 times the logits' error, 4 u (d + 16) A + 4 u (A + 64) in units of log2, A = max sum |q k| log2(e) / sqrt(d),
  and by 2^-21 for exp2 and the reciprocal of the sum."""
import math

import pytest
import torch

from oracle import q_oracle as Q
from tests.test_gpu_qcache import U, _cca, _gen, _stored

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 32), (8, 2, 64), (8, 2, 128), (4, 1, 256), (24, 2, 64)]


def _half_step(x):
    """Half a step of bf16 at |x|."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -126))) - 8)


def _put(cca, k, v):
    B, S = k.shape[:2]
    cache = cca.new_qcache(B, S)
    cca.qcache_append(cache, k.cuda(), v.cuda())
    cache["len"].fill_(S)
    return cache


@pytest.mark.parametrize("hq,hk,dh", HEADS)
@pytest.mark.parametrize("S", [1, 40, 700, 3001])
@pytest.mark.parametrize("v_exp", [20, 0, -30])
def test_large_logits_beside_values_of_any_size(hq, hk, dh, S, v_exp):
    """Logits of 2^30 and more: one row has all the weight, and the output is that row, whatever its size."""
    cca = _cca(hq, hk, dh)
    gen = _gen(dh + S)
    k = (2.0 ** 15 * torch.randn(1, S, hk, dh, generator=gen)).bfloat16()
    v = (2.0 ** v_exp * torch.randn(1, S, hk, dh, generator=gen)).bfloat16()
    q = (2.0 ** 15 * torch.randn(1, hq, dh, generator=gen)).bfloat16()
    cache = _put(cca, k, v)
    o = cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(1, S)).cpu().double()
    assert cca.last_status() == 0
    ks, vs = _stored(cache, "k"), _stored(cache, "v")
    g = hq // hk
    for i in range(hq):
        terms = ks[0, i // g] * q[0, i].double()
        logits = terms.sum(-1) * math.log2(math.e) / math.sqrt(dh)
        top = logits.topk(min(2, S)).values
        A = float(terms.abs().sum(-1).max()) * math.log2(math.e) / math.sqrt(dh)
        if S > 1 and float(top[0] - top[1]) < 8 * U * (dh + 17) * A + 64:
            continue                              # too near each other for fp32: either may win
        want = vs[0, i // g, int(logits.argmax())]
        assert ((o[0, i] - want).abs() <= _half_step(torch.maximum(want.abs(), o[0, i].abs())) + (2.0 ** -15 + 2.0 ** -20) * want.abs()).all(), i
    cca.close()


@pytest.mark.parametrize("hq,hk,dh", HEADS)
@pytest.mark.parametrize("S", [33, 333, 2500])
@pytest.mark.parametrize("low,high", [(-45, 44), (-20, 20), (-45, -25), (25, 44)])
def test_values_of_any_size_side_by_side(hq, hk, dh, S, low, high):
    """Every group of 32 channels of every row has a size of its own: each output channel is as exact as if it were alone."""
    cca = _cca(hq, hk, dh)
    gen = _gen(dh + S + high)
    k, v = (torch.randn(1, S, hk, dh, generator=gen).bfloat16() for _ in range(2))
    v = v * torch.exp2(torch.randint(low, high + 1, (1, 1, hk, dh // 32), generator=gen).float()).repeat_interleave(32, -1).bfloat16()
    if S == 333:                                  # and from row to row
        v = v * torch.exp2(torch.randint(0, 4, (1, S, hk, 1), generator=gen).float()).bfloat16()
    q = (2 * torch.randn(1, hq, dh, generator=gen)).bfloat16()
    cache = _put(cca, k, v)
    o = cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(1, S)).cpu().double()
    assert cca.last_status() == 0
    ks, vs = _stored(cache, "k"), _stored(cache, "v")
    ref, p = Q.attention(q, ks, vs, [S], hq // hk)
    for i in range(hq):
        j = i // (hq // hk)
        A = float((q[0, i].double().abs() * ks[0, j].abs()).sum(-1).max()) * math.log2(math.e) / math.sqrt(dh)
        rel = math.log(2) * (4 * U * (dh + 16) * A + 4 * U * (A + 64)) + 2.0 ** -21
        tol = _half_step(torch.maximum(ref[0, i].abs(), o[0, i].abs())) + \
            (2.0 ** -15 + rel + 2.0 ** -23 * (S / 8 + 136)) * (p[0, i] @ vs[0, j].abs())
        err = (o[0, i] - ref[0, i]).abs()
        assert (err <= tol).all(), (i, float((err / tol).max()))
    cca.close()


@pytest.mark.parametrize("hq,hk,dh", HEADS)
def test_a_small_value_of_much_weight_beside_a_large_one_of_little(hq, hk, dh):
    """Rows 8 apart, one with a far larger logit, the other with a far larger value, so that both count for the output."""
    cca = _cca(hq, hk, dh)
    gen = _gen(dh)
    S, bits = 16, 40.0
    base = torch.ones(dh)
    q = torch.ones(1, hq, dh).bfloat16()
    unit = bits * math.sqrt(dh) / math.log2(math.e) / dh             # a key of `unit` everywhere gives a logit of `bits`
    k = torch.zeros(1, S, hk, dh)
    k[:, 3] = unit * base
    v = torch.zeros(1, S, hk, dh)
    v[:, 3] = torch.randn(1, hk, dh, generator=gen)
    v[:, 11] = 2.0 ** bits * torch.randn(1, hk, dh, generator=gen)
    cache = _put(cca, k.bfloat16(), v.bfloat16())
    o = cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(1, S)).cpu().double()
    ks, vs = _stored(cache, "k"), _stored(cache, "v")
    ref, p = Q.attention(q, ks, vs, [S], hq // hk)
    rel = math.log(2) * (4 * U * (dh + 16) * 2 * bits + 4 * U * (2 * bits + 64)) + 2.0 ** -21
    for i in range(hq):
        tol = _half_step(torch.maximum(ref[0, i].abs(), o[0, i].abs())) + (2.0 ** -15 + rel + 2.0 ** -23 * 138) * (p[0, i] @ vs[0, i // (hq // hk)].abs())
        assert ((o[0, i] - ref[0, i]).abs() <= tol).all(), (i, float(((o[0, i] - ref[0, i]).abs() / tol).max()))
    cca.close()
