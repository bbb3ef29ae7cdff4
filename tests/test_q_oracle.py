"""Pins of the 4-bit oracle: the format's byte order written out, its rounding bound, eviction on hand-made cases."""
import math

import pytest
import torch

from oracle import q_oracle as Q


@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_pack_places_every_channel_once(d):
    gen = torch.Generator().manual_seed(d)
    codes = torch.randint(-7, 8, (5, d), generator=gen)
    rows = Q.pack(codes)
    assert rows.shape == (5, d // 2) and rows.dtype == torch.uint8
    assert torch.equal(Q.unpack(rows), codes)
    assert sorted((b, m) for b, _, m in Q._places(d)) == [(b, m) for b in range(d // 2) for m in (0, 3)]


def test_pack_by_hand():
    codes = torch.zeros(128, dtype=torch.int64)
    codes[0], codes[2] = -5, 3           # group 0, i = 0, j = 0: byte 0
    codes[33 + 4 * 7] = 7                # group 1, i = 7, j = 1: byte 8 * 7 + 2 + 1
    rows = Q.pack(codes)
    assert int(rows[0]) == 0x80 | 5 | (3 << 3)
    assert int(rows[59]) == 7
    assert int(rows.sum()) == (0x80 | 5 | 24) + 7


def test_quantise_error_is_at_most_half_a_step():
    gen = torch.Generator().manual_seed(3)
    x = (torch.randn(64, 256, generator=gen) * torch.logspace(-3, 3, 64)[:, None]).bfloat16()
    c, s = Q.quantise(x)
    step = s.repeat_interleave(32, -1)
    # the scale is rounded to bf16 (2^-8 of itself): the largest channel may lie 7 * 2^-8 of a step beyond 7 steps
    assert ((Q.values(c, s) - x.double()).abs() <= step * 0.5 * (1 + 2**-20)).all()
    assert int(c.abs().max()) == 7


def test_quantise_edges():
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    x[1, 5] = float("inf")
    x[2, 6] = float("nan")
    x[3] = torch.linspace(-7, 7, 32).bfloat16()
    c, s = Q.quantise(x)
    assert float(s[0, 0]) == 0 and not c[0].any()
    assert math.isnan(float(s[1, 0])) and math.isnan(float(s[2, 0])) and not c[1:3].any()
    assert float(s[3, 0]) == 1.0 and int(c[3, 0]) == -7 and int(c[3, 31]) == 7


def test_evict_by_hand():
    w = [5.0, 1.0, 4.0, 1.0, 9.0, 0.0]
    pos = [0, 1, 2, 3, 4, 5]
    # the newest two are kept whatever they weigh; of the others the two heaviest
    assert Q.evict(w, pos, 6, 4, 2, 6) == [(4, 1), (5, 3)]
    # equal weights: the lower row stays
    assert Q.evict([1.0] * 6, pos, 6, 4, 0, 6) == []
    assert Q.evict([1.0] * 6, pos, 6, 4, 1, 6) == [(5, 3)]
    nan = float("nan")
    assert Q.evict([nan, 1.0, nan, float("-inf")], [0, 1, 2, 3], 4, 2, 0, 4) == [(3, 0)]
    assert Q.evict(w, pos, 4, 4, 2, 6) == []
    assert Q.evict(w, pos, 6, 0, 0, 6) == []


def test_attention_against_brute_force_and_empty():
    gen = torch.Generator().manual_seed(5)
    q, k, v = torch.randn(2, 4, 8, generator=gen), torch.randn(2, 2, 5, 8, generator=gen), torch.randn(2, 2, 5, 8, generator=gen)
    o, p = Q.attention(q, k, v, [3, 0], 2)
    assert not o[1].any() and not p[1].any() and not p[0, :, 3:].any()
    for i in range(4):
        e = [math.exp(float((q[0, i] * k[0, i // 2, r]).sum()) / math.sqrt(8)) for r in range(3)]
        ref = sum(e[r] * v[0, i // 2, r].double() for r in range(3)) / sum(e)
        assert (o[0, i] - ref).abs().max() < 1e-6
