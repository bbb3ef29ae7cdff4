"""Attention weights that rows of a 4-bit cache gather under large logits, against 64 bits.

A weight is 2^(logit - maximum) times the reciprocal of the sum, so rows whose logits are the same number get the same weight whatever its
size: (heads of the group) / rows, off by 2^-20 for exp2, the reciprocal and the sums (fp32, rows of one warp added 4 at a time)."""
import math

import pytest
import torch

from tests.test_gpu_qcache import _cca, _gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,dh", [(4, 2, 32), (8, 2, 64), (8, 2, 128), (4, 1, 256), (24, 2, 64), (6, 2, 64)])
@pytest.mark.parametrize("S", [3, 100, 900, 5000])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 9, 2.0 ** 15, 2.0 ** 30])
def test_weights_of_rows_with_equal_logits(hq, hk, dh, S, size):
    cca = _cca(hq, hk, dh)
    gen = _gen(dh + S)
    k = (size * torch.randn(1, 1, hk, dh, generator=gen)).bfloat16().expand(1, S, hk, dh).contiguous()
    v = torch.randn(1, S, hk, dh, generator=gen).bfloat16()
    q = (size * torch.randn(1, hq, dh, generator=gen)).bfloat16()
    cache = cca.new_qcache(1, S)
    cca.qcache_append(cache, k.cuda(), v.cuda())
    cache["len"].fill_(S)
    cca.qcache_attention(q.cuda(), cache, S, cca.alloc_qcache_workspace(1, S))
    w = cache["weight"].cpu().double()
    assert cca.last_status() == 0
    want = hq // hk / S
    assert (w - want).abs().max() <= (2.0 ** -20 + 2.0 ** -24 * (S / 4 + 16)) * want, float((w / want).max())
    cca.close()


@pytest.mark.parametrize("S", [200, 4000])
def test_weights_of_a_row_that_has_it_all(S):
    cca = _cca(8, 2, 128)
    gen = _gen(S)
    k = torch.zeros(1, S, 2, 128)
    k[:, S // 3] = 2.0 ** 30
    cache = cca.new_qcache(1, S)
    cca.qcache_append(cache, k.bfloat16().cuda(), torch.randn(1, S, 2, 128, generator=gen).bfloat16().cuda())
    cache["len"].fill_(S)
    cca.qcache_attention((2.0 ** 30 * torch.ones(1, 8, 128)).bfloat16().cuda(), cache, S, cca.alloc_qcache_workspace(1, S))
    want = torch.zeros(1, 2, S)
    want[:, :, S // 3] = 4
    assert torch.equal(cache["weight"].cpu(), want)
    cca.close()
