"""Attention over pages of values that are infinite: a channel is what 64 bits give, infinite, or no number where both infinities meet.  Weights here
are far above the smallest fp32 number."""
import math

import pytest
import torch

from oracle import pages_oracle as P
from tests.test_gpu_paged_attention import U, cached
from tests.test_gpu_pages import make

pytestmark = pytest.mark.gpu
INF = float("inf")


def put(pages, size, b, row, j, channel, value):
    pages["v"][int(pages["table"][b, row // size]), j, row % size, channel] = value


def check_infinite(cca, pages, q, lens, o):
    """Infinite and NaN channels as in 64 bits; the others within the tolerances of the finite tests."""
    pool, g, dh = P.Pool.of(pages), cca.cfg.n_q_heads // cca.cfg.n_kv_heads, cca.cfg.head_dim
    o = o.cpu().double()
    for b, n in enumerate(lens):
        k, v = pool.rows(b, n)
        want, _, p = P.attention(q[b], k, v, g)
        fine = torch.isfinite(want)
        assert torch.equal(torch.isnan(o[b]), torch.isnan(want)), b
        assert torch.equal(o[b][torch.isinf(want)], want[torch.isinf(want)]), b
        assert bool(torch.isfinite(o[b][fine]).all()), b
        for i in range(q.shape[1]):
            A = float((k[i // g].abs() @ q[b, i].double().abs()).max()) * math.log2(math.e) / math.sqrt(dh)
            rel = math.log(2) * (2 * U * (dh + 16) * A + 4 * U * (A + 64)) + 2.0 ** -20 + 2.0 ** -16 + n * U
            tol = 2 * rel * (p[i] @ v[i // g].abs()) + 2.0 ** -8 * want[i].abs() + 1e-30
            assert bool(((o[b, i] - want[i]).abs()[fine[i]] <= tol[fine[i]]).all()), (b, i)


@pytest.mark.parametrize("hq,hk,dh", [(4, 4, 32), (8, 2, 64), (8, 1, 64), (6, 1, 128), (4, 1, 256), (9, 1, 256)])
@pytest.mark.parametrize("lens,max_len,launches", [([1, 2, 40], 40, 1), ([1000, 33, 300], 1024, 1), ([5000, 1, 70], 40000, 2)])
def test_infinite_values(hq, hk, dh, lens, max_len, launches):
    cca = make(hk, dh, hq)
    size = 16
    pages = cached(cca, size, lens, dh + hq, wide=-(-max_len // size))
    for b, n in enumerate(lens):
        for j in range(hk):
            for x in range(6):                                 # six channels of a head hold one infinity, or several, anywhere
                row = (x * 7919 + 31 * j) % n
                put(pages, size, b, row, j, 3 + 4 * x, INF if x % 2 else -INF)
            put(pages, size, b, n - 1, j, 3, -INF)
            put(pages, size, b, 0, j, 3, -INF)
            put(pages, size, b, n - 1, j, 7, -INF)             # against +inf elsewhere, unless the row is the same
            put(pages, size, b, n // 2, j, 30, float("nan"))
    q = torch.randn(len(lens), hq, dh, generator=torch.Generator().manual_seed(3)).bfloat16()
    ws = cca.alloc_paged_workspace(len(lens), max_len)
    ws.fill_(255)
    before = cca.launch_count()
    o = cca.paged_attention(q.cuda(), pages, max_len, ws)
    torch.cuda.synchronize()
    assert cca.launch_count() - before == launches and cca.last_status() == 0
    check_infinite(cca, pages, q, lens, o)
    cca.close()


@pytest.mark.parametrize("hq", [4, 8])
@pytest.mark.parametrize("turn", [1, -1])
def test_infinite_values_under_a_moving_maximum(hq, turn):
    """Logits that rise, or fall, by 40 from end to end: an infinity in the first, the last and a middle row outlives every change of the maximum."""
    cca = make(1, 128, hq)
    n = 900
    pages = cached(cca, 16, [n], 1)
    pool = pages["table"][0, :-(-n // 16)].long()
    ramp = turn * torch.arange(57 * 16, device="cuda").view(57, 16).float() / 2
    pages["k"][pool, 0, :, 0] = ramp.bfloat16()
    q = torch.zeros(1, hq, 128)
    q[..., 0] = 1.0
    for x, row in enumerate((0, n - 1, n // 2)):
        put(pages, 16, 0, row, 0, 5 + x, INF if x != 1 else -INF)
    o = cca.paged_attention(q.bfloat16().cuda(), pages, n, cca.alloc_paged_workspace(1, n))
    torch.cuda.synchronize()
    check_infinite(cca, pages, q.bfloat16(), [n], o)
    assert bool((o[0, :, 5] == INF).all()) and bool((o[0, :, 6] == -INF).all()) and bool((o[0, :, 7] == INF).all())
    cca.close()
