"""A workspace made for the longest caches, used for shorter ones too."""
import pytest
import torch

from tests.test_gpu_qcache import _cca

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,dh,B,made,calls", [(8, 2, 128, 1, 16500, (13697, 15000, 16384)), (8, 2, 128, 1, 8448, (5593, 8192)),
                                                   (8, 2, 128, 4, 5001, (3329, 4736))])
def test_a_workspace_for_long_caches_serves_shorter_ones(hq, hk, dh, B, made, calls):
    """Attention and eviction of a cache that grows, in one workspace: the same as in one of its own length."""
    cca = _cca(hq, hk, dh)
    gen = torch.Generator(device="cuda").manual_seed(made)
    k, v = (torch.randn(B, made, hk, dh, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(B, hq, dh, generator=gen, device="cuda").bfloat16()
    nxt = torch.full((B,), made, dtype=torch.int32, device="cuda")
    one = cca.alloc_qcache_workspace(B, made)
    for n in calls:
        seen = []
        for ws in (one, cca.alloc_qcache_workspace(B, n)):
            ws.fill_(255)
            cache = cca.new_qcache(B, made)
            cca.qcache_append(cache, k[:, :n].contiguous(), v[:, :n].contiguous())
            cache["len"].fill_(n)
            o = cca.qcache_attention(q, cache, n, ws)
            cca.qcache_evict(cache, n // 2, 10, nxt, n, ws)
            seen.append((o, cache))
        assert torch.equal(seen[0][0], seen[1][0])
        for name in seen[0][1]:
            assert torch.equal(seen[0][1][name], seen[1][1][name]), name
    assert cca.last_status() == 0
    cca.close()
