"""Attention over pages where the units of rows are shared out over all CTAs and joined in a second launch, at every head size and number of heads a pass:
that this form runs is read off the launches of the call (two; the clusters' form has one).  Tolerances are those of the cluster form's tests."""
import pytest
import torch

from tests.test_gpu_paged_attention import cached, check
from tests.test_gpu_pages import ints, make

pytestmark = pytest.mark.gpu


def shared_out(cca, size, lens, seed, max_len, status=0, pages=None, out=None, lse=None):
    """(pages, q, o, lse) of a call that is known to take the second launch."""
    pages = pages or cached(cca, size, lens, seed, wide=-(-max_len // size))
    B, hq, dh = len(lens), cca.cfg.n_q_heads, cca.cfg.head_dim
    q = torch.randn(B, hq, dh, generator=torch.Generator().manual_seed(seed + 1)).bfloat16()
    ws = cca.alloc_paged_workspace(B, max_len)
    ws.fill_(255)                                              # NaN wherever a kernel reads what nobody wrote
    lse = torch.full((B, hq), 7.0, device="cuda") if lse is None else lse
    before = cca.launch_count()
    o = cca.paged_attention(q.cuda(), pages, max_len, ws, out=out, lse=lse)
    torch.cuda.synchronize()
    assert cca.launch_count() - before == 2
    assert cca.last_status() == status
    return pages, q, o, lse


@pytest.mark.parametrize("dh", [32, 64, 128, 256])
@pytest.mark.parametrize("g", [1, 4, 6, 8, 11])
def test_one_long_sequence(dh, g):
    cca = make(1, dh, g)
    n = 16384 if dh < 256 or g < 8 else 7001
    pages, q, o, lse = shared_out(cca, 16, [n], dh + g, 16384)
    check(cca, pages, q, [n], o, lse)
    cca.close()


@pytest.mark.parametrize("dh", [32, 64, 128, 256])
@pytest.mark.parametrize("g", [3, 7])
def test_few_ragged_sequences(dh, g):
    """Runs that begin and end inside a CTA's part, in pages that end inside a unit; one sequence is empty, one a single row."""
    cca = make(2, dh, 2 * g)
    lens = [4099, 0, 1, 2500]
    pages, q, o, lse = shared_out(cca, 40, lens, dh + g, 40000)
    check(cca, pages, q, lens, o, lse)
    cca.close()


@pytest.mark.parametrize("dh,B,hk,max_len", [(32, 35, 1, 102400), (64, 35, 1, 51200), (128, 35, 1, 25600), (256, 18, 1, 25600), (64, 7, 5, 51200),
                                             (256, 9, 2, 25600)])
@pytest.mark.parametrize("g", [2, 4, 5, 8])
def test_a_warp_joins_a_head(dh, B, hk, max_len, g):
    """As many runs as leave each a few CTAs: a warp joins a head's parts.  All of one length under the bound, and one of many CTAs among short ones."""
    cca = make(hk, dh, hk * g)
    for lens in ([701 + 13 * b for b in range(B)], [5000 if b == B // 2 else 90 * (b % 3) for b in range(B)]):
        pages, q, o, lse = shared_out(cca, 64, lens, B + g, max_len)
        check(cca, pages, q, lens, o, lse)
    cca.close()


def test_sequences_outside_the_bound_and_not_in_use():
    """One too long is left as it is and told of; one that is not in use is left as it is without a word."""
    cca = make(1, 64, 4)
    lens = [9000, 60, 50, 20, 0]
    pages = cached(cca, 16, lens, 2, wide=1200)
    pages["len"].copy_(ints(9000, 16385, -1, 20, 0))
    out, lse = torch.full((5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 4), 7.0, device="cuda")
    _, q, _, _ = shared_out(cca, 16, lens, 2, 16384, status=122, pages=pages, out=out, lse=lse)
    assert bool((out[1:3] == 7).all()) and bool((lse[1:3] == 7).all())
    check(cca, pages, q, [9000, 0, 0, 20, 0], out, lse, only=(0, 3, 4))
    pages["len"].copy_(ints(9000, 60, -7, 20, 0))
    out.fill_(7)
    lse.fill_(7)
    _, q, _, _ = shared_out(cca, 16, lens, 2, 16384, pages=pages, out=out, lse=lse)
    assert bool((out[2] == 7).all()) and bool((lse[2] == 7).all())
    check(cca, pages, q, [9000, 60, 0, 20, 0], out, lse, only=(0, 1, 3, 4))
    cca.close()


@pytest.mark.parametrize("dh,g", [(64, 4), (256, 6)])
def test_rows_without_a_page_are_left_out(dh, g):
    """Entries outside the pool: single ones, all of a CTA's part of a run, and all of a sequence."""
    cca = make(1, dh, g)
    lens = [9000, 90, 6400, 33]
    pages = cached(cca, 16, lens, 6, wide=1024)
    n = pages["refs"].numel()
    pages["table"][0, 2], pages["table"][0, 24], pages["table"][1, 0] = -1, n, -2147483648
    pages["table"][0, 100:300] = -1                            # 3200 rows: more than a CTA's part
    pages["table"][2, :400] = n + 5
    pages, q, o, lse = shared_out(cca, 16, lens, 6, 16384, status=122, pages=pages)
    check(cca, pages, q, lens, o, lse)
    assert not o[2].any() and bool((lse[2] == -float("inf")).all())
    cca.close()


def test_the_same_every_time():
    cca = make(1, 256, 6)
    lens = [5000, 77, 0, 2300]
    pages, q, o, lse = shared_out(cca, 64, lens, 11, 16384)
    for _ in range(20):
        _, _, again, l2 = shared_out(cca, 64, lens, 11, 16384, pages=pages)
        assert torch.equal(again, o) and torch.equal(l2, lse)
    cca.close()
