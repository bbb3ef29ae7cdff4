"""Sequences that are not in use (a negative length) in the calls that go by the length."""
import pytest
import torch

from oracle import pages_oracle as P
from tests.test_gpu_pages import bits, filled, ints, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 40])
def test_read_by_length_gives_zeros(n):
    cca = make(2, 64)
    pages = filled(cca, 30, 8, 5, 6)
    ws = cca.alloc_pages_workspace(30, 5, 6)
    cca.pages_reserve(pages, 48, ws)
    pages["len"].copy_(ints(0, -1, 5, -30, 47))
    pool = P.Pool.of(pages)
    for _ in range(3):                                         # whatever the new tensors held
        torch.full((1 << 22,), 7.0, device="cuda")
        got = cca.paged_read(pages, n)
        for g, w in zip(got, pool.read(n)):
            assert torch.equal(bits(g), bits(w))
        assert not got[0][1].any() and not got[1][1].any() and not got[0][3].any() and not got[1][3].any()
    first = [0, -1, 5, -30, 47]                                # by a start of its own the same sequences are read as they are
    for g, w in zip(cca.paged_read(pages, n, ints(first)), pool.read(n, first)):
        assert torch.equal(bits(g), bits(w))
    assert cca.last_status() == 0
    cca.close()
