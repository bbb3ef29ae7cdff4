"""Reads of more rows than the library covers are refused by name, before memory for them is asked for."""
import pytest
import torch

from tests.test_gpu_pages import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,n", [(1, (1 << 24) + 1), (3, 1 << 40), (2, 1 << 62), (65, 1 << 24), (1025, 1 << 20)])
def test_too_many_rows(B, n):
    from paper_2510_04476_b200.binding import CcaError
    cca = make(2, 32)
    pages = cca.new_pages(4, 4, B, 3)
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    with pytest.raises(CcaError, match="unsupported"):
        cca.paged_read(pages, n)
    assert torch.cuda.max_memory_allocated() == held and cca.last_status() == 0
    cca.close()
