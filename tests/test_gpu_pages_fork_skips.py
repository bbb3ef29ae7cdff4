"""Forks of pairs that are skipped: they count as if they were not there, whatever they are skipped for."""
import pytest

from oracle import pages_oracle as P
from tests.test_gpu_pages import filled, ints, make, same

pytestmark = pytest.mark.gpu

# (parent, child): the last pair of child 0 that is not skipped counts, be it its own parent; 3 is not in use, 4's rows have no room
PAIRS = [((1, 3), (0, 0)), ((1, 4), (0, 0)), ((1, -7), (0, 0)), ((1, 2, 3, 4), (0, 0, 0, 0)), ((3, 1), (0, 0)), ((1, 0, 3), (0, 0, 0)),
         ((2, 3), (3, 3)), ((3, 4), (0, 1)), ((2, 4, 1, 3), (0, 0, 2, 2))]


def state(cca, B, wide):
    """0 to 2 hold rows; 3 is not in use and holds pages, 4 says that it has more rows than its table has room for; the others are empty."""
    pages = filled(cca, 40, 4, B, wide)
    ws = cca.alloc_pages_workspace(40, B, wide)
    cca.pages_reserve(pages, 10, ws, ints([10, 7, 3, 2, 9] + [0] * (B - 5)))
    pages["len"].copy_(ints([10, 7, 3, -1, 4 * wide + 1] + [0] * (B - 5)))
    return pages, ws


@pytest.mark.parametrize("B,wide", [(6, 6), (70, 300)])
@pytest.mark.parametrize("parent,child", PAIRS)
def test_skipped_pairs_do_not_count(B, wide, parent, child):
    cca = make(1, 32)
    pages, ws = state(cca, B, wide)
    pool = P.Pool.of(pages)
    fill = B - len(parent) if B > 64 else 0                    # many pairs: two launches instead of one
    more = list(range(5, 5 + min(fill, B - 5)))
    parent, child = [*parent, *more], [*child, *more]
    cca.pages_fork(pages, ints(parent), ints(child), ws)
    assert pool.fork(parent, child) == 122
    same(pages, pool)
    assert cca.last_status() == 122
    cca.close()
