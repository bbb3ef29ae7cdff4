"""Pins of the pages oracle where something is skipped: worked out by hand."""
from oracle import pages_oracle as P
from tests.test_pages_oracle import pool


def test_read_of_sequences_not_in_use():
    s = pool(4, 4, [[0, 1], [2, 3], [1, -1]], [6, -1, 2])
    k, v = s.read(3)                                           # by the length: nothing of the second
    assert not k[1].any() and not v[1].any()
    assert (k[0, :2] == s.k[1, :, 2:].transpose(0, 1)).all() and not k[0, 2].any() and (k[2, 0] == s.k[1, :, 2]).all()
    k, v = s.read(3, [-1, -1, -1])                             # by a start of its own: row -1 is none, the others are
    assert not k[:, 0].any() and (k[1, 1:] == s.k[2, :, :2].transpose(0, 1)).all() and (v[1, 1:] == s.v[2, :, :2].transpose(0, 1)).all()


def test_fork_counts_the_last_pair_that_is_not_skipped():
    def state():                                               # 2 is not in use, 3 says 9 rows of a table of 8
        return pool(9, 4, [[0, 1], [2, -1], [3, -1], [4, 5]], [8, 3, -1, 9])
    for later in (2, 3, 4, -1):                                # 1 -> 0, then a pair that is skipped
        s = state()
        assert s.fork([1, later], [0, 0]) == P.MISSING
        assert s.table == [[2, -1], [2, -1], [3, -1], [4, 5]] and s.len == [3, 3, -1, 9]
        assert s.refs == [0, 0, 2, 1, 1, 1, 0, 0, 0]
    s = state()
    assert s.fork([2, 1, 3, 0], [0, 0, 0, 0]) == P.MISSING     # the last that counts: its own parent
    assert s.table == [[0, 1], [2, -1], [3, -1], [4, 5]] and s.refs == [1, 1, 1, 1, 1, 1, 0, 0, 0]
