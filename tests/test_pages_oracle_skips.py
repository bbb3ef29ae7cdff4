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
