"""Entries of a batch that name one row of a paged cache, some of which take no part."""
import pytest

from oracle import paged as orc
from tests.paged_common import GpuCache

# rows, offsets, starts, numbers of accepted tokens: row 1 is named by an entry that takes no part, and then by one that does
CASES = [([1, 1, 0], [-1, 4, 8, 12], [40, 40, 20]),         # offsets that begin below zero
         ([1, 1, 0], [9, 4, 8, 12], [40, 40, 20]),          # offsets that run backwards
         ([1, 1, 0], [0, 4, 8, 12], [-1, 40, 20]),          # no start
         ([1, 1, 1], [-1, 4, 8, 12], [40, 40, 40])]         # and a third, behind the one that takes part
LENGTHS = [[24, 42, 0], [24, 42, 0], [24, 42, 0], [24, 42, 0]]


def prepared(c):
    c.extend(c.batch([0, 1], [20, 40]))
    c.extend(c.batch([1, 0], [4, 4]))


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
def test_the_first_that_takes_part(case):
    rows, cu, start = CASES[case]
    c = GpuCache(60, 16, 3, 12)
    prepared(c)
    x = c.batch(rows, cu=cu, total=12, max_n=4, start=start)
    path = [0, 0, 0, 0, 1, 3, 0, 0, 0, 1, 2, 3]
    c.accept(x, path, [2, 2, -1])
    assert c.lens.tolist() == LENGTHS[case]


def test_the_rule_by_hand():
    """The oracle's: row 1 keeps tokens 1 and 3 of its four, whatever a void entry ahead says of it; a second one that could be is left out."""
    for rows, cu, start in CASES:
        c = orc.Cache(60, 16, 3, 12)
        c.extend([0, 20, 60], [0, 1], 60)
        c.extend([0, 4, 8], [1, 0], 8)
        c.accept(cu, rows, 12, start, [0, 0, 0, 0, 1, 3, 0, 0, 0, 1, 2, 3], [2, 2, -1])
        assert c.lens.tolist() == [24, 42, 0]
    c = orc.Cache(60, 16, 3, 12)
    c.extend([0, 20, 60], [0, 1], 60)
    c.extend([0, 4, 8], [1, 0], 8)
    c.accept([0, 4, 8], [1, 1], 8, [40, 40], [0, 1, 2, 3, 0, 1, 2, 3], [1, 2])
    assert c.lens.tolist() == [24, 41, 0] and c.status == orc.ENTRY
