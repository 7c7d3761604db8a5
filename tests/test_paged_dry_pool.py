"""The oracle of the cache in pages where the pool runs dry: a slot's length is the number of
its tokens that were appended and kept, counted one by one."""
import pytest

from oracle import paged as O
from tests.paged_schedule import Held, schedule


@pytest.mark.parametrize("seed", range(6))
def test_lengths_are_of_tokens_that_were_appended(seed):
    batch, width, page = 5, 5, 32
    t, held, keep = O.Tables(batch, 9, 4, page), Held(batch), None
    lacked = 0
    for n_new, next_keep in schedule(seed, batch, 60, width, 3 * page):
        _, missing = t.step(n_new, keep, width)
        held.end([0] * batch if keep is None else keep)
        assert t.lens == [len(x) for x in held.tokens]
        held.begin(n_new, missing)
        keep, lacked = next_keep, lacked + sum(m > 0 for m in missing)
    assert lacked > 10


def test_a_slot_without_pages_keeps_nothing_new():
    t = O.Tables(1, 2, 4, 32)
    t.step([62])
    assert t.step([5], keep=[62], width=5) == ([[-1] * 5], [1])
    t.step([1], keep=[2])                                    # two of none
    assert t.lens == [62]


def test_keep_more_than_there_is():
    t = O.Tables(2, 8, 4, 32)
    assert t.step([40, 129])[1] == [0, 5]
    t.step([0, 0], keep=[2 ** 31 - 1, 2 ** 31 - 1])
    assert t.lens == [40, 0]
