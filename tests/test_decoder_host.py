"""What decoder.py keeps on the host: pages, tables, lengths.  (No layers, no GPU.)"""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200.decoder import Decoder, PagePool


def pool_state(pool):
    return list(pool.free), [list(h) for h in pool.held], pool.table.clone()


def same(a, b):
    return a[0] == b[0] and a[1] == b[1] and torch.equal(a[2], b[2])


def test_reserve_gives_all_or_nothing():
    pool = PagePool(5, 4, 2, 64, "cpu")
    pool.reserve(0, 9)
    assert len(pool.held[0]) == 3 and pool.table[0, :3].tolist() == pool.held[0]
    before = pool_state(pool)
    with pytest.raises(ls.LeanStreamError) as e:
        pool.reserve(1, 12)
    assert e.value.code == ls.LS_ERR_CAPACITY and same(before, pool_state(pool))
    pool.reserve(1, 8)
    assert not pool.free and sorted(pool.held[0] + pool.held[1]) == list(range(5))


def test_a_sequence_beyond_its_table_is_refused():
    pool = PagePool(50, 4, 2, 16, "cpu")
    pool.reserve(0, 16)
    before = pool_state(pool)
    with pytest.raises(ls.LeanStreamError) as e:
        pool.reserve(0, 17)
    assert e.value.code == ls.LS_ERR_CAPACITY and same(before, pool_state(pool))


@pytest.mark.parametrize("pages", [3, 4, 5])
def test_a_step_without_room_changes_nothing(pages):
    """Three sequences, a page for each, then no page for all of them: lengths and pages stay; with a page given back it goes on."""
    pool = PagePool(pages, 2, 3, 64, "cpu")
    d, x = Decoder([], pool, 3), torch.zeros(3, 8)
    d.step(x), d.step(x)
    before = pool_state(pool)
    for _ in range(2):
        with pytest.raises(ls.LeanStreamError) as e:
            d.step(x)
        assert e.value.code == ls.LS_ERR_CAPACITY and d.lens == [2, 2, 2] and same(before, pool_state(pool))
    pool.free += [100, 101, 102][: 6 - pages]
    d.step(x)
    assert d.lens == [3, 3, 3] and all(len(h) == 2 for h in pool.held) and not pool.free
