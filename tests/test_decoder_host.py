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


@pytest.mark.parametrize("seqs", [1, 3])
def test_a_prefix_can_be_extended(seqs):
    """A second share_prefix keeps the first one's pages in front; every page is in one place."""
    pool = PagePool(40, 4, seqs, 128, "cpu")
    one, d = Decoder([], pool, 1), Decoder([], pool, seqs)
    x = torch.zeros(1, 8)
    for _ in range(10):
        one.step(x)
    d.lens[0] = one.lens[0]
    first = pool.held[0][:2]
    d.share_prefix(0)
    assert d.prefix_len == 8 and d.prefix_pages.tolist() == first and d.lens == [8] * seqs and len(pool.free) == 38
    if seqs > 1:
        d.step(torch.zeros(seqs, 8))
        with pytest.raises(ls.LeanStreamError) as e:
            d.share_prefix(0)
        assert e.value.code == ls.LS_ERR_STATE
        for b in range(seqs):
            pool.release(b)
        d.lens = [8] * seqs
        d.share_prefix(1)
        assert d.prefix_len == 8 and d.prefix_pages.tolist() == first and d.lens == [8] * seqs
        return
    for _ in range(7):
        d.step(x)
    own = list(pool.held[0])
    assert d.lens == [15] and len(own) == 2 and pool.table[0, 2:4].tolist() == own
    d.share_prefix(0)
    assert d.prefix_len == 12 and d.prefix_pages.tolist() == first + own[:1] and d.lens == [12]
    assert sorted(pool.free + d.prefix_held) == list(range(40)) and pool.held == [[]]
    d.step(x)
    assert d.lens == [13] and pool.table[0, 3].item() == pool.held[0][0]
    d.share_prefix(0)  # less than a page more: the prefix stays
    assert d.prefix_len == 12 and d.prefix_pages.tolist() == first + own[:1] and d.lens == [12] and pool.held == [[]]
