"""What of the 4-bit cache needs no GPU: refusals of the C ABI (argument checks happen before anything touches a device), block sizes, the
oracle's layout against itself, and tables with shared pages."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200.decoder import Decoder, PagePool

BLOCK = 16 * (128 + 16)
GOOD = dict(device=0, dtype=0, n_q_heads=8, n_kv_heads=2, head_dim=128, group=64, page_size=16, n_pages=4, d_pages=256, page_stride=2 * BLOCK, head_stride=BLOCK,
            max_seqs=2, max_q_len=1)


def desc(**kw):
    d = ls.ls_paged_kv4_desc()
    d.struct_size = C.sizeof(ls.ls_paged_kv4_desc)
    for k, v in {**GOOD, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=8), "struct_size"), (dict(dtype=2), "dtype"), (dict(n_kv_heads=3), "n_kv_heads"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(n_q_heads=0), "n_q_heads"),
    (dict(head_dim=96), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(head_dim=512), "head_dim"), (dict(group=16), "group"), (dict(group=256), "group"),
    (dict(head_dim=64, group=128), "group"), (dict(page_size=0), "page_size"), (dict(page_size=24), "page_size"), (dict(page_size=-16), "page_size"),
    (dict(n_pages=0), "n_pages"), (dict(d_pages=None), "pages"), (dict(d_pages=264), "misaligned"), (dict(page_stride=BLOCK - 16), "stride"),
    (dict(page_stride=2 * BLOCK + 8), "stride"), (dict(head_stride=BLOCK + 4), "stride"), (dict(head_stride=-BLOCK), "stride"), (dict(max_seqs=-1), "max_seqs"),
    (dict(max_q_len=0), "max_q_len"), (dict(max_seqs=1 << 20, max_q_len=1 << 20), "too large"), (dict(d_rope=256, rope_dim=3, rope_positions=4), "rope_dim"),
    (dict(d_rope=256, rope_dim=130, rope_positions=4), "rope_dim"), (dict(d_rope=256, rope_dim=64, rope_positions=0), "rope"),
    (dict(d_rope=258, rope_dim=64, rope_positions=1), "rotation"),
])
def test_create_refuses(bad, word):
    out = C.c_void_p(1)
    assert ls.lib().ls_paged_kv4_create(C.byref(desc(**bad)), C.byref(out)) == ls.LS_ERR_INVALID
    assert word in ls.last_error() and out.value is None


def test_null_handles():
    L = ls.lib()
    out = C.c_void_p()
    assert L.ls_paged_kv4_create(None, C.byref(out)) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv4_create(C.byref(desc()), None) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv4_destroy(None) == ls.LS_OK
    v = C.c_int32(0)
    assert L.ls_paged_kv4_status(None, C.byref(v)) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv4_append(None, None, 0, None, 0, 16, 256, 16, 256, 1, 16, 16, 16, 1, 1, 1, None) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv4_attend(None, 16, 1024, 16, 1024, None, 1, 1, 16, 16, 1, 1, 0, 1.0, None) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv4_read(None, 16, 256, 16, 256, 1, 16, 16, 16, 1, 1, 1, None) == ls.LS_ERR_INVALID


@pytest.mark.parametrize("page,D,group", [(16, 64, 32), (48, 128, 64), (128, 256, 128), (16, 128, 128)])
def test_block_bytes(page, D, group):
    assert ls.ls_paged_kv4_block_bytes(page, D, group) == orc.block_bytes(page, D, group) == page * (D + 8 * D // group)


@pytest.mark.parametrize("bad", [(8, 128, 64), (16, 32, 32), (16, 64, 128), (16, 128, 48)])
def test_block_bytes_refuses(bad):
    with pytest.raises(ls.LeanStreamError) as e:
        ls.ls_paged_kv4_block_bytes(*bad)
    assert e.value.code == ls.LS_ERR_INVALID


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,group", [(64, 64), (128, 32), (256, 64)])
def test_the_oracle_reads_what_it_stores(dtype, D, group):
    """Every slot of a block: no two share a byte's half, and what is held is within half a step (and the scale's rounding) of what came in."""
    rng = np.random.RandomState(D + group)
    page = 32
    block = np.zeros((1, 1, orc.block_bytes(page, D, group)), np.uint8)
    k, v = (orc.to16(rng.randn(page, D), dtype) for _ in range(2))
    for slot in rng.permutation(page):
        orc.put(block[0, 0], slot, k[slot], v[slot], group, dtype)
    for parts, x in zip(orc.held(block, page, D, group, dtype), (k, v)):
        codes, scale, zero = (a[0, :, 0] for a in parts)
        assert codes.min() == 0 and codes.max() == 15
        # a scale is off by half a step of the type, 2^-8 (bf16) at most: fifteen of them by 15 x 2^-8 of a step
        assert (np.abs(orc.values((codes, scale, zero)) - x) <= scale * (0.5 + 15 * 2.0 ** -8)).all()


def test_a_shared_prefix_stands_in_every_table():
    pool = PagePool(40, 16, 3, 128, "cpu")
    one, d = Decoder([], pool, 1), Decoder([], pool, 3)
    for _ in range(37):
        one.step(torch.zeros(1, 8))
    d.lens[0] = one.lens[0]
    d.share_prefix(0)
    assert d.prefix_len == 32 and all(pool.table[b, :2].tolist() == d.prefix_held for b in range(3))
    d.step(torch.zeros(3, 8))
    assert all(pool.table[b, :3].tolist() == d.prefix_held + pool.held[b] for b in range(3)) and d.lens == [33] * 3
