"""What a 4-bit cache's handle allocates: the workspace of the rows that it can be called with, and no more."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls
from test_gpu_kv4_attend import Batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_few_rows_need_little_workspace():
    """Sixteen handles for one query head to a key head, two groups: pieces of four rows, two for each of 12 warps and every processor (7.5 MB), where sixteen
    rows of eight warps would be 20 MB."""
    pages = torch.zeros(4, 8, ls.ls_paged_kv4_block_bytes(16, 128, 64), dtype=torch.uint8, device=DEV)
    make = lambda: ls.ls_paged_kv4_create(pages, 8, 128, 16, max_seqs=4, max_q_len=1)
    make().close()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    handles = [make() for _ in range(16)]
    used = before - torch.cuda.mem_get_info()[0]
    for h in handles:
        h.close()
    assert used < 16 * 12 * 2 ** 20, used


@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (128, 128), (256, 64)])
@pytest.mark.parametrize("per,q_len", [(1, 1), (2, 1), (3, 2), (5, 1), (3, 3), (4, 4), (17, 1)])
def test_handles_made_for_just_so_many_rows(D, group, per, q_len):
    """Every shape that the rows of a handle's calls can have, fewer tokens than it was made for among them."""
    b = Batch(D=D, group=group, heads=2 * per, hk=2, q_len=q_len, lens=[70, 0, 300])
    kv = b.handle()
    b.attend(kv)
    b.check()
    for m in range(1, q_len):  # the last tokens alone
        part = Batch(D=D, group=group, heads=2 * per, hk=2, q_len=m, lens=[70, 0, 300])
        part.pages, part.table, part.table_np = b.pages, b.table, b.table_np
        part.attend(kv)
        part.check()
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()
