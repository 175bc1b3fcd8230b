"""ls_paged_kv_attend where order and ranges are at stake: what warps hand to each other at the ends of pieces, windows and
lengths near the end of 32 bits, weights far below the largest."""
import numpy as np
import pytest
import torch

from test_gpu_paged_kv import DEV, Batch, f64

from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,hk", [(8, 8), (16, 1)])
@pytest.mark.parametrize("keys", [60, 128, 300])
def test_maxima_that_rise_in_the_last_tile_of_a_piece(dtype, heads, hk, keys):
    """Narrow pieces whose last tile raises the reference of every row (a piece of one tile always does; longer ones by keys in rising
    order): the maxima that the four warps exchange there are not the sums that they exchange right behind, call after call."""
    b = Batch(dtype=dtype, heads=heads, hk=hk, D=64, lens=[keys - (i * 7) % 50 for i in range(96)], std=8.0, seed=keys)
    for s, n in enumerate(b.lens):
        at = torch.arange(n, device=DEV)
        pg, sl = b.table[s, at // b.page].long(), at % b.page
        k = b.kp[pg, sl]
        b.kp[pg, sl] = k[(k[:, 0].float() @ b.q[s, 0].float().mean(0)).argsort()]
    kv = b.handle()
    b.attend(kv)
    b.check()
    out, lse = b.out.clone(), b.lse.clone()
    for _ in range(200):
        b.out.fill_(float("nan"))
        b.attend(kv)
        assert torch.equal(out, b.out) and torch.equal(lse, b.lse)
    assert ls.ls_paged_kv_status(kv) == 0
    kv.close()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30])
@pytest.mark.parametrize("prefix,q_len", [(0, 4), (0, 9), (150, 4), (150, 9)])
@pytest.mark.parametrize("D", [128, 96])
def test_a_window_beyond_every_length_is_none(window, prefix, q_len, D):
    """Such a window is a way to say 'no window', also for sequences shorter than q_len (whose first tokens see nothing)."""
    kw = dict(D=D, prefix=prefix, q_len=q_len, lens=[1, 2, 3, 0, prefix + 40, prefix + 1, 300 + prefix], seed=q_len)
    b = Batch(window=window, **kw)
    kv = b.handle()
    b.attend(kv)
    b.check()
    plain = Batch(window=0, **kw)
    kv0 = plain.handle()
    plain.attend(kv0)
    plain.check()
    assert ls.ls_paged_kv_status(kv) == 0 and ls.ls_paged_kv_status(kv0) == 0
    kv.close(), kv0.close()
    # only short sequences: nobody pulls the first key that is seen down
    b = Batch(window=window, D=D, prefix=prefix, q_len=q_len, lens=[1, 2], seed=q_len)
    kv = b.handle()
    b.attend(kv)
    b.check()
    kv.close()
