"""Pointers that do not lie at a multiple of their element's size are refused (a kernel's access through them would fault)."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls
from test_decoder_ops_host import NORM


@pytest.mark.parametrize("bad", [
    dict(x=258), dict(xo=770), dict(y=513), dict(h=1025), dict(g=2049), dict(wp=2050), dict(wn=2049), dict(x=257, xt=0, t=0), dict(xo=769, xt=1, t=1),
    dict(y=514, t=2), dict(h=1026, t=2), dict(g=2050, t=2, gs=64),
])
def test_norm(bad):
    assert ls.lib().ls_block_norm(*{**NORM, **bad}.values()) == ls.LS_ERR_INVALID
    assert "misaligned" in ls.last_error()


@pytest.mark.gpu
def test_append_and_attend():
    dev = "cuda:0"
    kp, vp = (torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device=dev) for _ in range(2))
    kv = ls.ls_paged_kv_create(kp, vp, 4, max_seqs=2, max_q_len=1)
    p = torch.zeros(1 << 16, dtype=torch.uint8, device=dev).data_ptr()
    L = ls.lib()
    good = dict(q=p, qs=256, o=p + 4096, os=256, lse=p + 8192, n=2, m=1, sl=p + 12288, t=p + 16384, tw=2, ts=2, pp=p + 20480, pl=8, w=0, sc=0.1, st=None)
    for bad in (dict(q=p + 1), dict(o=p + 4097), dict(lse=p + 8194), dict(sl=p + 12289), dict(t=p + 16386), dict(pp=p + 20482)):
        assert L.ls_paged_kv_attend(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID, bad
        assert "misaligned" in ls.last_error()
    assert L.ls_paged_kv_attend(kv.handle, *good.values()) == ls.LS_OK
    good = dict(q=p, qs=256, qo=p + 4096, qos=256, k=p + 8192, ks=128, v=p + 12288, vs=128, n=1, seq=p + 16384, pos=p + 16400, t=p + 20480, ns=2, tw=2, ts=2, st=None)
    for bad in (dict(q=p + 1), dict(qo=p + 4097), dict(k=p + 8193), dict(v=p + 12289), dict(seq=p + 16385), dict(pos=p + 16402), dict(t=p + 20481)):
        assert L.ls_paged_kv_append(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID, bad
        assert "misaligned" in ls.last_error()
    assert L.ls_paged_kv_append(kv.handle, *good.values()) == ls.LS_OK
    assert ls.ls_paged_kv_status(kv) == 0
    kv.close()
