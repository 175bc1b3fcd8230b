"""Refusals of ls_paged_kv_* and ls_block_norm (argument checks happen before anything touches a device)."""
import ctypes as C

import pytest

from paper_2609_03079_b200 import binding as ls

GOOD = dict(device=0, dtype=0, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=4, d_k=256, d_v=4096, page_stride=16 * 256,
            token_stride=256, head_stride=128, max_seqs=2, max_q_len=1)


def desc(**kw):
    d = ls.ls_paged_kv_desc()
    d.struct_size = C.sizeof(ls.ls_paged_kv_desc)
    for k, v in {**GOOD, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=8), "struct_size"), (dict(dtype=2), "dtype"), (dict(n_kv_heads=3), "n_kv_heads"), (dict(n_kv_heads=0), "n_kv_heads"),
    (dict(n_q_heads=0), "n_q_heads"), (dict(head_dim=100), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(head_dim=264), "head_dim"),
    (dict(page_size=0), "page_size"), (dict(n_pages=0), "n_pages"), (dict(d_k=None), "pages"), (dict(d_v=None), "pages"), (dict(d_k=257), "misaligned"),
    (dict(head_stride=-1), "stride"), (dict(max_seqs=-1), "max_seqs"), (dict(max_q_len=0), "max_q_len"),
    (dict(d_rope=256, rope_dim=3, rope_positions=4), "rope_dim"), (dict(d_rope=256, rope_dim=130, rope_positions=4), "rope_dim"),
    (dict(d_rope=256, rope_dim=64, rope_positions=0), "rope"), (dict(d_rope=258, rope_dim=64, rope_positions=1), "rotation"),
])
def test_create_refuses(bad, word):
    out = C.c_void_p(1)
    assert ls.lib().ls_paged_kv_create(C.byref(desc(**bad)), C.byref(out)) == ls.LS_ERR_INVALID
    assert word in ls.last_error() and out.value is None


def test_null_handles():
    L = ls.lib()
    out = C.c_void_p()
    assert L.ls_paged_kv_create(None, C.byref(out)) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv_create(C.byref(desc()), None) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv_destroy(None) == ls.LS_OK
    v = C.c_int32(0)
    assert L.ls_paged_kv_status(None, C.byref(v)) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv_append(None, None, 0, None, 0, 16, 256, 16, 256, 1, 16, 16, 16, 1, 1, 1, None) == ls.LS_ERR_INVALID
    assert L.ls_paged_kv_attend(None, 16, 1024, 16, 1024, None, 1, 1, 16, 16, 1, 1, None, 0, 0, 1.0, None) == ls.LS_ERR_INVALID


NORM = dict(x=256, xs=64, xt=2, y=512, ys=64, t=0, xo=768, xos=64, h=1024, hs=64, n=2, d=64, post=0, wp=None, g=None, gs=0, scale=1.0, pre=0, wn=None,
            eps=1e-5, st=None)


@pytest.mark.parametrize("bad,word", [
    (dict(n=-1), "n must"), (dict(d=0), "d must"), (dict(d=16385), "d must"), (dict(t=3), "dtype"), (dict(xt=1), "residual"), (dict(xt=7), "residual"),
    (dict(post=2), "norm"), (dict(pre=-1), "norm"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(x=None), "required"),
    (dict(xo=None, h=None), "required"), (dict(y=None, g=2048), "needs"), (dict(y=None, wp=2048), "needs"), (dict(xs=63), "stride"), (dict(ys=63), "stride"),
    (dict(xos=63), "stride"), (dict(hs=0), "stride"), (dict(g=2048, gs=63), "stride"),
])
def test_norm_refuses(bad, word):
    a = {**NORM, **bad}
    assert ls.lib().ls_block_norm(*a.values()) == ls.LS_ERR_INVALID
    assert word in ls.last_error()


def test_an_empty_norm_is_nothing_to_do():
    assert ls.lib().ls_block_norm(*{**NORM, "n": 0}.values()) == ls.LS_OK
