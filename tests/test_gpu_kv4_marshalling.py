"""Every check that stands between Python and the pointers of ls_paged_kv4_append, _attend and _read: what is refused, that it says which
operand, and that the next call works; and pointers off their element's alignment at the C ABI."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, M, H, HK, D, PAGE, WIDTH = 3, 2, 8, 2, 64, 16, 4
V, T, L = ValueError, TypeError, ls.LeanStreamError


def z(*shape, dtype=torch.bfloat16, device=DEV):
    return torch.zeros(*shape, dtype=dtype, device=device)


def i32(*shape, device=DEV):
    return torch.zeros(*shape, dtype=torch.int32, device=device)


def pages():
    return z(5, HK, ls.ls_paged_kv4_block_bytes(PAGE, D), dtype=torch.uint8)


@pytest.fixture(scope="module")
def kv():
    handle = ls.ls_paged_kv4_create(pages(), H, D, PAGE, max_seqs=B, max_q_len=M)
    yield handle
    handle.close()


def refused(call, kv, good, bad, word, error):
    args = {**good(), **bad()}
    with pytest.raises(error) as e:
        call(kv, **args)
    assert word in str(e.value), str(e.value)
    call(kv, **good())
    torch.cuda.synchronize()


def append_good():
    return dict(q=z(B, H, D), k=z(B, HK, D), v=z(B, HK, D), q_out=z(B, H, D), seq=i32(B), pos=i32(B), table=i32(B, WIDTH))


@pytest.mark.parametrize("bad,word", [
    (lambda: dict(q=3), "q"), (lambda: dict(q=None), "together"), (lambda: dict(q_out=None), "together"), (lambda: dict(k=None), "k"), (lambda: dict(table=None), "table"),
    (lambda: dict(k=z(HK, D)), "k:"), (lambda: dict(v=z(B + 1, HK, D)), "tokens"), (lambda: dict(seq=i32(B - 1)), "tokens"), (lambda: dict(pos=i32(B + 1)), "tokens"),
    (lambda: dict(k=z(B, HK, D, dtype=torch.float16)), "k:"), (lambda: dict(v=z(B, HK, D, device="cpu")), "v:"), (lambda: dict(k=z(B, HK + 1, D)), "k:"),
    (lambda: dict(k=z(HK, B, D).transpose(0, 1)), "k:"), (lambda: dict(v=z(B, HK, 2 * D)[..., ::2]), "v:"), (lambda: dict(q=z(B, H - 1, D)), "q:"),
    (lambda: dict(q_out=z(B, H, D, dtype=torch.float16)), "q_out:"), (lambda: dict(table=i32(B, WIDTH).long()), "table:"), (lambda: dict(seq=i32(2 * B)[::2]), "seq:"),
    (lambda: dict(pos=i32(B).float()), "pos:"),
])
def test_append_refuses(kv, bad, word):
    refused(lambda kv, **a: ls.ls_paged_kv4_append(kv, **a), kv, append_good, bad, word, V)


def attend_good():
    return dict(q=z(B, M, H, D), out=z(B, M, H, D), seq_len=i32(B), table=i32(B, WIDTH), lse=z(B, M, H, dtype=torch.float32))


@pytest.mark.parametrize("bad,word,error", [
    (lambda: dict(q=None), "q", V), (lambda: dict(out=0), "out", V), (lambda: dict(seq_len=None), "seq_len", V), (lambda: dict(table=None), "table", V),
    (lambda: dict(q=z(H, D)), "q:", V), (lambda: dict(out=z(B * M, H, D)), "out:", V), (lambda: dict(q=z(B, M, H, D, dtype=torch.float16)), "q:", V),
    (lambda: dict(out=z(B, M, H, D, device="cpu")), "out:", V), (lambda: dict(q=z(M, B, H, D).transpose(0, 1)), "evenly", V), (lambda: dict(seq_len=i32(B + 1)), "one row", V),
    (lambda: dict(table=i32(B - 1, WIDTH)), "one row", V), (lambda: dict(seq_len=i32(B).long()), "seq_len:", V), (lambda: dict(table=i32(WIDTH, B).t()), "table:", V),
    (lambda: dict(lse=z(B, M, H)), "lse:", V), (lambda: dict(lse=z(B, H, dtype=torch.float32)), "lse:", V), (lambda: dict(window=2 ** 31), "32 bits", V),
    (lambda: dict(window="w"), "int", T), (lambda: dict(scale="s"), "", T), (lambda: dict(window=-1), "negative", L), (lambda: dict(scale=0.0), "scale", L),
    (lambda: dict(scale=float("nan")), "scale", L), (lambda: dict(scale=float("inf")), "scale", L), (lambda: dict(q=z(B, M + 1, H, D), out=z(B, M + 1, H, D), lse=None), "created for", L),
    (lambda: dict(q=z(B + 1, M, H, D), out=z(B + 1, M, H, D), lse=None, seq_len=i32(B + 1), table=i32(B + 1, WIDTH)), "created for", L),
])
def test_attend_refuses(kv, bad, word, error):
    refused(lambda kv, **a: ls.ls_paged_kv4_attend(kv, **a), kv, attend_good, bad, word, error)


def read_good():
    return dict(k_out=z(B, HK, D), v_out=z(B, HK, D), seq=i32(B), pos=i32(B), table=i32(B, WIDTH))


@pytest.mark.parametrize("bad,word,error", [
    (lambda: dict(k_out=1), "k_out", V), (lambda: dict(v_out=z(B, HK, D + 8)), "v_out:", V), (lambda: dict(k_out=z(B + 1, HK, D)), "k_out:", V), (lambda: dict(k_out=z(B, HK * D)), "k_out:", V),
    (lambda: dict(v_out=z(B, HK, D, dtype=torch.float16)), "v_out:", V), (lambda: dict(v_out=z(B, HK, D, device="cpu")), "v_out:", V), (lambda: dict(k_out=z(B, HK, 2 * D)[..., ::2]), "k_out:", V),
    (lambda: dict(seq=None), "seq", V), (lambda: dict(pos=i32(B + 1)), "tokens", V), (lambda: dict(seq=i32(B).long()), "seq:", V), (lambda: dict(pos=i32(B, device="cpu")), "pos:", V),
    (lambda: dict(table=i32(B * WIDTH)), "table:", V), (lambda: dict(k_out=None, v_out=None), "one of", L),
])
def test_read_refuses(kv, bad, word, error):
    refused(lambda kv, **a: ls.ls_paged_kv4_read(kv, **a), kv, read_good, bad, word, error)


def test_caches_of_the_other_kind_and_closed_ones_are_refused():
    """A 16-bit cache's handle is none of a 4-bit cache's, and the other way round."""
    k4 = ls.ls_paged_kv4_create(pages(), H, D, PAGE, max_seqs=B, max_q_len=M)
    k16 = ls.ls_paged_kv_create(z(5, PAGE, HK, D), z(5, PAGE, HK, D), H, max_seqs=B, max_q_len=M)
    for f, other, good in ((ls.ls_paged_kv4_append, k16, append_good), (ls.ls_paged_kv4_attend, k16, attend_good), (ls.ls_paged_kv4_read, k16, read_good),
                           (ls.ls_paged_kv_append, k4, append_good), (ls.ls_paged_kv_attend, k4, attend_good)):
        with pytest.raises(ValueError):
            f(other, **good())
    k4.close()
    k4.close()
    with pytest.raises(ValueError):
        ls.ls_paged_kv4_attend(k4, **attend_good())
    with pytest.raises(ls.LeanStreamError):
        ls.ls_paged_kv4_status(k4)
    k16.close()


def test_nothing_to_do():
    k = ls.ls_paged_kv4_create(pages(), H, D, PAGE)
    e = lambda n: z(0, n, D)
    ls.ls_paged_kv4_append(k, e(H), e(HK), e(HK), e(H), i32(0), i32(0), i32(B, WIDTH))
    ls.ls_paged_kv4_read(k, e(HK), e(HK), i32(0), i32(0), i32(B, WIDTH))
    with pytest.raises(ls.LeanStreamError):  # made for appends and reads only
        ls.ls_paged_kv4_attend(k, **attend_good())
    assert ls.ls_paged_kv4_status(k) == 0
    k.close()


def test_pointers_off_their_alignment(kv):
    p = z(1 << 17, dtype=torch.uint8).data_ptr()
    C = ls.lib()

    def each(call, good, *bads):
        for bad in bads:
            assert call(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID, bad
            assert "misaligned" in ls.last_error()
        assert call(kv.handle, *good.values()) == ls.LS_OK

    each(C.ls_paged_kv4_attend, dict(q=p, qs=512, o=p + 4096, os=512, lse=p + 8192, n=2, m=1, sl=p + 12288, t=p + 16384, tw=2, ts=2, w=0, sc=0.1, st=None),
         dict(q=p + 1), dict(o=p + 4097), dict(lse=p + 8194), dict(sl=p + 12289), dict(t=p + 16386))
    each(C.ls_paged_kv4_append, dict(q=p, qs=512, qo=p + 4096, qos=512, k=p + 8192, ks=128, v=p + 12288, vs=128, n=1, seq=p + 16384, pos=p + 16400, t=p + 20480, ns=2, tw=2, ts=2, st=None),
         dict(q=p + 1), dict(qo=p + 4097), dict(k=p + 8193), dict(v=p + 12289), dict(seq=p + 16385), dict(pos=p + 16402), dict(t=p + 20481))
    each(C.ls_paged_kv4_read, dict(k=p, ks=128, v=p + 4096, vs=128, n=2, seq=p + 8192, pos=p + 8256, t=p + 12288, ns=2, tw=2, ts=2, st=None),
         dict(k=p + 1), dict(v=p + 4097), dict(seq=p + 8193), dict(pos=p + 8258), dict(t=p + 12290))
    good = dict(q=p, qs=512, o=p + 4096, os=512, lse=None, n=2, m=1, sl=p + 12288, t=p + 16384, tw=2, ts=2, w=0, sc=0.1, st=None)
    for bad, word in ((dict(qs=511), "stride"), (dict(os=0), "stride"), (dict(ts=1), "table_stride"), (dict(n=-1), "negative"), (dict(tw=-1), "negative"), (dict(q=None), "required"),
                      (dict(t=None), "table")):
        assert C.ls_paged_kv4_attend(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID and word in ls.last_error(), bad
    assert ls.ls_paged_kv4_status(kv) == 0
