"""Every check that stands between Python and the pointers of ls_paged_kv_append, ls_paged_kv_attend and ls_block_norm: what is refused,
that it says which operand, and that the next call works."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, M, H, HK, D, PAGE, WIDTH = 3, 2, 8, 2, 64, 16, 4


def z(*shape, dtype=torch.bfloat16, device=DEV):
    return torch.zeros(*shape, dtype=dtype, device=device)


def i32(*shape, device=DEV):
    return torch.zeros(*shape, dtype=torch.int32, device=device)


@pytest.fixture(scope="module")
def kv():
    handle = ls.ls_paged_kv_create(z(5, PAGE, HK, D), z(5, PAGE, HK, D), H, max_seqs=B, max_q_len=M)
    yield handle
    handle.close()


def refused(call, kv, good, bad, word, error):
    args = {**good(), **bad()}
    with pytest.raises(error) as e:
        call(kv, **args)
    assert word in str(e.value), str(e.value)
    call(kv, **good())
    torch.cuda.synchronize()


V, T, L = ValueError, TypeError, ls.LeanStreamError


def append(kv, q, k, v, q_out, seq, pos, table, **kw):
    ls.ls_paged_kv_append(kv, q, k, v, q_out, seq, pos, table, **kw)


def append_good():
    return dict(q=z(B, H, D), k=z(B, HK, D), v=z(B, HK, D), q_out=z(B, H, D), seq=i32(B), pos=i32(B), table=i32(B, WIDTH))


@pytest.mark.parametrize("bad,word", [
    (lambda: dict(q=3), "q"), (lambda: dict(q=None), "together"), (lambda: dict(q_out=None), "together"), (lambda: dict(q_out=[1]), "q_out"),
    (lambda: dict(k=None), "k"), (lambda: dict(v="v"), "v"), (lambda: dict(seq=None), "seq"), (lambda: dict(pos=0), "pos"), (lambda: dict(table=None), "table"),
    (lambda: dict(k=z(HK, D)), "k:"), (lambda: dict(k=z(1, B, HK, D)), "k:"), (lambda: dict(v=z(B + 1, HK, D)), "tokens"), (lambda: dict(v=z(HK, D)), "tokens"),
    (lambda: dict(seq=i32(B - 1)), "tokens"), (lambda: dict(pos=i32(B + 1)), "tokens"),
    (lambda: dict(k=z(B, HK, D, dtype=torch.float16)), "k:"), (lambda: dict(v=z(B, HK, D, dtype=torch.float32)), "v:"),
    (lambda: dict(k=z(B, HK, D, device="cpu")), "k:"), (lambda: dict(v=z(B, HK, D, device="cpu")), "v:"),
    (lambda: dict(k=z(B, HK + 1, D)), "k:"), (lambda: dict(v=z(B, HK, D + 8)), "v:"), (lambda: dict(k=z(HK, B, D).transpose(0, 1)), "k:"),
    (lambda: dict(v=z(B, HK, 2 * D)[..., ::2]), "v:"), (lambda: dict(k=z(B, HK, 2 * D)[..., :D]), "k:"),
    (lambda: dict(q=z(B + 1, H, D)), "as many tokens"), (lambda: dict(q_out=z(B - 1, H, D)), "as many tokens"), (lambda: dict(q=z(B, H * D)), "as many tokens"),
    (lambda: dict(q=z(B, H - 1, D)), "q:"), (lambda: dict(q_out=z(B, H, D, dtype=torch.float16)), "q_out:"), (lambda: dict(q=z(B, H, D, device="cpu")), "q:"),
    (lambda: dict(q_out=z(H, B, D).transpose(0, 1)), "q_out:"),
    (lambda: dict(table=i32(B, WIDTH).long()), "table:"), (lambda: dict(table=i32(B * WIDTH)), "table:"), (lambda: dict(table=i32(B, WIDTH, device="cpu")), "table:"),
    (lambda: dict(table=i32(WIDTH, B).t()), "table:"),
    (lambda: dict(seq=i32(B).long()), "seq:"), (lambda: dict(pos=i32(B, device="cpu")), "pos:"), (lambda: dict(seq=i32(2 * B)[::2]), "seq:"),
    (lambda: dict(pos=i32(B).float()), "pos:"),
])
def test_append_refuses(kv, bad, word):
    refused(append, kv, append_good, bad, word, V)


def attend(kv, q, out, seq_len, table, **kw):
    ls.ls_paged_kv_attend(kv, q, out, seq_len, table, **kw)


def attend_good():
    return dict(q=z(B, M, H, D), out=z(B, M, H, D), seq_len=i32(B), table=i32(B, WIDTH), prefix_pages=i32(2), prefix_len=20, lse=z(B, M, H, dtype=torch.float32))


@pytest.mark.parametrize("bad,word,error", [
    (lambda: dict(q=None), "q", V), (lambda: dict(out=0), "out", V), (lambda: dict(seq_len=None), "seq_len", V), (lambda: dict(table=None), "table", V),
    (lambda: dict(q=z(H, D)), "q:", V), (lambda: dict(q=z(1, B, M, H, D)), "q:", V), (lambda: dict(out=z(B, M, H, D + 8)), "out:", V),
    (lambda: dict(out=z(B * M, H, D)), "out:", V), (lambda: dict(q=z(B, M, H, D, dtype=torch.float16)), "q:", V), (lambda: dict(q=z(B, M, H, D, device="cpu")), "q:", V),
    (lambda: dict(out=z(B, M, H, D, dtype=torch.float32)), "out:", V), (lambda: dict(out=z(B, M, H, D, device="cpu")), "out:", V),
    (lambda: dict(q=z(B, M, H + 1, D), out=z(B, M, H + 1, D)), "q:", V), (lambda: dict(q=z(B, M, D, H).transpose(2, 3)), "q:", V),
    (lambda: dict(q=z(M, B, H, D).transpose(0, 1)), "evenly", V), (lambda: dict(out=z(B, M + 1, H, D)[:, :M]), "evenly", V),
    (lambda: dict(seq_len=i32(B + 1)), "one row", V), (lambda: dict(table=i32(B - 1, WIDTH)), "one row", V), (lambda: dict(seq_len=i32(B).long()), "seq_len:", V),
    (lambda: dict(seq_len=i32(B, device="cpu")), "seq_len:", V), (lambda: dict(seq_len=i32(2 * B)[::2]), "seq_len:", V), (lambda: dict(table=i32(B, WIDTH).long()), "table:", V),
    (lambda: dict(table=i32(WIDTH, B).t()), "table:", V),
    (lambda: dict(prefix_pages=None), "prefix_pages", V), (lambda: dict(prefix_pages=i32(1)), "too few", V), (lambda: dict(prefix_pages=i32(2).long()), "prefix_pages:", V),
    (lambda: dict(prefix_pages=i32(2, device="cpu")), "prefix_pages:", V), (lambda: dict(prefix_pages=i32(4)[::2]), "prefix_pages:", V),
    (lambda: dict(lse=z(B, M, H)), "lse:", V), (lambda: dict(lse=z(B, H, dtype=torch.float32)), "lse:", V), (lambda: dict(lse=z(B, M, H, dtype=torch.float32, device="cpu")), "lse:", V),
    (lambda: dict(lse=z(B, M, 2 * H, dtype=torch.float32)[..., ::2]), "lse:", V), (lambda: dict(lse=1.0), "lse", V),
    (lambda: dict(window=2 ** 31), "32 bits", V), (lambda: dict(prefix_len=2 ** 40), "too few", V), (lambda: dict(prefix_len=-2 ** 40), "32 bits", V),
    (lambda: dict(window="w"), "int", T), (lambda: dict(prefix_len=1.5), "int", T), (lambda: dict(scale="s"), "", T), (lambda: dict(window=2 ** 70), "", OverflowError),
    (lambda: dict(window=-1), "negative", L), (lambda: dict(prefix_len=-1), "negative", L), (lambda: dict(scale=0.0), "scale", L), (lambda: dict(scale=float("nan")), "scale", L),
    (lambda: dict(q=z(B, M + 1, H, D), out=z(B, M + 1, H, D), lse=None), "created for", L),
    (lambda: dict(q=z(B + 1, M, H, D), out=z(B + 1, M, H, D), lse=None, seq_len=i32(B + 1), table=i32(B + 1, WIDTH)), "created for", L),
])
def test_attend_refuses(kv, bad, word, error):
    refused(attend, kv, attend_good, bad, word, error)


def norm(kv, x, y, x_out, h, **kw):
    ls.ls_block_norm(x, y, x_out, h, **kw)


F32 = torch.float32


def norm_good():
    return dict(x=z(4, 48, dtype=F32), y=z(4, 48), x_out=z(4, 48, dtype=F32), h=z(4, 48), post_norm=True, w_post=z(48, dtype=F32), gate=z(4, 48), w_pre=z(48, dtype=F32))


@pytest.mark.parametrize("bad,word,error", [
    (lambda: dict(x=None), "x", V), (lambda: dict(y=1), "y", V), (lambda: dict(x_out=1), "x_out", V), (lambda: dict(h=()), "h", V), (lambda: dict(gate=1), "gate", V),
    (lambda: dict(w_post=2), "w_post", V), (lambda: dict(w_pre=2), "w_pre", V),
    (lambda: dict(x=z(2, 2, 48, dtype=F32)), "x:", V), (lambda: dict(x=z(4, 48, dtype=F32, device="cpu")), "x:", V), (lambda: dict(x=z(4, 96, dtype=F32)[:, ::2]), "x:", V),
    (lambda: dict(y=z(3, 48)), "y:", V), (lambda: dict(y=z(4, 40)), "y:", V), (lambda: dict(y=z(48)), "y:", V), (lambda: dict(y=z(4, 48, device="cpu")), "y:", V),
    (lambda: dict(y=z(48, 4).t()), "y:", V), (lambda: dict(h=z(4, 48, dtype=torch.float16)), "one type", V), (lambda: dict(h=z(4, 40)), "h:", V),
    (lambda: dict(h=z(4, 48, device="cpu")), "h:", V), (lambda: dict(x_out=z(4, 48)), "x_out", V), (lambda: dict(x_out=z(5, 48, dtype=F32)), "x_out:", V),
    (lambda: dict(x_out=z(4, 48, dtype=F32, device="cpu")), "x_out:", V),
    (lambda: dict(gate=z(4, 48, dtype=torch.float16)), "one type", V), (lambda: dict(gate=z(47)), "gate:", V), (lambda: dict(gate=z(3, 48)), "gate:", V),
    (lambda: dict(gate=z(48, device="cpu")), "gate:", V), (lambda: dict(gate=z(96)[::2]), "gate:", V),
    (lambda: dict(w_post=z(48)), "w_post:", V), (lambda: dict(w_post=z(47, dtype=F32)), "w_post:", V), (lambda: dict(w_post=z(48, dtype=F32, device="cpu")), "w_post:", V),
    (lambda: dict(w_pre=z(96, dtype=F32)[::2]), "w_pre:", V), (lambda: dict(w_pre=z(49, dtype=F32)), "w_pre:", V),
    (lambda: dict(x=z(4, 48, dtype=torch.float64), x_out=None), "dtype", V), (lambda: dict(y=i32(4, 48), h=None, gate=None), "dtype", V),
    (lambda: dict(eps="e"), "", T), (lambda: dict(scale=None), "", T),
    (lambda: dict(x=z(4, 48, dtype=torch.float16), x_out=None), "residual", L), (lambda: dict(x_out=None, h=None), "required", L), (lambda: dict(y=None, gate=None), "needs", L),
    (lambda: dict(y=None, w_post=None), "needs", L), (lambda: dict(eps=-1.0), "eps", L), (lambda: dict(x=z(1, 48, dtype=F32).expand(4, 48)), "stride", L),
])
def test_norm_refuses(kv, bad, word, error):
    refused(norm, kv, norm_good, bad, word, error)


def test_a_closed_cache_is_refused():
    k = ls.ls_paged_kv_create(z(5, PAGE, HK, D), z(5, PAGE, HK, D), H, max_seqs=B, max_q_len=M)
    k.close()
    k.close()
    with pytest.raises(ValueError):
        append(k, **append_good())
    with pytest.raises(ValueError):
        attend(k, **attend_good())
    with pytest.raises(ls.LeanStreamError):
        ls.ls_paged_kv_status(k)
