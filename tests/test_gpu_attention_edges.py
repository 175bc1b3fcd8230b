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


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,hk,seqs,prefix", [(2, 2, 1, 0), (16, 1, 1, 0), (32, 1, 1, 0), (64, 1, 3, 1500), (20, 1, 3, 1500)])
@pytest.mark.parametrize("far", [17.5, 20.0])
def test_many_keys_far_below_a_strong_one(dtype, heads, hk, seqs, prefix, far):
    """A strong key in every tile, whose value is zero, beside 127 keys e^-far below it: what they weigh together is all of the output.
    Tolerance: a weight is rounded to 16 bits relative to itself (u), in fp16 by no more than 2^-32 of the row's largest (its smallest
    step is 2^-24, weights are held 2^7 above what the sum divides by); the output once more."""
    b = Batch(dtype=dtype, heads=heads, hk=hk, D=64, page=64, lens=[prefix + 1500 + 10 * s for s in range(seqs)], prefix=prefix, seed=7)
    b.q.zero_()
    b.q[..., 0] = 16.0  # the score is 2 k[0]
    gen = torch.Generator(device=DEV).manual_seed(11)
    pages = [(b.prefix_pages, 0, prefix)] if prefix else []
    pages += [(b.table[s], prefix, n) for s, n in enumerate(b.lens)]
    for ids, lo, hi in pages:
        p = torch.arange(lo, hi, device=DEV)
        pg, sl = ids[p // b.page].long(), p % b.page
        strong = p % 128 == 64
        k = torch.zeros(hi - lo, hk, 64, device=DEV)
        k[strong, :, 0] = far / 2
        v = 200 + 800 * torch.rand(hi - lo, hk, 64, generator=gen, device=DEV)
        v[strong] = 0
        b.kp[pg, sl], b.vp[pg, sl] = k.to(b.kp.dtype), v.to(b.vp.dtype)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    u = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    for s, n in enumerate(b.lens):
        p = np.arange(n)
        ids = np.where(p < prefix, b.prefix_np[np.minimum(p // b.page, max(len(b.prefix_np) - 1, 0))] if prefix else 0, b.table_np[s][p // b.page])
        k, v = f64(b.kp)[ids, p % b.page], f64(b.vp)[ids, p % b.page]
        for h in range(heads):
            kh, vh = k[:, h * hk // heads], v[:, h * hk // heads]
            w = np.exp(2 * kh[:, 0] - far)
            ref, absv = (w @ vh) / w.sum(), vh.sum(0) / w.sum()
            tol = (2 * u + 2.0 ** -18) * ref + (2.0 ** -32 * absv if dtype == "fp16" else 0.0) + 2.0 ** -24
            got = f64(b.out[s, 0, h])
            assert (np.abs(got - ref) <= tol).all(), (s, h, got[:3], ref[:3], tol[:3])
            assert abs(float(b.lse[s, 0, h]) - (far + np.log(w.sum()))) <= 2.0 ** -16
    assert ls.ls_paged_kv_status(kv) == 0
    kv.close()


@pytest.mark.parametrize("D,heads", [(64, 2), (96, 2), (64, 40)])
@pytest.mark.parametrize("q_len", [1, 3])
def test_positions_near_the_end_of_32_bits(D, heads, q_len):
    """A table that reaches 2^31 positions (all of them slots of one page), lengths at and beyond the last position that is counted: the
    last keys are seen, longer lengths are reported and cut there."""
    page, last = 65536, 2 ** 31 - 65536
    gen = torch.Generator(device=DEV).manual_seed(0)
    kp, vp = (torch.randn(1, page, 1, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(1, q_len, heads, D, generator=gen, device=DEV).bfloat16()
    table = torch.zeros(1, 2 ** 31 // page, dtype=torch.int32, device=DEV)
    kv = ls.ls_paged_kv_create(kp, vp, heads, max_seqs=1, max_q_len=q_len)
    for n, status in ((last, 0), (2 ** 31 - 1, ls.LS_ERR_INVALID), (last - 7, 0), (2 ** 31 - 200, ls.LS_ERR_INVALID)):
        out = torch.full_like(q, float("nan"))
        ls.ls_paged_kv_attend(kv, q, out, torch.tensor([n], dtype=torch.int32, device=DEV), table, window=150)
        assert ls.ls_paged_kv_status(kv) == status
        for i in range(q_len):
            hi = min(n, last) - q_len + i + 1
            p = torch.arange(hi - 150, hi, device=DEV) % page
            k, v = kp[0, p, 0].double(), vp[0, p, 0].double()
            w = torch.softmax(q[0, i].double() @ k.T * D ** -0.5, -1)
            assert ((out[0, i].double() - w @ v).abs() <= 2.0 ** -8 * (w @ v.abs() * 1.1 + (w @ v).abs()) + 2.0 ** -24).all()
    with pytest.raises(ls.LeanStreamError, match="prefix_len"):
        ls.ls_paged_kv_attend(kv, q, out, torch.tensor([n], dtype=torch.int32, device=DEV), table, table[0], last + 1, window=150)
    kv.close()


def test_a_handle_is_ready_for_any_stream_when_it_is_made():
    """A report of a call right behind the handle's creation, or behind a status call, on a stream that does not wait for the default
    one is not wiped by their clearing (which the default stream may be late with)."""
    st = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    b = Batch(D=64, lens=[200, 90])
    b.table[0, 2] = -1
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(torch.cuda.default_stream()):
            for _ in range(20):
                busy @ busy
        kv = b.handle()
        for _ in range(3):
            b.attend(kv, stream=st)
            assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID
        b.attend(kv, stream=st)
        assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID and ls.ls_paged_kv_status(kv) == 0
        kv.close()
