"""ls_paged_kv4_attend on values that are hard to sum: groups of very different sizes, constant and huge values, sums over very many keys.
Bounds are those of test_gpu_kv4_attend, for each component by itself, but for products of weights and scales under fp16's normal numbers: a group's
scales count times a power of two that brings the largest of them, s, between 1 and 64, and the largest product of a row (of any group) stands at 2^4 or above
when it is met, so that a key adds up to 2^-25 x 8 / 2^4 x 64 of w s: 2^-20 n s in all, with the largest weight at most 1."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls
from test_gpu_kv4_attend import DEV, U, Batch, f64

pytestmark = pytest.mark.gpu
# heads, key heads, tokens: two rows to a key head (a column for each group of them, where there are several), eight, sixteen
ROWS = [(4, 2, 1), (8, 1, 1), (16, 2, 2)]


def store(b, make):
    """Replaces the values of a batch: make(n) -> [n, hk, D] for each sequence (keys are drawn anew)."""
    kv = ls.ls_paged_kv4_create(b.pages, b.heads, b.D, b.page, dtype=orc.DT[b.dtype], group=b.group)
    gen = torch.Generator(device=DEV).manual_seed(77)
    for i, n in enumerate(b.lens):
        if n:
            k = torch.randn(n, b.hk, b.D, generator=gen, device=DEV)
            pos = torch.arange(n, dtype=torch.int32, device=DEV)
            ls.ls_paged_kv4_append(kv, None, k.to(orc.DT[b.dtype]), make(n).to(orc.DT[b.dtype]), None, torch.full_like(pos, i), pos, b.table)
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()


def run(b):
    kv = b.handle()
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()


def check_each_component(b):
    """As Batch.check, with nothing absolute in the bound but half of the type's smallest step, and what the head says of small products."""
    ref, _, e, absqk = orc.attend(f64(b.q), b.pages.cpu().numpy(), b.page, b.group, b.dtype, b.lens, b.table_np, b.window, b.scale)
    got, n = f64(b.out), max(b.lens)
    scales = orc.held(b.pages.cpu().numpy(), b.page, b.D, b.group, b.dtype)[1][1]
    top = np.zeros(ref.shape)
    for i, length in enumerate(b.lens):
        pos = np.arange(length)
        s = scales[b.table_np[i][pos // b.page], pos % b.page].max(0)
        top[i] = np.repeat(s, b.heads // b.hk, 0)
    ds = absqk * b.scale * 2.0 ** -21
    tol = ((2 * ds + 2.0 ** -18)[..., None] * e["absout"] + 2.0 ** -11 * e["rounded"] + 2.0 ** -20 * n * top + 2.0 ** -20 * e["parts"]
           + U[b.dtype] * np.abs(ref) * (1 + 2.0 ** -6) + (2.0 ** -25 if b.dtype == "fp16" else 2.0 ** -134))
    assert np.isfinite(got).all(), "not finite"
    over = np.abs(got - ref) / tol
    assert over.max() <= 1, f"off by {over.max():.3g} times the bound at {np.unravel_index(over.argmax(), over.shape)}"


@pytest.mark.parametrize("heads,hk,q_len", ROWS)
@pytest.mark.parametrize("D,group", [(64, 64), (128, 32), (128, 64), (128, 128), (256, 128)])
@pytest.mark.parametrize("dtype,size", [("bf16", 1.0), ("bf16", 1e17), ("bf16", 1e38), ("bf16", 1e-20), ("fp16", 60000.0)])
def test_constant_values(dtype, size, D, group, heads, hk, q_len):
    """Values that are the same within each group (all scales are 0), of one size or of random signs."""
    for signs in (False, True):
        b = Batch(dtype=dtype, heads=heads, hk=hk, q_len=q_len, D=D, group=group, lens=[400, 17])
        store(b, lambda n: size * (torch.randint(0, 2, (n, hk, D // group), device=DEV) * 2.0 - 1 if signs else torch.ones(n, hk, D // group, device=DEV)).repeat_interleave(group, -1))
        run(b)
        check_each_component(b)


@pytest.mark.parametrize("heads,hk,q_len", ROWS)
@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("dtype,octaves", [("bf16", 20), ("bf16", 28), ("bf16", 60), ("fp16", 20)])
def test_groups_of_very_different_sizes(dtype, octaves, D, group, heads, hk, q_len):
    """Values whose groups differ by 2^octaves: by group, the same for all tokens, and drawn for each token and group."""
    groups = D // group
    top = 10 if dtype == "fp16" else octaves // 2
    by_group = 2.0 ** (top - octaves * torch.arange(groups, device=DEV) / (groups - 1)).repeat_interleave(group)
    for each in (False, True):
        b = Batch(dtype=dtype, heads=heads, hk=hk, q_len=q_len, D=D, group=group, lens=[700, 45], std=3.0, seed=octaves)
        gen = torch.Generator(device=DEV).manual_seed(5)

        def make(n):
            v = torch.randn(n, hk, D, generator=gen, device=DEV)
            return v * (2.0 ** (top - octaves * torch.rand(n, hk, groups, generator=gen, device=DEV))).repeat_interleave(group, -1) if each else v * by_group

        store(b, make)
        run(b)
        check_each_component(b)


@pytest.mark.parametrize("heads,hk,q_len", ROWS)
@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (128, 128), (256, 64)])
@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** -100), ("bf16", 2.0 ** -60), ("bf16", 2.0 ** 80), ("bf16", 2.0 ** 106), ("bf16", 2.0 ** 125), ("fp16", 2.0 ** 13)])
def test_values_of_any_size(dtype, size, D, group, heads, hk, q_len):
    """All groups alike, from tiny numbers to the type's largest (heads of one group: up to 2^108, as the header says)."""
    if D == group and size > 2.0 ** 108:
        size = 2.0 ** 107
    b = Batch(dtype=dtype, heads=heads, hk=hk, q_len=q_len, D=D, group=group, lens=[400, 45], std=3.0)
    gen = torch.Generator(device=DEV).manual_seed(9)
    store(b, lambda n: size * torch.randn(n, hk, D, generator=gen, device=DEV).clamp(-3.5, 3.5))
    run(b)
    check_each_component(b)


def even_page(hk, D, group, keys, seed=0):
    """fp16 values whose scales, zeros and codes are exact in few bits: scale k / 256 (64 <= k < 128), zero a multiple of 1 / 8 in [-4, -2]."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    shape = (keys, hk, D // group, 1)
    s, z = torch.randint(64, 128, shape, generator=gen, device=DEV) / 256.0, torch.randint(-32, -15, shape, generator=gen, device=DEV) / 8.0
    u = torch.randint(0, 16, (keys, hk, D // group, group), generator=gen, device=DEV)
    u[..., 3], u[..., 17] = 0, 15
    return (s * u + z).flatten(-2)


def check_flat(b, R, seqs):
    """One page of ``b`` listed R times by each of ``seqs`` sequences, queries of zero: the page's mean.  All weights are equal.  A warp sums
    runs of up to 2^14 keys.  Of a run's mean are rounded: weights times scales, 2^-11 of `rounded`; sums of their products with codes, up to 1024 times by at most
    2^-23 of at most the run's sum over codes from the middle and that of 1024 keys over codes from 0 (a sixteenth of a run, whose codes are up to 15 and not 4 in the
    mean): 2^-12 of it; a lane's sums of weights, and of weights times the middles 8 s + z (2 at most), up to 4096 times by 2^-24 of what is there so
    far, on average half: 2^-13.  Then come the runs' and pieces' joins, 2^-23 each, and the last rounding.  A few tokens to a sequence: all but the last
    see some keys less, which count for q_len / keys."""
    b.q.zero_()
    ref, lse, e, _ = orc.attend(f64(b.q), b.pages.cpu().numpy(), b.page, b.group, b.dtype, b.lens, b.table_np, 0, b.scale)
    table = b.table[:, :1].expand(seqs, R).contiguous()
    q, lens = b.q.expand(seqs, -1, -1, -1).contiguous(), torch.full((seqs,), R * b.page, dtype=torch.int32, device=DEV)
    out, got_lse = torch.full_like(q, float("nan")), torch.full(q.shape[:3], float("nan"), device=DEV)
    kv = b.handle(max_seqs=seqs)
    ls.ls_paged_kv4_attend(kv, q, out, lens, table, lse=got_lse)
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()
    joins = R * b.page / 2 ** 14 + 12
    want, mean = ref[:, -1:], np.abs(ref[:, -1:])
    tol = U[b.dtype] * mean + (2.0 ** -11 + 2.0 ** -12 + b.q_len / (R * b.page)) * e["rounded"][:, -1:] + 2.0 ** -13 * (2 + mean) + joins * 2.0 ** -23 * (2 + mean) + 2.0 ** -25
    over = np.abs(f64(out) - want) / tol
    assert over.max() <= 1, f"off by {over.max():.3g} times the bound (of {tol.max():.2e}); outputs are of size {mean.mean():.2e}"
    assert np.abs(f64(got_lse) - np.log(R * b.page)).max() <= 2.0 ** -13 + joins * 2.0 ** -23 + 2.0 ** -20


@pytest.mark.parametrize("heads,D,group", [(2, 128, 64), (8, 128, 128), (8, 128, 64), (8, 64, 32), (8, 256, 32), (16, 128, 64), (16, 64, 64)])
def test_a_warp_that_sums_half_a_million_keys(heads, D, group):
    """As many sequences as there are warps, so that each has one to itself."""
    b = Batch(dtype="fp16", heads=heads, hk=1, D=D, group=group, page=1024, lens=[1024])
    store(b, lambda n: even_page(1, D, group, n))
    check_flat(b, 512, 12 * torch.cuda.get_device_properties(0).multi_processor_count)


@pytest.mark.parametrize("heads", [1, 8, 16])
def test_means_of_sequences_of_many_millions(heads):
    """As many sequences as processors, 48 million keys each."""
    b = Batch(dtype="fp16", heads=heads, hk=1, D=64, group=64, page=16384, lens=[16384])
    store(b, lambda n: even_page(1, 64, 64, n))
    check_flat(b, 2930, torch.cuda.get_device_properties(0).multi_processor_count)


@pytest.mark.parametrize("D,group,heads,hk,q_len", [(128, 64, 4, 2, 1), (128, 128, 8, 1, 1), (128, 32, 8, 1, 1), (128, 64, 16, 2, 2), (256, 64, 8, 1, 1)])
@pytest.mark.parametrize("size", [0.0, 1e3, 1e30])
def test_other_rows_of_a_tile(size, D, group, heads, hk, q_len):
    """Queries of one row of a key head as they were, all others of quite another size: each row within its own bound."""
    b = Batch(D=D, group=group, heads=heads, hk=hk, q_len=q_len, lens=[900, 333], vstd=1.0)
    per = heads // hk
    for row in {0, per - 1}:
        q = b.q.clone()
        b.q[:, :, [r for r in range(heads) if r % per != row]] *= size
        run(b)
        b.lse.fill_(float("nan"))
        b.attend(kv := b.handle())
        b.check()
        kv.close()
        b.q = q


@pytest.mark.parametrize("heads,D,group", [(2, 128, 32), (8, 64, 64), (16, 64, 32)])
@pytest.mark.parametrize("seqs", [1, 20, 333])
def test_means_of_shares_that_begin_and_end_inside_sequences(seqs, heads, D, group):
    """Long sequences cut among the teams anywhere: runs of a share, its pieces, their joins."""
    b = Batch(dtype="fp16", heads=heads, hk=1, D=D, group=group, page=4096, lens=[4096])
    store(b, lambda n: even_page(1, D, group, n))
    check_flat(b, 4000 if seqs < 100 else 777, seqs)


@pytest.mark.parametrize("heads,q_len,window", [(2, 1, 0), (8, 1, 37000), (8, 2, 36000), (4, 2, 0)])
def test_runs_of_sequences_with_windows_and_missing_pages(heads, q_len, window):
    """Each warp has a sequence of 40000 keys or a little less (three runs) to itself (with up to eight rows; sixteen are cut anywhere), all over the same
    pages, one of which, in the second run, is missing."""
    lens = [40000 - 13 * i for i in range(4)]
    one = Batch(heads=heads, hk=1, page=64, lens=lens[:1], q_len=q_len, window=window, D=64, std=3.0)
    S = 12 * torch.cuda.get_device_properties(0).multi_processor_count
    q, table = one.q.expand(S, -1, -1, -1).contiguous(), one.table.expand(S, -1).contiguous()
    seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV).repeat(-(-S // 4))[:S]
    kv = one.handle(max_seqs=S)
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:3], float("nan"), device=DEV)

    def call():
        ls.ls_paged_kv4_attend(kv, q, out, seq_len, table, window=window, lse=lse)

    call()
    assert ls.ls_paged_kv4_status(kv) == 0
    first, first_lse = out.clone(), lse.clone()
    for i, n in enumerate(lens):
        if heads * q_len <= 8:
            assert torch.equal(out[i::4], out[i:i + 1].expand_as(out[i::4])) and torch.equal(lse[i::4], lse[i:i + 1].expand_as(lse[i::4]))
        for at in (i, i + 4 * (S // 8), i + 4 * ((S - i - 1) // 4)):
            one.lens, one.out, one.lse = [n], out[at:at + 1], lse[at:at + 1]
            one.check()
    call()
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    # without a page of the second run: as if its keys were not there, the others' weights the larger
    table[:, 300] = -1
    call()
    assert ls.ls_paged_kv4_status(kv) == -1
    K, V = (orc.values(x)[:, :, 0] for x in orc.held(one.pages.cpu().numpy(), 64, 64, 64, "bf16"))
    for i, n in enumerate(lens):
        for m in range(q_len):
            hi = n - q_len + m + 1
            pos = np.arange(max(0, hi - window) if window else 0, hi)
            pos = pos[pos // 64 != 300]
            at = one.table_np[0][pos // 64], pos % 64
            s = f64(one.q)[0, m] @ K[at].T * one.scale
            top = s.max(1, keepdims=True)
            w = np.exp(s - top)
            ref = w @ V[at] / w.sum(1, keepdims=True)
            assert np.abs(f64(lse[i, m]) - (top[:, 0] + np.log(w.sum(1)))).max() <= 2.0 ** -14  # scores of up to 40, to 2^-20 of them
            # as the bounds of the file's head, values of unit variance, scales of up to 1/2
            assert np.abs(f64(out[i, m]) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 2.0 ** -11 * 4
    kv.close()
