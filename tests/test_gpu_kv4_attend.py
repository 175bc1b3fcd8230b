"""ls_paged_kv4_attend against the plain 64-bit form over what the pages hold, at the sizes, layouts and masks where it can go wrong.

Bounds, with u = 2^-8 (bf16) or 2^-11 (fp16) for the last rounding:
  scores: fp32 sums of q (s u + z), which may truncate: ds = 2^-21 sum |q| (s u + |z|) scale;
  a weight: exponent of an inexact score, 2 ds + 2^-18, of sum w |v|;
  weights times scales in fp16: 2^-11 of sum w s |u - 8|, and, as the largest of a row stands at 2^4 or above when it is met, 2^-25 x 8 / 2^4
  of it for every key whose product falls under the smallest normal number: 2^-26 n max(w s);
  sums of the parts in fp32 (16 s and z, up to n terms in runs of 16 keys): 2^-20 of sum w (16 s + |z|)."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def f64(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """A filled cache: positions that belong to a sequence hold data, all other bytes are 255 (scales and zeros that are NaN), and table
    entries that need not be read are far outside the pool."""

    def __init__(self, dtype="bf16", heads=8, hk=2, D=128, group=64, page=16, lens=(5,), q_len=1, window=0, seed=0, std=2.0, q_view="plain", vstd=None, strided=False):
        self.__dict__.update(dtype=dtype, heads=heads, hk=hk, D=D, group=group, page=page, lens=list(lens), q_len=q_len, window=window)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        dt, B = orc.DT[dtype], len(lens)
        width = max(1, max(-(-n // page) for n in lens))
        total = sum(-(-n // page) for n in lens) + 2
        block = ls.ls_paged_kv4_block_bytes(page, D, group)
        raw = torch.full((total, hk, block + 16), 255, dtype=torch.uint8, device=DEV)
        self.pages = raw[:, :, 16:] if strided else raw[:, :, :block].contiguous()
        ids = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        table = np.full((B, width), 2 ** 30, dtype=np.int32)
        for b, n in enumerate(lens):
            for j in range(-(-n // page)):
                table[b, j] = ids.pop()
        self.table_np, self.table = table, torch.from_numpy(table).to(DEV)
        self.seq_len = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        filler = ls.ls_paged_kv4_create(self.pages, heads, D, page, dtype=dt, group=group)
        for b, n in enumerate(lens):
            if n:
                k, v = (torch.randn(n, hk, D, generator=gen, device=DEV) for _ in range(2))
                if vstd:  # values whose size differs from token to token
                    v = v * torch.exp(torch.randn(n, 1, 1, generator=gen, device=DEV) * vstd)
                pos = torch.arange(n, dtype=torch.int32, device=DEV)
                ls.ls_paged_kv4_append(filler, None, k.to(dt), v.to(dt), None, torch.full_like(pos, b), pos, self.table)
        assert ls.ls_paged_kv4_status(filler) == 0
        filler.close()
        self.q = (torch.randn(B, q_len, heads, D, generator=gen, device=DEV) * std).to(dt)
        if q_view == "fused":  # a slice of a wider projection
            wide = torch.zeros(B, q_len, heads + 2 * hk, D, dtype=dt, device=DEV)
            wide[:, :, :heads] = self.q
            self.q = wide[:, :, :heads]
        self.out = torch.full((B, q_len, heads, D), float("nan"), dtype=dt, device=DEV)
        if q_view == "misaligned":
            flat = torch.zeros(2, self.q.numel() + 1, dtype=dt, device=DEV)
            flat[0, 1:] = self.q.reshape(-1)
            self.q = flat[0, 1:].view(B, q_len, heads, D)
            flat = torch.full((self.out.numel() + 1,), float("nan"), dtype=dt, device=DEV)
            self.out = flat[1:].view(B, q_len, heads, D)
        self.lse = torch.full((B, q_len, heads), float("nan"), device=DEV)
        self.scale = D ** -0.5

    def handle(self, max_seqs=None, max_q_len=None):
        return ls.ls_paged_kv4_create(self.pages, self.heads, self.D, self.page, dtype=orc.DT[self.dtype], group=self.group, max_seqs=max_seqs or len(self.lens),
                                      max_q_len=max_q_len or self.q_len)

    def attend(self, kv, **kw):
        ls.ls_paged_kv4_attend(kv, self.q, self.out, self.seq_len, self.table, window=self.window, lse=self.lse, **kw)

    def check(self):
        torch.cuda.synchronize()
        ref, lse, e, absqk = orc.attend(f64(self.q), self.pages.cpu().numpy(), self.page, self.group, self.dtype, self.lens, self.table_np, self.window, self.scale)
        got, got_lse = f64(self.out), f64(self.lse)
        assert np.isfinite(got).all(), "not finite"
        n = max(self.lens + [1])
        ds = absqk * self.scale * 2.0 ** -21
        tol = ((2 * ds + 2.0 ** -18)[..., None] * e["absout"] + 2.0 ** -11 * e["rounded"] + 2.0 ** -26 * n * e["top"] + 2.0 ** -20 * e["parts"]
               + U[self.dtype] * np.abs(ref) * (1 + 2.0 ** -6) + 2.0 ** -24)
        bad = np.abs(got - ref) - tol
        assert bad.max() <= 0, f"out off by {np.abs(got - ref).max():.3e}, over by {bad.max():.3e} at {np.unravel_index(bad.argmax(), bad.shape)}"
        empty = np.isneginf(lse)
        assert np.isneginf(got_lse[empty]).all() and (got[empty] == 0).all()
        lt = ds + n * 2.0 ** -24 + 2.0 ** -18 + np.abs(np.where(empty, 0, lse)) * 2.0 ** -22
        d = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, lse))
        assert (d <= lt).all(), f"lse off by {d.max():.3e}"


def run_case(repeat=2, **kw):
    b = Batch(**kw)
    kv = b.handle()
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == 0
    b.check()
    first = b.out.clone()
    for _ in range(repeat):
        b.out.fill_(float("nan"))
        b.attend(kv)
        torch.cuda.synchronize()
        assert torch.equal(first, b.out), "the same call twice differs"
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 300, 1000])
def test_single_token_lengths(dtype, D, n):
    run_case(dtype=dtype, D=D, lens=[n], seed=n)


@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("q_len", [1, 2, 3, 4, 9])
def test_groups_and_rows(D, group, q_len):
    """4 query heads to a key head: 4, 8, 12, 16 and 36 rows, one and two tiles of them."""
    run_case(D=D, group=group, q_len=q_len, lens=[70, 0, 333], seed=group)
    run_case(D=D, group=group, q_len=q_len, lens=[50, 129], dtype="fp16", page=48, window=40, seed=group + 1)


@pytest.mark.parametrize("heads,hk", [(1, 1), (4, 4), (8, 1), (7, 1), (12, 4), (71, 1), (128, 1), (40, 8), (64, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_head_layouts(heads, hk, D):
    run_case(heads=heads, hk=hk, D=D, lens=[70, 0, 300], seed=heads)
    run_case(heads=heads, hk=hk, D=D, lens=[210, 0, 180, 131], q_len=2, seed=heads + 1, dtype="fp16")


@pytest.mark.parametrize("page", [16, 32, 48, 64, 128, 208])
@pytest.mark.parametrize("strided", [False, True])
def test_pages(page, strided):
    run_case(page=page, lens=[1, page - 1, page, page + 1, 5 * page + 3], strided=strided, seed=page)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 300, 2 ** 31 - 1])
@pytest.mark.parametrize("q_len", [1, 5])
def test_windows(window, q_len):
    run_case(window=window, q_len=q_len, lens=[3, 16, 17, 290, 0, 500], seed=window % 1000)


@pytest.mark.parametrize("q_len", [1, 3, 8, 20])
def test_sequences_shorter_than_the_queries(q_len):
    """Tokens that stand before their sequence's start see nothing: zeros and -inf."""
    run_case(q_len=q_len, lens=[1, 2, 0, 7, 19, 40], seed=q_len)
    run_case(q_len=q_len, lens=[1, 2, 0, 7, 19, 40], window=3, seed=q_len, dtype="fp16", D=64)


@pytest.mark.parametrize("q_view", ["fused", "misaligned"])
def test_query_views(q_view):
    run_case(q_view=q_view, lens=[33, 100], q_len=3)
    run_case(q_view=q_view, lens=[33, 100], D=64, dtype="fp16")


@pytest.mark.parametrize("lens", [[4000], [4097, 1], [1] * 300, [17] * 700, [0] * 5, [0, 0, 2500, 0], list(range(0, 640, 5))])
@pytest.mark.parametrize("hk", [1, 2])
def test_cuts(lens, hk):
    """Long units over many teams, many short units, empty sequences in front, between and behind."""
    run_case(lens=lens, heads=2 * hk, hk=hk, seed=len(lens))


@pytest.mark.parametrize("lens,heads,hk", [([30000], 8, 1), ([9000, 20000, 123], 16, 2), ([2000] * 12, 8, 8)])
def test_long(lens, heads, hk):
    run_case(lens=lens, heads=heads, hk=hk, page=64, D=64)
    run_case(lens=lens, heads=heads, hk=hk, page=64, D=128, group=128, dtype="fp16", q_len=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("std", [0.0, 1e-3, 30.0])
def test_score_ranges(dtype, std):
    """Flat rows, and rows that one key takes (the running reference has to move many times)."""
    run_case(dtype=dtype, std=std, lens=[600, 45])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_of_very_different_sizes(dtype):
    run_case(dtype=dtype, vstd=2.0, lens=[700, 45], std=3.0)


def test_rising_scores():
    """Every tile's largest score is above the last one's by far more than the reference's room."""
    b = Batch(lens=[800], heads=2, hk=1, std=1.0)
    kv = ls.ls_paged_kv4_create(b.pages, 2, 128, 16, max_seqs=1, max_q_len=1)
    k = torch.zeros(800, 1, 128, device=DEV)
    k[:, 0, :] = torch.linspace(0, 40, 800, device=DEV)[:, None] * torch.linspace(0.5, 1, 128, device=DEV)
    v = torch.randn(800, 1, 128, device=DEV)
    pos = torch.arange(800, dtype=torch.int32, device=DEV)
    ls.ls_paged_kv4_append(kv, None, k.bfloat16(), v.bfloat16(), None, torch.zeros_like(pos), pos, b.table)
    b.q.fill_(1.0)
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == 0
    b.check()
    kv.close()


def test_a_token_that_is_not_finite_stays_with_those_who_see_it():
    """Four draft tokens; the key of the last one and a value of the third hold NaN: earlier tokens are as without them."""
    b = Batch(lens=[50, 20], q_len=4, heads=4, hk=2)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    clean = b.out.clone()
    pos = torch.tensor([48, 49], dtype=torch.int32, device=DEV)
    k, v = (torch.randn(2, 2, 128, device=DEV).bfloat16() for _ in range(2))
    k[1], v[0, 0, 3] = float("inf"), float("nan")
    ls.ls_paged_kv4_append(kv, None, k, v, None, torch.zeros_like(pos), pos, b.table)
    b.attend(kv)
    torch.cuda.synchronize()
    assert torch.equal(b.out[1], clean[1]) and torch.equal(b.out[0, :2], clean[0, :2])
    assert torch.isnan(b.out[0, 2, :2, :64]).all() and torch.isfinite(b.out[0, 2, :2, 64:]).all() and torch.isfinite(b.out[0, 2, 2:]).all()
    assert torch.isnan(b.out[0, 3]).all()
    kv.close()


def test_lengths_and_pages_that_are_out_of_range():
    b = Batch(lens=[40, 64, 33], q_len=1)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    clean = b.out.clone()
    b.seq_len[1] = 10 ** 9  # beyond the table: as the table's 64
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == -1
    assert torch.equal(b.out, clean)
    b.seq_len[1] = -3
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == -1
    assert (b.out[1] == 0).all() and torch.isneginf(b.lse[1]).all() and torch.equal(b.out[0], clean[0]) and torch.equal(b.out[2], clean[2])
    b.seq_len[1] = 64
    b.table[0, 1], b.table[2, 2] = -7, b.pages.shape[0]
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == -1
    got = b.out.clone()
    # the same with those pages' positions left out: attention over what remains
    keep = [p for p in range(40) if p // 16 != 1]
    ref = []
    table = b.table_np.copy()
    K, V = (orc.values(x) for x in orc.held(b.pages.cpu().numpy(), 16, 128, 64, "bf16"))
    pos = np.array(keep)
    k, v = K[table[0][pos // 16], pos % 16], V[table[0][pos // 16], pos % 16]
    q = f64(b.q)[0, 0]
    for h in range(8):
        s = k[:, h // 4] @ q[h] * b.scale
        w = np.exp(s - s.max())
        ref.append((w / w.sum()) @ v[:, h // 4])
    assert np.abs(f64(got[0, 0]) - np.array(ref)).max() < 2.0 ** -8 * 4 * 2
    assert torch.equal(got[1], clean[1]) and torch.isfinite(got).all()
    kv.close()


def test_rows_behind_the_batch_stay_as_they_were():
    b = Batch(lens=[40, 0, 33], q_len=2)
    kv = b.handle(max_seqs=8, max_q_len=5)
    big = torch.full((6, 2, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    b.out, b.lse = big[:3], torch.full((3, 2, 8), float("nan"), device=DEV)
    b.attend(kv)
    b.check()
    assert (big[3:] == 7.0).all()
    kv.close()


def test_streams_graphs_and_other_lengths_in_between():
    """A captured call replayed on new lengths, an eager call of another handle between, both on a stream that is not the default one."""
    b, other = Batch(lens=[900, 30], heads=16, hk=2), Batch(lens=[300] * 5, D=64, seed=9)
    kv, kv2 = b.handle(), other.handle()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        b.attend(kv)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            b.attend(kv)
        for lens in ([900, 30], [17, 0], [0, 0], [899, 29], [1, 30]):
            b.lens = lens
            b.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
            b.out.fill_(float("nan"))
            graph.replay()
            other.attend(kv2)
            graph.replay()
            b.check()
            other.check()
    assert ls.ls_paged_kv4_status(kv) == 0 and ls.ls_paged_kv4_status(kv2) == 0
    kv.close()
    kv2.close()


def test_calls_back_to_back():
    """Append, attention, append ... without a wait between: each sees what the one before stored."""
    B, steps = 3, 40
    b = Batch(lens=[steps] * B, heads=4, hk=2)
    final = b.handle()
    b.pages.fill_(255)
    gen = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(steps, B, 2, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    seq = torch.arange(B, dtype=torch.int32, device=DEV)
    lens = [torch.full((B,), t + 1, dtype=torch.int32, device=DEV) for t in range(steps)]
    outs = torch.empty(steps, B, 1, 4, 128, dtype=torch.bfloat16, device=DEV)
    for t in range(steps):
        ls.ls_paged_kv4_append(final, None, k[t], v[t], None, seq, lens[t] - 1, b.table)
        ls.ls_paged_kv4_attend(final, b.q, outs[t], lens[t], b.table, lse=b.lse)
    torch.cuda.synchronize()
    for t in (0, 15, 16, 39):
        b.lens, b.out = [t + 1] * B, outs[t]
        ls.ls_paged_kv4_attend(final, b.q, outs[t], lens[t], b.table, lse=b.lse)
        assert ls.ls_paged_kv4_status(final) == 0
        b.check()
    final.close()


@pytest.mark.parametrize("q_len", [1, 4])
def test_idle_slots(q_len):
    """Most slots of a batch idle, a few long: the idle ones take no part, wherever they stand; rows that lie off 16 bytes too."""
    lens = [0] * 120
    for i, n in ((0, 700), (1, 1), (63, 1500), (64, 2), (118, 33)):
        lens[i] = n
    run_case(lens=lens, q_len=q_len, seed=q_len)
    run_case(lens=lens[1:], q_len=q_len, D=64, dtype="fp16", q_view="misaligned", window=50)
    run_case(lens=[3] * 150 + [5000], q_len=q_len, heads=4, hk=1)


def test_a_table_without_columns_and_no_lse():
    b = Batch(lens=[20, 5])
    kv = b.handle()
    b.attend(kv)
    out = torch.full_like(b.out, float("nan"))
    ls.ls_paged_kv4_attend(kv, b.q, out, b.seq_len, b.table, lse=None)
    assert ls.ls_paged_kv4_status(kv) == 0 and torch.equal(out, b.out)
    ls.ls_paged_kv4_attend(kv, b.q, out, b.seq_len, b.table[:, :0].contiguous(), lse=b.lse)
    assert ls.ls_paged_kv4_status(kv) == -1  # (lengths beyond a table of nothing)
    assert (out == 0).all() and torch.isneginf(b.lse).all()
    ls.ls_paged_kv4_attend(kv, b.q, out, torch.zeros_like(b.seq_len), b.table[:, :0].contiguous())
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()


def test_tables_of_all_positions():
    """Tables of 2^31 positions: a launch's line of blocks cannot hold all sequences, or, refused, not even one."""
    b = Batch(lens=[2050, 0, 37, 1024, 1], heads=8, hk=4, page=1024)
    kv = b.handle()
    wide = torch.full((5, 2 ** 21), 2 ** 30, dtype=torch.int32, device=DEV)
    wide[:, : b.table.shape[1]] = b.table
    b.table = wide
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == 0
    b.check()
    kv.close()
    many = Batch(lens=[40], heads=16, hk=16, page=1024)
    kv = many.handle()
    with pytest.raises(ls.LeanStreamError, match="too large"):
        ls.ls_paged_kv4_attend(kv, many.q, many.out, many.seq_len, wide[:1])
    many.attend(kv)
    many.check()
    kv.close()


def test_shares_of_sequences_of_many_millions():
    """One page listed R times by as many sequences as there are processors, each a share of its own: the page's own result, and a log of
    the sum that is larger by log R.  A warp adds up R 512 / 12 pairs of tiles; a pair adds up to 4 2^-24 of rounding to the sum of weights and
    2 2^-23 to the sums of values."""
    page, R = 16384, 2930
    b = Batch(lens=[page], heads=1, hk=1, D=64, page=page)
    kv = b.handle()
    b.attend(kv)
    b.check()
    kv.close()
    S = torch.cuda.get_device_properties(0).multi_processor_count
    kv = b.handle(max_seqs=S)
    table = b.table[:, :1].expand(S, R).contiguous()
    out, lse = torch.full((S, 1, 1, 64), float("nan"), dtype=b.q.dtype, device=DEV), torch.full((S, 1, 1), float("nan"), device=DEV)
    ls.ls_paged_kv4_attend(kv, b.q.expand(S, -1, -1, -1).contiguous(), out, torch.full((S,), R * page, dtype=torch.int32, device=DEV), table, lse=lse)
    assert ls.ls_paged_kv4_status(kv) == 0
    room = R * 512 / 12 * 2.0 ** -22
    _, _, e, _ = orc.attend(f64(b.q), b.pages.cpu().numpy(), page, b.group, b.dtype, b.lens, b.table_np, 0, b.scale)
    assert (np.abs(f64(out) - f64(b.out)) <= 2 * room * e["parts"] + 2.0 ** -8 * np.abs(f64(out)) + 2.0 ** -8 * np.abs(f64(b.out))).all()
    assert (np.abs(f64(lse) - f64(b.lse) - np.log(R)) <= 2 * room).all()
    kv.close()


def test_two_handles_at_once():
    """Two caches' calls on two streams, many times: neither sees the other's workspace."""
    one, two = Batch(lens=[900, 30, 0, 2000], heads=16, hk=2, seed=3), Batch(lens=[900, 30, 0, 2000], heads=16, hk=2, seed=4)
    k1, k2 = one.handle(), two.handle()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(50):
        with torch.cuda.stream(s1):
            one.attend(k1)
        with torch.cuda.stream(s2):
            two.attend(k2)
    assert ls.ls_paged_kv4_status(k1) == 0 and ls.ls_paged_kv4_status(k2) == 0
    one.check()
    two.check()
    k1.close()
    k2.close()


@pytest.mark.parametrize("D,group", [(64, 32), (128, 32), (128, 64), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("per,q_len", [(1, 1), (1, 2), (2, 1), (1, 3), (3, 1), (2, 2), (4, 1), (1, 4), (5, 1)])
def test_few_rows(D, group, per, q_len):
    """Rows of which several copies, one for each group, fit 8 columns, and just more than that."""
    run_case(D=D, group=group, heads=3 * per, hk=3, q_len=q_len, lens=[70, 0, 1, 333, 2], seed=D + per)
    run_case(D=D, group=group, heads=3 * per, hk=3, q_len=q_len, lens=[50, 129, 2000], dtype="fp16", page=48, window=40, vstd=2.0, std=5.0, seed=group + per)


@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (256, 32)])
def test_few_rows_and_tokens_that_are_not_finite(D, group):
    """As above for two draft tokens of one head: NaN stays with the group, and with the token, that sees it."""
    b = Batch(lens=[50, 20], q_len=2, heads=2, hk=2, D=D, group=group)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    clean = b.out.clone()
    pos = torch.tensor([48, 49], dtype=torch.int32, device=DEV)
    k, v = (torch.randn(2, 2, D, device=DEV).bfloat16() for _ in range(2))
    v[0, 0, group + 3] = float("nan")
    k[1, 1, 0] = float("inf")
    ls.ls_paged_kv4_append(kv, None, k, v, None, torch.zeros_like(pos), pos, b.table)
    b.attend(kv)
    torch.cuda.synchronize()
    assert torch.equal(b.out[1], clean[1])
    hit = torch.zeros(2, 2, D, dtype=torch.bool, device=DEV)
    hit[:, 0, group:2 * group] = True
    hit[1, 1] = True
    assert torch.equal(torch.isnan(b.out[0]), hit)
    kv.close()


@pytest.mark.parametrize("heads,q_len", [(4, 1), (16, 1), (16, 2)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), 2.0 ** 125])
def test_a_query_that_is_not_finite_keeps_to_its_row(heads, q_len, what):
    """Few rows, 8 rows and 16 rows to a key head; one component of one row (2^119 times the scale and above count as not finite)."""
    b = Batch(lens=[50, 400], heads=heads, hk=2, q_len=q_len)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    clean, good, lse = b.q.clone(), b.out.clone(), b.lse.clone()
    b.q[1, 0, 1, 77] = what
    b.attend(kv)
    assert ls.ls_paged_kv4_status(kv) == 0
    assert torch.isnan(b.out[1, 0, 1]).all() and torch.isnan(b.lse[1, 0, 1])
    b.q, b.out[1, 0, 1], b.lse[1, 0, 1] = clean, good[1, 0, 1], lse[1, 0, 1]
    b.check()
    kv.close()


@pytest.mark.parametrize("heads,q_len", [(4, 1), (16, 1), (16, 2)])
@pytest.mark.parametrize("std", [2.0 ** -120, 2.0 ** -60, 2.0 ** 26, 2.0 ** 60, 2.0 ** 105, 2.0 ** 114])
def test_queries_of_any_size(heads, q_len, std):
    """The last place of a large score is far more than a weight's room: one key is left, and its value."""
    run_case(lens=[50, 400], heads=heads, hk=2, q_len=q_len, std=std)
    run_case(lens=[50, 400], heads=heads, hk=2, q_len=q_len, std=std, group=32)


@pytest.mark.parametrize("heads,group", [(2, 32), (4, 64), (16, 64), (32, 128)])
def test_scores_far_below_zero(heads, group):
    """All of them: the largest is still found, and the outputs are sums of values with weights of one."""
    b = Batch(lens=[50, 400], heads=heads, hk=2, group=group)
    kv = b.handle()
    n = 400
    k = torch.full((n, 2, 128), 1e6, device=DEV, dtype=torch.bfloat16)
    v = torch.ones(n, 2, 128, device=DEV, dtype=torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    ls.ls_paged_kv4_append(kv, None, k, v, None, torch.full_like(pos, 1), pos, b.table)
    for size in (1.0, 1e6, 1e26):  # scores about -1e9, -1e15, -1e35
        b.q.fill_(-size)
        b.attend(kv)
        assert ls.ls_paged_kv4_status(kv) == 0
        score = -128 * float(b.q[1, 0, 0, 0].abs().item()) * float(k[0, 0, 0].item()) * b.scale
        assert (b.out[1] - 1).abs().max() <= 2.0 ** -8, size
        assert (b.lse[1].double() / score - 1).abs().max() <= 2.0 ** -20, size
    kv.close()
