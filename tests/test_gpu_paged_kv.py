"""ls_paged_kv_append and ls_paged_kv_attend against the plain 64-bit forms, at the sizes, layouts and masks where they can go
wrong.  Tolerances come from the formats: u = 2^-8 (bf16) or 2^-11 (fp16) for a rounding to 16 bits, 2^-24 in fp32."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc
from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def f64(t):
    return t.detach().double().cpu().numpy()


def make_pool(gen, n_pages, page, hk, D, dtype, layout):
    """Two pools viewed as [pages, page, heads, dim] and filled with NaN; layouts: token-major, head-major, keys and values
    interleaved in one buffer, or at an odd element offset with padded strides."""
    if layout == "head":
        k, v = (torch.full((n_pages, hk, page, D), float("nan"), dtype=dtype, device=DEV).transpose(1, 2) for _ in range(2))
    elif layout == "both":
        kv = torch.full((n_pages, 2, page, hk, D), float("nan"), dtype=dtype, device=DEV)
        k, v = kv[:, 0], kv[:, 1]
    elif layout == "odd":
        st = (page * (hk * (D + 3) + 1), hk * (D + 3) + 1, D + 3, 1)
        k, v = (torch.full((n_pages * st[0] + 1,), float("nan"), dtype=dtype, device=DEV)[1:].as_strided((n_pages, page, hk, D), st, 1) for _ in range(2))
    else:
        k, v = (torch.full((n_pages, page, hk, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    return k, v


class Batch:
    """A filled cache: every position that belongs to a sequence (or the prefix) holds data, everything else NaN."""

    def __init__(self, dtype="bf16", heads=8, hk=2, D=128, page=16, layout="token", lens=(5,), q_len=1, prefix=0, window=0, seed=0, std=2.0,
                 q_view="plain"):
        self.__dict__.update(dtype=dtype, heads=heads, hk=hk, D=D, page=page, lens=list(lens), q_len=q_len, prefix=prefix, window=window)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        dt, B = DT[dtype], len(lens)
        first, n_prefix = prefix // page, -(-prefix // page)
        width = max(1, max([-(-n // page) for n in lens] + [n_prefix]))
        total = n_prefix + sum(max(0, -(-n // page) - first) for n in lens) + 3
        self.kp, self.vp = make_pool(gen, total, page, hk, D, dt, layout)
        ids = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        pre = [ids.pop() for _ in range(n_prefix)]
        table = np.full((B, width), 2 ** 30, dtype=np.int32)  # entries that must not be read are far outside the pool
        rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dt)
        pk, pv = rnd(max(prefix, 1), hk, D), rnd(max(prefix, 1), hk, D)
        for p in range(prefix):
            self.kp[pre[p // page], p % page], self.vp[pre[p // page], p % page] = pk[p], pv[p]
        for b, n in enumerate(lens):
            for j in range(first, -(-n // page)):
                table[b, j] = ids.pop()
            if n > prefix:
                k, v = rnd(n - prefix, hk, D), rnd(n - prefix, hk, D)
                p = torch.arange(prefix, n, device=DEV)
                pg = torch.from_numpy(table[b]).to(DEV)[p // page].long()
                self.kp[pg, p % page], self.vp[pg, p % page] = k, v
        self.table_np, self.prefix_np = table, np.array(pre, dtype=np.int32)
        self.table = torch.from_numpy(table).to(DEV)
        self.prefix_pages = torch.tensor(pre, dtype=torch.int32, device=DEV) if pre else None
        self.seq_len = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.q = (torch.randn(B, q_len, heads, D, generator=gen, device=DEV) * std).to(dt)
        if q_view == "fused":  # a slice of a wider projection
            wide = torch.zeros(B, q_len, heads + 2 * hk, D, dtype=dt, device=DEV)
            wide[:, :, :heads] = self.q
            self.q = wide[:, :, :heads]
        elif q_view == "misaligned":
            flat = torch.zeros(self.q.numel() + 1, dtype=dt, device=DEV)
            flat[1:] = self.q.reshape(-1)
            self.q = flat[1:].view(B, q_len, heads, D)
        self.out = torch.full((B, q_len, heads, D), float("nan"), dtype=dt, device=DEV)
        self.lse = torch.full((B, q_len, heads), float("nan"), device=DEV)
        self.scale = D ** -0.5

    def handle(self, max_seqs=None, max_q_len=None):
        return ls.ls_paged_kv_create(self.kp, self.vp, self.heads, max_seqs=max_seqs or len(self.lens), max_q_len=max_q_len or self.q_len)

    def attend(self, kv, **kw):
        ls.ls_paged_kv_attend(kv, self.q, self.out, self.seq_len, self.table, self.prefix_pages, self.prefix, window=self.window, lse=self.lse, **kw)

    def check(self):
        torch.cuda.synchronize()
        ref, lse, absout, absv, absqk = orc.attend(f64(self.q), f64(self.kp), f64(self.vp), self.lens, self.table_np, self.prefix_np, self.prefix,
                                                   self.window, self.scale)
        got, got_lse = f64(self.out), f64(self.lse)
        assert np.isfinite(got).all(), "not finite"
        u = U[self.dtype]
        ds = (absqk * self.scale * 2.0 ** -21)[..., None]  # fp32 scores, sums that may truncate: 4 half-ulps of sum |q k|
        rel = u + 2 * ds + 2.0 ** -18                     # one weight: rounded to 16 bits, exponent of an inexact score
        tol = rel * absout + u * np.abs(ref) + (2.0 ** -25 * absv if self.dtype == "fp16" else 0.0) + 2.0 ** -24
        bad = np.abs(got - ref) - tol
        assert bad.max() <= 0, f"out off by {np.abs(got - ref).max():.3e}, over by {bad.max():.3e} at {np.unravel_index(bad.argmax(), bad.shape)}"
        empty = np.isneginf(lse)
        assert np.isneginf(got_lse[empty]).all() and (got[empty] == 0).all()
        n = max(self.lens + [1])
        lt = ds[..., 0] + n * 2.0 ** -24 + 2.0 ** -18 + np.abs(np.where(empty, 0, lse)) * 2.0 ** -22
        d = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, lse))
        assert (d <= lt).all(), f"lse off by {d.max():.3e}"


def run_case(**kw):
    b = Batch(**kw)
    kv = b.handle()
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == 0
    b.check()
    first = b.out.clone()
    for _ in range(3):
        b.out.fill_(float("nan"))
        b.attend(kv)
        torch.cuda.synchronize()
        assert torch.equal(first, b.out), "the same call twice differs"
    assert ls.ls_paged_kv_status(kv) == 0
    kv.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 300, 1000])
def test_single_token_lengths(dtype, D, n):
    run_case(dtype=dtype, D=D, lens=[n], seed=n)


@pytest.mark.parametrize("heads,hk", [(1, 1), (4, 4), (8, 1), (7, 1), (12, 4), (71, 1), (128, 1), (40, 8), (64, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_head_layouts(heads, hk, D):
    run_case(heads=heads, hk=hk, D=D, lens=[70, 0, 300], seed=heads)
    run_case(heads=heads, hk=hk, D=D, lens=[210, 0, 180, 131], prefix=130, q_len=2, seed=heads + 1, dtype="fp16")


@pytest.mark.parametrize("D", [8, 24, 80, 96, 112, 192, 256])
def test_other_head_dims(D):
    run_case(D=D, lens=[33, 0, 140], prefix=20, q_len=2, seed=D)
    run_case(D=D, heads=3, hk=3, lens=[400], seed=D, dtype="fp16")


@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 40, 64, 128, 136, 256])
@pytest.mark.parametrize("layout", ["token", "head", "both", "odd"])
def test_page_sizes_and_layouts(page, layout):
    run_case(page=page, layout=layout, lens=[150, 260, 1, 0, 155], prefix=145, seed=page)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("prefix", [1, 16, 127, 128, 129, 250, 256, 513])
def test_shared_prefix(dtype, prefix):
    """Ends of the prefix inside and at the edges of pages and tiles; sequences that end before it, at it and behind it."""
    lens = [prefix + n for n in (1, 2, 40, 128, 129, 200)] + [prefix, max(prefix - 3, 0), 0, 1]
    run_case(dtype=dtype, lens=lens, prefix=prefix, seed=prefix)


@pytest.mark.parametrize("seqs", [1, 3, 16, 17, 31, 32, 33, 65, 100])
@pytest.mark.parametrize("heads,hk", [(8, 2), (3, 3)])
def test_batch_sizes_on_a_prefix(seqs, heads, hk):
    rng = np.random.default_rng(seqs)
    run_case(heads=heads, hk=hk, D=64, lens=[300 + int(x) for x in rng.integers(0, 60, seqs)], prefix=300, seed=seqs)


@pytest.mark.parametrize("heads,hk,q_len,seqs", [(40, 40, 2, 1), (8, 8, 1, 1), (64, 8, 1, 2), (64, 8, 3, 1), (20, 20, 1, 3)])
@pytest.mark.parametrize("prefix,own", [(7021, 61), (0, 9000), (2500, 2500)])
@pytest.mark.parametrize("page", [16, 128])
def test_long_pieces(heads, hk, q_len, seqs, prefix, own, page):
    """Pieces of many tiles on every lane, several batches of page numbers, one row or a few."""
    run_case(heads=heads, hk=hk, q_len=q_len, lens=[prefix + own + 17 * b for b in range(seqs)], prefix=prefix, page=page, seed=heads + page)


@pytest.mark.parametrize("seqs", [384, 385, 1000])
def test_more_sequences_than_threads(seqs):
    rng = np.random.default_rng(seqs)
    lens = [0 if x < 10 else int(x) for x in rng.integers(0, 170, seqs)]
    run_case(heads=2, hk=1, D=64, lens=lens, prefix=33, seed=seqs)
    run_case(heads=2, hk=2, D=64, lens=lens, window=40, seed=seqs)


def test_two_handles_on_two_streams():
    """Two caches, two streams, many calls in flight: nothing of one call's workspace is another's."""
    bs = [Batch(lens=[400, 33, 0, 280], prefix=32, seed=s) for s in (1, 2)]
    kvs = [b.handle() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for _ in range(50):
        for b, kv, st in zip(bs, kvs, streams):
            b.attend(kv, stream=st)
    torch.cuda.synchronize()
    for b, kv in zip(bs, kvs):
        assert ls.ls_paged_kv_status(kv) == 0
        b.check()
        kv.close()


def test_calls_that_depend_on_each_other_back_to_back():
    """append -> attend -> norm on one stream with no wait between them, many times: each sees what the one before wrote."""
    B, heads, hk, D, page = 3, 8, 2, 128, 16
    gen = torch.Generator(device=DEV).manual_seed(0)
    kp, vp = (torch.zeros(40, page, hk, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.arange(39, dtype=torch.int32, device=DEV).view(B, 13)
    kv = ls.ls_paged_kv_create(kp, vp, heads, max_seqs=B, max_q_len=1, rope=rope_table(208, D))
    n = 150
    x = torch.randn(n, B, heads * D, generator=gen, device=DEV)
    w = (torch.randn(heads * D, (heads + 2 * hk) * D, generator=gen, device=DEV) * (heads * D) ** -0.5).bfloat16()
    seq = torch.arange(B, dtype=torch.int32, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[:, None].expand(n, B).contiguous()
    length = pos + 1

    def pass_(wait):
        kp.zero_(), vp.zero_()
        got = []
        for t in range(n):
            h = torch.empty(B, heads * D, dtype=torch.bfloat16, device=DEV)
            ls.ls_block_norm(x[t], None, None, h)
            if wait: torch.cuda.synchronize()
            q, k, v = (h @ w).view(B, heads + 2 * hk, D).split([heads, hk, hk], 1)
            qo, o = torch.empty(B, heads, D, dtype=torch.bfloat16, device=DEV), torch.empty(B, heads, D, dtype=torch.bfloat16, device=DEV)
            if wait: torch.cuda.synchronize()
            ls.ls_paged_kv_append(kv, q, k, v, qo, seq, pos[t], table)
            if wait: torch.cuda.synchronize()
            ls.ls_paged_kv_attend(kv, qo, o, length[t], table)
            if wait: torch.cuda.synchronize()
            xo = torch.empty_like(x[t])
            ls.ls_block_norm(x[t], o.view(B, -1), xo, None, post_norm=True)
            got.append(xo)
        torch.cuda.synchronize()
        return torch.stack(got)

    assert torch.equal(pass_(False), pass_(True))
    assert ls.ls_paged_kv_status(kv) == 0
    kv.close()


@pytest.mark.parametrize("q_len", [2, 3, 8, 31, 33, 130])
@pytest.mark.parametrize("prefix", [0, 150])
def test_several_tokens(q_len, prefix):
    """Tokens before position 0 (sequences shorter than q_len) see nothing; more rows than one tile holds."""
    run_case(q_len=q_len, prefix=prefix, lens=[prefix + q_len, prefix + q_len + 37, 1, 0, prefix + 140], seed=q_len)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("prefix,q_len", [(0, 1), (0, 5), (200, 1), (200, 4)])
def test_window(window, prefix, q_len):
    run_case(window=window, prefix=prefix, q_len=q_len, lens=[prefix + 10, prefix + 130, 300 + prefix, 5, 0, prefix + 513], seed=window)


@pytest.mark.parametrize("q_view", ["fused", "misaligned"])
def test_query_strides(q_view):
    run_case(q_view=q_view, lens=[40, 200, 300], prefix=33, q_len=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scores_that_grow_along_the_row(dtype):
    """Keys sorted so that the running maximum rises by far more than 2^8 over the tiles, and falls again."""
    for rising in (True, False):
        b = Batch(dtype=dtype, lens=[900], heads=4, hk=1, std=8.0, seed=3)
        order = torch.arange(900, device=DEV)
        pg, sl = b.table[0, order // b.page].long(), order % b.page
        k = b.kp[pg, sl]
        s = (k[:, 0].float() @ b.q[0, 0].float().mean(0))
        k = k[s.argsort(descending=not rising)]
        b.kp[pg, sl] = k
        kv = b.handle()
        b.attend(kv)
        b.check()
        kv.close()


def test_masked_places_may_hold_anything():
    """Unused slots and pages are NaN in every test here; also infinities of both signs, and the type's lowest value."""
    for fill in (float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min):
        b = Batch(lens=[37, 0, 150, 90], prefix=30, window=60, q_len=3)
        for t in (b.kp, b.vp):
            t[torch.isnan(t)] = fill
        kv = b.handle()
        b.attend(kv)
        torch.cuda.synchronize()
        b2 = Batch(lens=[37, 0, 150, 90], prefix=30, window=60, q_len=3)
        kv2 = b2.handle()
        b2.attend(kv2)
        b2.check()
        assert torch.equal(b.out, b2.out) and torch.equal(b.lse, b2.lse)
        kv.close(); kv2.close()


def test_scores_of_minus_infinity_and_the_lowest_value():
    """Keys that make the score -inf weigh nothing; keys at the type's lowest value make scores of about -1e38 in fp32."""
    b = Batch(lens=[200], heads=2, hk=1)
    b.q.fill_(1.0)
    p = torch.arange(0, 100, device=DEV)
    b.kp[b.table[0, p // b.page].long(), p % b.page] = float("-inf")
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    keep = np.arange(100, 200)
    k, v = (f64(t)[b.table_np[0, keep // b.page], keep % b.page][:, 0] for t in (b.kp, b.vp))
    s = k.sum(1) * b.scale
    w = np.exp(s - s.max())
    ref = (w / w.sum()) @ v
    assert np.abs(f64(b.out)[0, 0, 0] - ref).max() <= 2.0 ** -7 * np.abs(v).max()
    b.kp[b.table[0, p // b.page].long(), p % b.page] = torch.finfo(torch.bfloat16).min / 256
    b.attend(kv)
    torch.cuda.synchronize()
    assert np.abs(f64(b.out)[0, 0, 0] - ref).max() <= 2.0 ** -7 * np.abs(v).max()
    kv.close()


def test_larger_handle_smaller_calls_and_another_stream():
    b = Batch(lens=[300, 20, 0, 77], prefix=15)
    kv = b.handle(max_seqs=50, max_q_len=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.attend(kv, stream=s)
    s.synchronize()
    b.check()
    with torch.cuda.stream(s):
        b.out.fill_(float("nan"))
        b.attend(kv)
    s.synchronize()
    b.check()
    kv.close()


def test_no_lse_and_a_given_scale():
    b = Batch(lens=[300, 20])
    kv = b.handle()
    ls.ls_paged_kv_attend(kv, b.q, b.out, b.seq_len, b.table, scale=0.5)
    b.scale = 0.5
    ls.ls_paged_kv_attend(kv, b.q, torch.empty_like(b.out), b.seq_len, b.table, scale=0.5, lse=b.lse)
    b.check()
    kv.close()


def test_in_a_graph_with_changing_lengths():
    b = Batch(lens=[300, 20, 290, 310], prefix=256)
    kv = b.handle()
    b.attend(kv)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.attend(kv)
    for lens in ([300, 20, 290, 310], [257, 0, 256, 300], [1, 1, 1, 1]):
        b.lens = lens
        b.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        b.check()
    kv.close()


@pytest.mark.parametrize("D,page", [(128, 16), (96, 16), (128, 5)])
def test_out_of_range_entries_are_reported_and_not_read(D, page):
    b = Batch(D=D, page=page, lens=[200, 90], prefix=0)
    kv = b.handle()
    good = b.table.clone()
    b.table[0, 2] = 2 ** 30
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID and ls.ls_paged_kv_status(kv) == 0
    b.table[0, 2] = -1
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID
    b.table.copy_(good)
    b.seq_len[0] = 2 ** 31 - 1  # longer than its table: reported
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID
    b.seq_len[0] = -5
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID
    b.seq_len[0] = 200
    b.attend(kv)
    assert ls.ls_paged_kv_status(kv) == 0
    b.check()
    kv.close()


def test_offsets_beyond_32_bits():
    """Pools of more than 2^32 elements, the sequence in their last pages, through append and attention."""
    page, hk, D = 64, 8, 128
    n_pages = 2 ** 32 // (page * hk * D) + 40
    kp, vp = (torch.empty(n_pages, page, hk, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    n, heads = 1000, 16
    width = -(-n // page)
    table = torch.arange(n_pages - 1, n_pages - 1 - width, -1, dtype=torch.int32, device=DEV).view(1, -1)
    kv = ls.ls_paged_kv_create(kp, vp, heads, max_seqs=1, max_q_len=1)
    k, v = (torch.randn(n, hk, D, device=DEV).bfloat16() for _ in range(2))
    seq, pos = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    ls.ls_paged_kv_append(kv, None, k, v, None, seq, pos, table)
    p = pos.long()
    assert torch.equal(kp[table[0, p // page].long(), p % page], k) and torch.equal(vp[table[0, p // page].long(), p % page], v)
    q = torch.randn(1, heads, D, device=DEV).bfloat16()
    out = torch.empty_like(q)
    ls.ls_paged_kv_attend(kv, q, out, torch.tensor([n], dtype=torch.int32, device=DEV), table)
    assert ls.ls_paged_kv_status(kv) == 0
    qq, kk, vv = q[0].double().view(hk, 2, D), k.double().transpose(0, 1), v.double().transpose(0, 1)
    w = torch.softmax(qq @ kk.transpose(1, 2) * D ** -0.5, -1)
    ref, mag = (w @ vv).view(heads, D), (w @ vv.abs()).view(heads, D)
    assert ((out[0].double() - ref).abs() <= 2.0 ** -8 * (mag * 1.1 + ref.abs()) + 2.0 ** -24).all()
    kv.close()


# ---- append -----------------------------------------------------------------------------------------------------------------
def rope_table(n, r):
    a = np.arange(n)[:, None] * 10000.0 ** (-2.0 * np.arange(r // 2) / r)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float().to(DEV)


def append_case(dtype="bf16", heads=4, hk=2, D=64, page=16, layout="token", r=64, inter=False, seq=(0, 0, 1), pos=(3, 4, 30), fused=True, with_q=True,
                off=0, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, T = DT[dtype], len(seq)
    n_seqs, width = max(max(seq) + 1, 1), max(pos) // page + 2
    kp, vp = make_pool(gen, n_seqs * width + 2, page, hk, D, dt, layout)
    for t in (kp, vp):
        t.copy_(torch.randn(t.shape, generator=gen, device=DEV))
    table = torch.randperm(n_seqs * width, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(n_seqs, width).to(DEV)
    rope = rope_table(max(pos) + 1, r) if r else None
    rnd = lambda n: torch.randn(off + T * n * D, generator=gen, device=DEV).to(dt)[off:].view(T, n, D)
    q, k, v = rnd(heads + 2 * hk).split([heads, hk, hk], 1) if fused else (rnd(heads), rnd(hk), rnd(hk))
    q_out = torch.full((T, heads, D), float("nan"), dtype=dt, device=DEV)
    before = (kp.clone(), vp.clone())
    kv = ls.ls_paged_kv_create(kp, vp, heads, rope=rope, rope_interleaved=inter)
    sq, ps = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (seq, pos))
    ls.ls_paged_kv_append(kv, q if with_q else None, k, v, q_out if with_q else None, sq, ps, table)
    assert ls.ls_paged_kv_status(kv) == 0
    rt = None if rope is None else f64(rope)
    u = U[dtype]

    def close(got, ref, src, what):
        mag = np.abs(src)
        if r:
            m = mag[..., :r]
            pair = m.reshape(*m.shape[:-1], r // 2, 2).sum(-1).repeat(2, -1) if inter else np.concatenate([m[..., : r // 2] + m[..., r // 2:]] * 2, -1)
            tol = np.concatenate([u * np.abs(ref[..., :r]) + 3 * 2.0 ** -24 * pair + 2.0 ** -25, np.zeros_like(mag[..., r:])], -1)
        else:
            tol = np.zeros_like(mag)
        assert (np.abs(got - ref) <= tol).all(), what

    if with_q:
        close(f64(q_out), orc.rotate(f64(q), pos, rt, inter), f64(q), "queries")
    rk, rv, n = orc.append(f64(k), f64(v), f64(before[0]), f64(before[1]), seq, pos, f64(table).astype(int), rt, inter)
    gk, gv = f64(kp), f64(vp)
    assert np.array_equal(gv, rv)
    touched = np.zeros(gk.shape[:2], bool)
    for t in range(T):
        if seq[t] >= 0 and pos[t] >= 0:
            touched[int(table[seq[t], pos[t] // page]), pos[t] % page] = True
    assert touched.sum() == n and np.array_equal(gk[~touched], f64(before[0])[~touched])
    at = [t for t in range(T) if seq[t] >= 0 and pos[t] >= 0]
    if at:
        pg = [int(table[seq[t], pos[t] // page]) for t in at]
        sl = [pos[t] % page for t in at]
        close(gk[pg, sl], rk[pg, sl], f64(k)[at], "keys")
    kv.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,r", [(64, 64), (128, 128), (128, 64), (128, 0), (128, 16), (80, 80), (80, 20), (256, 128), (24, 10), (8, 2)])
def test_append_rotation(dtype, inter, D, r):
    append_case(dtype=dtype, inter=inter, D=D, r=r)


@pytest.mark.parametrize("layout", ["token", "head", "both", "odd"])
@pytest.mark.parametrize("page", [1, 5, 16, 64])
def test_append_layouts(layout, page):
    append_case(layout=layout, page=page, D=128, r=128, heads=8, hk=2, seq=[0] * 20 + [1] * 3, pos=list(range(7, 27)) + [0, 1, 64])


@pytest.mark.parametrize("fused,with_q,off", [(False, True, 0), (True, False, 0), (True, True, 1), (False, True, 4)])
def test_append_operands(fused, with_q, off):
    append_case(fused=fused, with_q=with_q, off=off, D=128, r=128, heads=7, hk=1)
    append_case(fused=fused, with_q=with_q, off=off, D=64, r=32, heads=40, hk=40, inter=True)


def test_append_padding_tokens_are_passed_over():
    append_case(seq=[0, -1, 1, 0, -1], pos=[5, 7, -1, 6, -3])


@pytest.mark.parametrize("heads,hk,D", [(1, 1, 64), (8, 1, 64), (8, 1, 128), (3, 3, 16), (71, 1, 128), (2, 2, 256)])
@pytest.mark.parametrize("T", [1, 5, 77])
def test_append_several_tokens_to_a_block(heads, hk, D, T):
    for with_q in (True, False):
        append_case(heads=heads, hk=hk, D=D, r=D, with_q=with_q, seq=[t % 2 for t in range(T)], pos=[3 + t // 2 for t in range(T)])


@pytest.mark.parametrize("T", [1, 2, 130, 600])
def test_append_many_tokens(T):
    append_case(heads=32, hk=8, D=128, r=128, seq=[0] * T, pos=list(range(11, 11 + T)))


def test_append_out_of_range_is_reported_and_not_written():
    kp, vp = (torch.zeros(4, 16, 2, 64, dtype=torch.float16, device=DEV) for _ in range(2))
    kv = ls.ls_paged_kv_create(kp, vp, 2, rope=rope_table(40, 64))
    k = torch.ones(1, 2, 64, dtype=torch.float16, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = i32(0, 1, 4, -1).view(1, 4)
    for seq, pos in ((1, 0), (0, 64), (0, 45), (0, 33), (0, 50)):  # no such sequence, behind the table, behind the rotation table, two pages outside the pool
        ls.ls_paged_kv_append(kv, None, k, k, None, i32(seq), i32(pos), table)
        assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID
    assert not kp.any() and not vp.any()
    kv.close()


def test_append_in_place_queries():
    kp, vp = (torch.zeros(4, 16, 2, 64, dtype=torch.float16, device=DEV) for _ in range(2))
    rope = rope_table(40, 64)
    kv = ls.ls_paged_kv_create(kp, vp, 4, rope=rope)
    qkv = torch.randn(1, 8, 64, device=DEV).half()
    q, k, v = qkv.split([4, 2, 2], 1)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    want = torch.empty(1, 4, 64, dtype=torch.float16, device=DEV)
    ls.ls_paged_kv_append(kv, q, k, v, want, i32(0), i32(33), i32(0, 1, 2).view(1, 3))
    ls.ls_paged_kv_append(kv, q, k, v, q, i32(0), i32(33), i32(0, 1, 2).view(1, 3))
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    kv.close()


def test_refusals_with_a_handle():
    b = Batch(lens=[20, 30], prefix=8)
    kv = b.handle()
    L, p = ls.lib(), b.q.data_ptr()
    good = dict(q=p, qs=1024, o=b.out.data_ptr(), os=1024, lse=None, n=2, m=1, sl=b.seq_len.data_ptr(), t=b.table.data_ptr(), tw=b.table.shape[1],
                ts=b.table.shape[1], pp=b.prefix_pages.data_ptr(), pl=8, w=0, sc=0.1, st=None)
    for bad, word in ((dict(n=3), "created for"), (dict(m=2), "created for"), (dict(n=-1), "negative"), (dict(pl=-1), "negative"), (dict(w=-1), "negative"),
                      (dict(q=None), "required"), (dict(sl=None), "required"), (dict(t=None), "required"), (dict(pp=None), "prefix"),
                      (dict(qs=1000), "stride"), (dict(os=1023), "stride"), (dict(ts=1), "table_stride"), (dict(sc=0.0), "scale"),
                      (dict(sc=float("nan")), "scale"), (dict(sc=float("inf")), "scale")):
        assert L.ls_paged_kv_attend(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID, bad
        assert word in ls.last_error(), (bad, ls.last_error())
    assert L.ls_paged_kv_attend(kv.handle, *{**good, "n": 0, "q": None}.values()) == ls.LS_OK
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device=DEV)
    i = torch.zeros(1, dtype=torch.int32, device=DEV)
    good = dict(q=None, qs=0, qo=None, qos=0, k=k.data_ptr(), ks=256, v=k.data_ptr(), vs=256, n=1, seq=i.data_ptr(), pos=i.data_ptr(),
                t=b.table.data_ptr(), ns=2, tw=b.table.shape[1], ts=b.table.shape[1], st=None)
    for bad, word in ((dict(n=-1), "negative"), (dict(k=None), "required"), (dict(v=None), "required"), (dict(seq=None), "required"), (dict(pos=None), "required"),
                      (dict(t=None), "required"), (dict(q=p, qs=1024), "together"), (dict(ks=255), "stride"), (dict(vs=0), "stride"), (dict(ts=0), "table_stride")):
        assert L.ls_paged_kv_append(kv.handle, *{**good, **bad}.values()) == ls.LS_ERR_INVALID, bad
        assert word in ls.last_error(), (bad, ls.last_error())
    assert L.ls_paged_kv_append(kv.handle, *{**good, "n": 0, "k": None}.values()) == ls.LS_OK
    kv.close()
    append_only = ls.ls_paged_kv_create(b.kp, b.vp, b.heads)
    with pytest.raises(ls.LeanStreamError):
        b.attend(append_only)
    append_only.close()
