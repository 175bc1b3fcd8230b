"""ls_paged_kv4_append and ls_paged_kv4_read against the 64-bit forms: what the pages hold is compared bit by bit, what is read back and
the turned queries to the rounding of their type (half a step: 2^-9 of a bf16's power of two, 2^-8 of its value at most; fp16 2^-11)."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200.decoder import rope_table

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = orc.DT
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def tokens(gen, T, H, D, dtype, layout, std=1.0):
    """[T, H, D] of random values: dense, as a slice of a wider projection, or at an odd element offset with an odd stride."""
    x = (torch.randn(T, H, D, generator=gen, device=DEV) * std).to(DT[dtype])
    if layout == "slice":
        wide = torch.zeros(T, H + 3, D, dtype=x.dtype, device=DEV)
        wide[:, 1:H + 1] = x
        return wide[:, 1:H + 1]
    if layout == "odd":
        flat = torch.zeros(T * (H * D + 1) + 1, dtype=x.dtype, device=DEV)
        y = flat[1:].as_strided((T, H, D), (H * D + 1, D, 1), 1)
        y.copy_(x)
        return y
    return x


class Cache:
    """Pages of random bytes and a table of shuffled pages for `seqs` sequences; strided: blocks of a larger pool, heads apart."""

    def __init__(self, dtype, H, HK, D, group, page, seqs, width, seed=0, strided=False, rope_dim=0, interleaved=False, positions=None, **kw):
        self.dtype, self.H, self.HK, self.D, self.group, self.page = dtype, H, HK, D, group, page
        gen = torch.Generator(device=DEV).manual_seed(seed)
        block = ls.ls_paged_kv4_block_bytes(page, D, group)
        assert block == orc.block_bytes(page, D, group)
        n = seqs * width + 2
        raw = torch.randint(0, 256, (n, HK + 1, block + 32), generator=gen, device=DEV, dtype=torch.uint8)
        self.pages = raw[:, 1:, 16:16 + block] if strided else raw[:, :HK, :block].contiguous()
        ids = torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:seqs * width]
        self.table_np = ids.view(seqs, width).numpy().astype(np.int32)
        self.table = i32(self.table_np)
        self.rope = rope_table(positions or page * width, rope_dim, device=DEV) if rope_dim else None
        self.interleaved = interleaved
        self.kv = ls.ls_paged_kv4_create(self.pages, H, D, page, dtype=DT[dtype], group=group, rope=self.rope, rope_interleaved=interleaved, **kw)
        self.before = self.pages.cpu().numpy().copy()

    def expect(self, k, v, seq, pos):
        """Pages after these tokens, computed on the host."""
        want = self.before.copy()
        rope = None if self.rope is None else f64(self.rope)
        kr = orc.to16(orc.rotate(f64(k), pos, rope, self.interleaved), self.dtype)
        vv = f64(v)
        for t, (b, p) in enumerate(zip(seq, pos)):
            if b >= 0 and p >= 0:
                for h in range(self.HK):
                    orc.put(want[self.table_np[b, p // self.page], h], p % self.page, kr[t, h], vv[t, h], self.group, self.dtype)
        return want


def check_append(dtype="bf16", H=8, HK=2, D=128, group=64, page=16, layout="dense", strided=False, rope_dim=0, interleaved=False, T=21, with_q=True, inplace=False,
                 seed=1, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    seqs, width = 3, -(-T // page) + 1
    c = Cache(dtype, H, HK, D, group, page, seqs, width, seed, strided, rope_dim, interleaved)
    rng = np.random.RandomState(seed)
    slots = rng.permutation(seqs * width * page)[:T]
    seq, pos = (slots // (width * page)).tolist(), (slots % (width * page)).tolist()
    if T > 4:
        seq[1], pos[2] = -1, -5  # padding
    k, v = (tokens(gen, T, HK, D, dtype, layout, std) for _ in range(2))
    q = tokens(gen, T, H, D, dtype, layout) if with_q else None
    q_np = f64(q) if with_q else None
    q_out = (q if inplace else tokens(gen, T, H, D, dtype, layout)) if with_q else None
    want = c.expect(k, v, seq, pos)
    ls.ls_paged_kv4_append(c.kv, q, k, v, q_out, i32(seq), i32(pos), c.table)
    assert ls.ls_paged_kv4_status(c.kv) == 0
    got = c.pages.cpu().numpy()
    assert (got == want).all(), f"{(got != want).sum()} bytes differ, first at {np.argwhere(got != want)[0]}"
    if with_q:
        rope = None if c.rope is None else f64(c.rope)
        ref = orc.rotate(q_np, pos, rope, interleaved)
        # two products and a difference in fp32 (2^-24 each of sum |x c|), then the type
        tol = U[dtype] * np.abs(ref) + 2.0 ** -22 * np.abs(q_np).max() + 2.0 ** -25
        assert (np.abs(f64(q_out) - ref) <= tol).all()
    # read back: all of it, and rows of padding left alone
    ko, vo = (torch.full((T, HK, D), 7.0, dtype=DT[dtype], device=DEV) for _ in range(2))
    ls.ls_paged_kv4_read(c.kv, ko, vo, i32(seq), i32(pos), c.table)
    assert ls.ls_paged_kv4_status(c.kv) == 0
    K, V = (orc.values(x) for x in orc.held(want, page, D, group, dtype))
    for t, (b, p) in enumerate(zip(seq, pos)):
        for out, ref in ((ko, K), (vo, V)):
            if b < 0 or p < 0:
                assert (out[t] == 7.0).all()
            else:
                r = ref[c.table_np[b, p // page], p % page]
                assert (np.abs(f64(out[t]) - r) <= U[dtype] * np.abs(r) * (1 + 2.0 ** -10) + 2.0 ** -24).all()
    c.kv.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
def test_shapes(dtype, D, group):
    check_append(dtype, D=D, group=group, rope_dim=D, page=32, seed=D + group)
    check_append(dtype, H=3, HK=3, D=D, group=group, rope_dim=D // 2, interleaved=True, page=48, seed=D + group + 1, std=30.0)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 33, 100])
@pytest.mark.parametrize("H,HK", [(1, 1), (5, 5), (12, 4), (40, 8)])
def test_tokens_and_heads(T, H, HK):
    check_append(H=H, HK=HK, T=T, rope_dim=128, seed=T)
    check_append("fp16", H=H, HK=HK, D=64, group=32, T=T, rope_dim=32, seed=T + 1, layout="slice")


@pytest.mark.parametrize("rope_dim", [0, 2, 6, 10, 16, 20, 24, 40, 64, 100, 126, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_rotations(rope_dim, interleaved, layout):
    check_append(rope_dim=rope_dim, interleaved=interleaved, layout=layout, seed=rope_dim, T=9)
    check_append("fp16", rope_dim=rope_dim, interleaved=interleaved, layout=layout, seed=rope_dim, T=5, inplace=True)


@pytest.mark.parametrize("layout", ["dense", "slice", "odd"])
@pytest.mark.parametrize("strided", [False, True])
def test_layouts(layout, strided):
    for kw in (dict(D=64, group=64), dict(D=128, group=32), dict(D=256, group=128)):
        check_append(layout=layout, strided=strided, rope_dim=64, seed=5, **kw)
        check_append("fp16", layout=layout, strided=strided, with_q=False, seed=6, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,group", [(64, 32), (128, 64), (256, 128)])
def test_what_values_can_be(dtype, D, group):
    """Equal components, ties between codes, one large component among tiny ones, the type's smallest and largest values, infinities and NaN:
    the bytes are the definition's, and a group that is not finite reads back as NaN without touching its neighbours."""
    T, HK, big = 12, 2, float(torch.finfo(DT[dtype]).max)
    c = Cache(dtype, 2, HK, D, group, 16, 1, 1)
    x = torch.randn(2, T, HK, D, generator=torch.Generator().manual_seed(3))
    x[:, 0] = 0.0
    x[:, 1] = -3.25
    x[:, 2] = torch.arange(D) % 31 * 0.5                           # range 15, scale 1: every other component is a tie
    x[:, 3] = torch.arange(D) % 31 * 0.25 - 100.0
    x[:, 4, :, ::32] = 1e4
    x[:, 5] *= torch.finfo(DT[dtype]).smallest_normal * 0.01
    x[:, 6, 0] = torch.where(torch.arange(D) % 2 == 0, big, big / 2)
    x[:, 7, 1, 5] = float("nan")
    x[:, 8, 0, D - 1] = float("inf")
    x[:, 9, 1, 0] = -float("inf")
    x[:, 10, 0, 3], x[:, 10, 0, 4] = big, -big                      # a range that bf16's 32 bits cannot hold, and fp16's can
    x = x.to(DT[dtype]).to(DEV)
    want = c.expect(x[0], x[1], [0] * T, list(range(T)))
    ls.ls_paged_kv4_append(c.kv, None, x[0], x[1], None, i32([0] * T), i32(range(T)), c.table)
    ko, vo = (torch.empty(T, HK, D, dtype=DT[dtype], device=DEV) for _ in range(2))
    ls.ls_paged_kv4_read(c.kv, ko, vo, i32([0] * T), i32(range(T)), c.table)
    got = c.pages.cpu().numpy()
    tiles = [(a, b) for a, b in zip(orc.held(got, 16, D, group, dtype), orc.held(want, 16, D, group, dtype))]
    for (gu, gs, gz), (wu, ws, wz) in tiles:
        assert (gu == wu).all() and np.array_equal(gs, ws, equal_nan=True) and np.array_equal(gz, wz, equal_nan=True)
    for out, parts in zip((ko, vo), orc.held(want, 16, D, group, dtype)):
        ref = orc.values(parts)[c.table_np[0, 0], :T]
        g = f64(out)
        assert (np.isnan(g) == np.isnan(ref)).all()
        fine = np.isfinite(ref) & (np.abs(ref) < big)
        assert (np.abs(g - ref)[fine] <= (U[dtype] * np.abs(ref) * (1 + 2.0 ** -10) + 2.0 ** -24)[fine]).all()
    assert np.isnan(f64(ko)[7, 1, :group]).all() and np.isfinite(f64(ko)[7, 0]).all()
    c.kv.close()


def test_out_of_range_is_skipped_and_reported():
    """Positions beyond the table or the rotation table, sequences beyond the batch, pages outside the pool: nothing is stored or read."""
    c = Cache("bf16", 4, 2, 128, 64, 16, 2, 2, rope_dim=128, positions=20)
    k, v = (torch.randn(1, 2, 128, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(1, 4, 128, device=DEV).bfloat16()
    bad_table = c.table.clone()
    bad_table[1, 0], bad_table[1, 1] = -1, c.pages.shape[0]
    out = torch.full((1, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    for b, p, table, reads in ((0, 20, c.table, True), (0, 32, c.table, False), (2, 0, c.table, False), (1, 3, bad_table, False), (1, 16, bad_table, False), (0, 2 ** 31 - 1, c.table, False)):
        qo = torch.zeros_like(q)
        ls.ls_paged_kv4_append(c.kv, q, k, v, qo, i32([b]), i32([p]), table)
        assert ls.ls_paged_kv4_status(c.kv) == -1 and ls.ls_paged_kv4_status(c.kv) == 0
        assert (c.pages.cpu().numpy() == c.before).all()
        if p >= 20:
            assert torch.equal(q, qo)  # beyond the rotation table: as it is
        if not reads:
            ls.ls_paged_kv4_read(c.kv, out, out, i32([b]), i32([p]), table)
            assert ls.ls_paged_kv4_status(c.kv) == -1 and (out == 7.0).all()
    c.kv.close()


def test_read_strides_and_single_outputs():
    c = Cache("fp16", 6, 3, 128, 32, 32, 2, 2, seed=4)
    k, v = (torch.randn(40, 3, 128, device=DEV).half() for _ in range(2))
    seq, pos = i32([t % 2 for t in range(40)]), i32([t // 2 * 3 % 64 for t in range(40)])
    ls.ls_paged_kv4_append(c.kv, None, k, v, None, seq, pos, c.table)
    ref_k, ref_v = (torch.empty(40, 3, 128, dtype=torch.float16, device=DEV) for _ in range(2))
    ls.ls_paged_kv4_read(c.kv, ref_k, ref_v, seq, pos, c.table)
    assert torch.isfinite(ref_k).all() and (ref_k - k).abs().max() < 0.5 and (ref_v - v).abs().max() < 0.5
    gen = torch.Generator(device=DEV).manual_seed(0)
    for layout in ("slice", "odd"):
        a, b = (tokens(gen, 40, 3, 128, "fp16", layout) for _ in range(2))
        ls.ls_paged_kv4_read(c.kv, a, None, seq, pos, c.table)
        ls.ls_paged_kv4_read(c.kv, None, b, seq, pos, c.table)
        assert torch.equal(a, ref_k) and torch.equal(b, ref_v)
    assert ls.ls_paged_kv4_status(c.kv) == 0
    c.kv.close()


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GB: tokens in its last pages."""
    block, HK = ls.ls_paged_kv4_block_bytes(64, 128, 64), 8
    n = (5 << 30) // (block * HK)
    pages = torch.empty(n, HK, block, dtype=torch.uint8, device=DEV)
    kv = ls.ls_paged_kv4_create(pages, 8, 128, 64, max_seqs=1, max_q_len=1)
    k, v = (torch.randn(64, HK, 128, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(1, 8, 128, device=DEV).bfloat16()
    res = []
    for page in (n - 1, 3):
        table, z, pos = i32([[page]]), i32([0] * 64), i32(range(64))
        ls.ls_paged_kv4_append(kv, None, k, v, None, z, pos, table)
        ko, vo, out = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
        ls.ls_paged_kv4_read(kv, ko, vo, z, pos, table)
        ls.ls_paged_kv4_attend(kv, q, out, i32([64]), table)
        res.append((ko, vo, out))
    assert ls.ls_paged_kv4_status(kv) == 0
    assert all(torch.equal(a, b) for a, b in zip(*res)) and (res[0][0].float() - k.float()).abs().max() < 0.5
    kv.close()
