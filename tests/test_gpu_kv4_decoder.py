"""The decoder with its keys and values in 4 bits: append, attention and read-back as a stack runs them, one after another."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as dorc
from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200 import decoder as dec
from paper_2609_03079_b200 import workload as wl

pytestmark = pytest.mark.gpu


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def stack(bits, B=3, heads=4, kv_heads=2, head_dim=64, group=64, page=16, post=True):
    return dec.build(wl.SPECS["tiny4"], 2, heads, kv_heads, head_dim, max_seqs=B, max_positions=128, page_size=page, post=post, kv_bits=bits, kv_group=group)


@pytest.mark.parametrize("head_dim,group", [(64, 32), (64, 64), (128, 128)])
def test_attention_half_of_the_first_layer(head_dim, group):
    """Against the 64-bit form over what the pages hold.  Tolerance: the block's output has passed six roundings to 16 bits (h, qkv, rotation,
    weights, attention, projection), each at most 2^-8 of its operand; relative to the block's increment, 8 x 2^-8 in the 2-norm."""
    d = stack(4, head_dim=head_dim, group=group, kv_heads=2, heads=4)
    L, B = d.layers[0], 3
    a, dt = L.att, L.att.w_qkv.dtype
    dev = torch.device("cuda", 0)
    toks = wl.make_tokens(wl.SPECS["tiny4"], 60)
    r16 = lambda v: torch.from_numpy(v).to(dt).double().numpy()
    for step in range(18):
        x_np = toks[3 * step:3 * step + 3]
        x = torch.from_numpy(x_np).to(dev)
        for b in range(B):
            d.pool.reserve(b, step + 1)
        lens = torch.full((B,), step + 1, dtype=torch.int32, device=dev)
        q, k, v = L.qkv(x)
        ls.ls_paged_kv4_append(L.kv, q, k, v, L.q[:B], d.seq, lens - 1, d.pool.table)
        ls.ls_paged_kv4_attend(L.kv, L.q[:B], L.o[:B], lens, d.pool.table)
        ls.ls_block_norm(x, L.o[:B].view(B, -1) @ a.w_out, x, None, post_norm=True, w_post=a.gain_post, gate=a.gate, scale=a.residual_scale, eps=L.eps)
        if step not in (0, 15, 16, 17):
            continue
        torch.cuda.synchronize()
        _, h, _ = dorc.block_norm(x_np.astype(np.float64), None, False, None, None, 1.0, True, f64(a.gain_pre), L.eps)
        y = r16(r16(h) @ f64(a.w_qkv)).reshape(B, L.heads + 2 * L.kv_heads, head_dim)
        q = r16(dorc.rotate(y[:, :L.heads], [step] * B, f64(L.kv.rope), False))
        out, _, _, _ = orc.attend(q[:, None], L.pages.cpu().numpy(), 16, group, "bf16" if dt == torch.bfloat16 else "fp16", [step + 1] * B, d.pool.table.cpu().numpy(), 0, head_dim ** -0.5)
        ref, _, _ = dorc.block_norm(x_np.astype(np.float64), r16(r16(out.reshape(B, -1)) @ f64(a.w_out)), True, f64(a.gain_post), f64(a.gate), a.residual_scale, False, None, L.eps)
        inc = np.linalg.norm(ref - x_np)
        assert np.linalg.norm(f64(x) - ref) <= 8 * 2.0 ** -8 * inc, (step, np.linalg.norm(f64(x) - ref) / inc)
    assert L.status() == 0
    d.close()


def test_what_is_read_back_is_what_a_16_bit_cache_holds_to_half_a_step():
    """The first layer's keys and values depend on the inputs alone: the same steps with both caches.  A step is (max - min) / 15 of a group; its
    scale is off by at most 2^-8, fifteen of them by 15 x 2^-8, and what is read back is rounded once more."""
    full, four = stack(16), stack(4)
    toks = wl.make_tokens(wl.SPECS["tiny4"], 60)
    for step in range(20):
        for d in (full, four):
            d.step(torch.from_numpy(toks[3 * step:3 * step + 3]).to("cuda:0"))
    torch.cuda.synchronize()
    for b in range(3):
        for x, y in zip(full.cached(b)[0], four.cached(b)[0]):
            assert x.shape == y.shape == (20, 2, 64)
            x, y = f64(x), f64(y)
            step = (x.max(-1, keepdims=True) - x.min(-1, keepdims=True)) / 15
            assert (np.abs(x - y) <= step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -8 * np.abs(x)).all()
    assert [L.status() for L in full.layers + four.layers] == [0] * 4
    full.close()
    four.close()


def test_sequences_that_share_a_prefix():
    """A prompt of one sequence becomes the prefix of three: its pages hold what they held, and three sequences that are given the same
    tokens stay the same."""
    toks = wl.make_tokens(wl.SPECS["tiny4"], 60)
    d = stack(4)
    one = dec.Decoder(d.layers, d.pool, 1)
    for t in range(32):
        one.step(torch.from_numpy(toks[t:t + 1]).to("cuda:0"))
    before = [k.clone() for kv in one.cached(0) for k in kv]
    d.lens[0] = one.lens[0]
    d.share_prefix(0)
    assert d.prefix_len == 32
    for t in range(32, 36):
        y = torch.from_numpy(toks[t:t + 1]).to("cuda:0").repeat(3, 1)
        d.step(y)
        torch.cuda.synchronize()
        assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2])
    for s in range(3):
        assert all(torch.equal(k[:32], x) for k, x in zip([k for kv in d.cached(s) for k in kv], before))
    assert [L.status() for L in d.layers] == [0] * 2
    d.close()


def test_a_step_captured_and_replayed():
    """A layer's step in a graph: replayed twice, it stores at the position that the device says, and equals the eager steps."""
    B = 2
    a, b = stack(4, B=B), stack(4, B=B)
    dev = torch.device("cuda", 0)
    toks = torch.from_numpy(wl.make_tokens(wl.SPECS["tiny4"], 20)).to(dev)
    L, x, pos, lens = b.layers[0], torch.empty(B, toks.shape[1], device=dev), torch.zeros(B, dtype=torch.int32, device=dev), torch.ones(B, dtype=torch.int32, device=dev)
    for d in (a, b):
        for s in range(B):
            d.pool.reserve(s, 20)

    def half(L, x, pos, lens, table):
        q, k, v = L.qkv(x)
        ls.ls_paged_kv4_append(L.kv, q, k, v, L.q[:B], b.seq, pos, table)
        ls.ls_paged_kv4_attend(L.kv, L.q[:B], L.o[:B], lens, table)

    x.copy_(toks[:B])
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        half(L, x, pos, lens, b.pool.table)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            half(L, x, pos, lens, b.pool.table)
        for t in range(9):
            x.copy_(toks[2 * t:2 * t + 2])
            pos.fill_(t)
            lens.fill_(t + 1)
            g.replay()
            half(a.layers[0], toks[2 * t:2 * t + 2].contiguous(), pos, lens, a.pool.table)
            st.synchronize()
            assert torch.equal(L.o[:B], a.layers[0].o[:B])
    assert L.status() == 0 and a.layers[0].status() == 0
    a.close()
    b.close()


def test_the_example_runs():
    dec.main(4)
