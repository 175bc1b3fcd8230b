"""A whole decoder layer (attention half and sparse FFN half) and a stack of them against the 64-bit oracles."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as dorc
from oracle import leanstream_oracle as orc
from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200 import decoder as dec
from paper_2609_03079_b200 import workload as wl

pytestmark = pytest.mark.gpu


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class OracleDecoder:
    """The same layers in 64 bits; keys and values per sequence, rounded to 16 bits where the library stores them."""

    def __init__(self, d, arrays):
        self.d = d
        self.ffn = [orc.OracleLayer.from_arrays(a) for a in arrays]
        self.cache = [[([], []) for _ in range(d.max_seqs)] for _ in d.layers]

    def attention(self, i, x, pos):
        L = self.d.layers[i]
        a, dt = L.att, L.att.w_qkv.dtype
        r16 = lambda v: torch.from_numpy(v).to(dt).double().numpy()
        _, h, _ = dorc.block_norm(x, None, False, None, None, 1.0, True, f64(a.gain_pre), L.eps)
        y = r16(r16(h) @ f64(a.w_qkv)).reshape(len(x), L.heads + 2 * L.kv_heads, L.head_dim)
        q, k, v = np.split(y, [L.heads, L.heads + L.kv_heads], 1)
        rope = f64(L.kv.rope)
        q, k = r16(dorc.rotate(q, pos, rope, False)), r16(dorc.rotate(k, pos, rope, False))
        out = np.zeros((len(x), L.heads * L.head_dim))
        G = L.heads // L.kv_heads
        for b in range(len(x)):
            K, V = self.cache[i][b]
            K.append(k[b]); V.append(v[b])
            for hd in range(L.heads):
                s = np.stack(K)[:, hd // G] @ q[b, hd] * L.head_dim ** -0.5
                w = np.exp(s - s.max())
                out[b, hd * L.head_dim:(hd + 1) * L.head_dim] = (w / w.sum()) @ np.stack(V)[:, hd // G]
        y = r16(r16(out) @ f64(a.w_out))
        x2, _, _ = dorc.block_norm(x, y, a.gain_post is not None, f64(a.gain_post), f64(a.gate), a.residual_scale, False, None, L.eps)
        return x2


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 2, 64), (2, 2, 128)])
def test_attention_half_of_each_layer(post, heads, kv_heads, head_dim):
    """Every layer's attention half from the same input as the oracle, over a prompt shared by the batch and the steps behind it.
    Tolerance: the block's output has passed seven roundings to 16 bits (h, qkv, rotation, weights, attention, projection, and the
    keys' and values' own), each at most 2^-8 of its operand; relative to the block's increment, 8 x 2^-8 in the 2-norm."""
    spec, B, prompt = wl.SPECS["tiny4"], 3, 37
    d = dec.build(spec, 2, heads, kv_heads, head_dim, max_seqs=B, max_positions=128, post=post)
    dev = torch.device("cuda", 0)
    O = OracleDecoder(d, wl.make_stack(spec, 2))
    toks = wl.make_tokens(spec, prompt + 12)
    L0 = d.layers[0]
    # the prompt: appended as one chunk of sequence 0 from the embeddings (the first layer's keys depend on nothing else)
    x = torch.from_numpy(toks[:32]).to(dev)
    d.pool.reserve(0, 32)
    q, k, v = L0.qkv(x)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=dev)
    ls.ls_paged_kv_append(L0.kv, None, k, v, None, i32([0] * 32), i32(list(range(32))), d.pool.table)
    for t in range(32):
        O.cache[0][0][0].append(None), O.cache[0][0][1].append(None)
    a, dt = L0.att, L0.att.w_qkv.dtype
    r16 = lambda z: torch.from_numpy(z).to(dt).double().numpy()
    _, h, _ = dorc.block_norm(f64(x), None, False, None, None, 1.0, True, f64(a.gain_pre), L0.eps)
    y = r16(r16(h) @ f64(a.w_qkv)).reshape(32, heads + 2 * kv_heads, head_dim)
    ko = r16(dorc.rotate(y[:, heads:heads + kv_heads], list(range(32)), f64(L0.kv.rope), False))
    for b in range(B):
        O.cache[0][b] = (list(ko), list(y[:, heads + kv_heads:]))
    d.lens[0] = 32
    d.share_prefix(0)
    assert d.prefix_len == 32
    for step in range(4):
        x_np = toks[32 + step * B: 32 + (step + 1) * B]
        x = torch.from_numpy(x_np).to(dev)
        for b in range(B):
            d.pool.reserve(b, d.lens[b] + 1, d.prefix_len)
            d.lens[b] += 1
        pos = [n - 1 for n in d.lens]
        ref = O.attention(0, x_np.astype(np.float64), pos)
        q, k, v = L0.qkv(x)
        ls.ls_paged_kv_append(L0.kv, q, k, v, L0.q[:B], d.seq, i32(pos), d.pool.table)
        ls.ls_paged_kv_attend(L0.kv, L0.q[:B], L0.o[:B], i32(d.lens), d.pool.table, d.prefix_pages, d.prefix_len)
        y = L0.o[:B].view(B, -1) @ a.w_out
        ls.ls_block_norm(x, y, x, None, post_norm=a.gain_post is not None, w_post=a.gain_post, gate=a.gate, scale=a.residual_scale, eps=L0.eps)
        torch.cuda.synchronize()
        inc = np.linalg.norm(ref - x_np)
        assert np.linalg.norm(f64(x) - ref) <= 8 * 2.0 ** -8 * inc, (step, np.linalg.norm(f64(x) - ref) / inc)
    assert ls.ls_paged_kv_status(L0.kv) == 0
    d.close()


def test_a_step_of_the_stack_is_its_parts():
    """Decoder.step equals the calls made one by one, and the FFN half equals the oracle's from the residual that it was given."""
    spec, B = wl.SPECS["tiny4"], 2
    arrays = wl.make_stack(spec, 2)
    d = dec.build(spec, 2, 4, 2, 64, max_seqs=B, max_positions=64, post=True)
    dev = torch.device("cuda", 0)
    for t in range(3):
        x0 = torch.from_numpy(wl.make_tokens(spec, 8)[2 * t:2 * t + 2]).to(dev)
        x = x0.clone()
        d.step(x)
        torch.cuda.synchronize()
        assert torch.isfinite(x).all() and not torch.equal(x, x0)
    # once more by hand from the same state
    x0 = torch.from_numpy(wl.make_tokens(spec, 8)[6:8]).to(dev)
    for b in range(B):
        d.pool.reserve(b, d.lens[b] + 1)
    lens = torch.tensor([n + 1 for n in d.lens], dtype=torch.int32, device=dev)
    want = x0.clone()
    for i, L in enumerate(d.layers):
        q, k, v = L.qkv(want)
        ls.ls_paged_kv_append(L.kv, q, k, v, L.q[:B], d.seq, lens - 1, d.pool.table)
        ls.ls_paged_kv_attend(L.kv, L.q[:B], L.o[:B], lens, d.pool.table)
        a = L.att
        ls.ls_block_norm(want, L.o[:B].view(B, -1) @ a.w_out, want, None, post_norm=True, w_post=a.gain_post, gate=a.gate, scale=a.residual_scale, eps=L.eps)
        before = f64(want)
        ls.ls_predict(L.ffn, want, L.k, L.sel)
        order = L.sel.order()
        ls.ls_sparse_ffn_step(L.ffn, None, want, want, L.sel, L.n_chunks)
        torch.cuda.synchronize()
        OL = orc.OracleLayer.from_arrays(arrays[i])
        for b in range(B):
            ref = before[b] + orc.sparse_ffn_step(OL, None, before[b].astype(np.float32), order, L.n_chunks, 0)["y"][0]
            inc = np.linalg.norm(ref - before[b])
            assert np.linalg.norm(f64(want)[b] - ref) <= 1e-3 * max(inc, 1e-6)
    x = x0.clone()
    d.step(x)
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    d.close()


def test_the_example_runs():
    dec.main()
