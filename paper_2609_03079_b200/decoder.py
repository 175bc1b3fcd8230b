"""A whole decoder layer on the library: the attention half (norm, projections, append, attention over the shared prefix and each
sequence's own pages, output projection, gated residual sum) and the activation-sparse FFN half (speculate, staged step).

    python -m paper_2609_03079_b200.decoder          # a small stack, a prompt shared by the batch, a few decode steps
    python -m paper_2609_03079_b200.decoder 4        # the same with its keys and values in 4 bits

The projections are ordinary matrix products and stay with PyTorch; everything else is a call of the C ABI.  The residual is
fp32, as the FFN half keeps it, and holds one row per sequence.
"""
from __future__ import annotations

import sys
from dataclasses import dataclass
from typing import List, Optional, Tuple

import torch

from . import binding as ls
from . import workload as wl


def rope_table(positions: int, dim: int, base: float = 10000.0, device=None) -> torch.Tensor:
    """[positions, dim]: cosines, then sines, of p * base^(-2 i / dim); angles in 64 bits, kept in 32."""
    i = torch.arange(dim // 2, dtype=torch.float64)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-2.0 * i / dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous().to(device)


class PagePool:
    """Hands out the pages of every layer's cache: one table of page numbers serves all layers (each has its own pool)."""

    def __init__(self, n_pages: int, page_size: int, max_seqs: int, max_positions: int, device):
        self.page_size = page_size
        self.free = list(range(n_pages))[::-1]
        self.table = torch.zeros(max_seqs, -(-max_positions // page_size), dtype=torch.int32, device=device)
        self.held: List[List[int]] = [[] for _ in range(max_seqs)]

    def reserve(self, seq: int, positions: int, first: int = 0) -> None:
        """Gives sequence ``seq`` pages for positions [first, positions) that it does not have yet (``first``: where its own start).
        Nothing changes if it cannot have all of them."""
        self.reserve_all([(seq, positions)], first)

    def reserve_all(self, wanted: List[Tuple[int, int]], first: int = 0) -> None:
        """``reserve`` for several (sequence, positions): all of them, or none."""
        start, need = first // self.page_size, []
        for seq, positions in wanted:
            at, end = start + len(self.held[seq]), -(-positions // self.page_size)
            if end > self.table.shape[1]:
                raise ls.LeanStreamError(ls.LS_ERR_CAPACITY, f"{positions} positions, the table holds {self.table.shape[1]} pages of {self.page_size}")
            need.append((seq, at, max(0, end - at)))
        if sum(n for _, _, n in need) > len(self.free):
            raise ls.LeanStreamError(ls.LS_ERR_CAPACITY, "no free page")
        for seq, at, n in need:
            if n:
                new = [self.free.pop() for _ in range(n)]
                self.table[seq, at:at + n] = torch.tensor(new, dtype=torch.int32, device=self.table.device)
                self.held[seq] += new

    def release(self, seq: int) -> None:
        self.free += self.held[seq]
        self.held[seq] = []


@dataclass
class AttentionWeights:
    w_qkv: torch.Tensor  # [d_model, (heads + 2 kv_heads) * head_dim], 16-bit
    w_out: torch.Tensor  # [heads * head_dim, d_model]
    gain_pre: Optional[torch.Tensor] = None   # float [d_model] or None
    gain_post: Optional[torch.Tensor] = None  # given: the attention block's output is normed before the residual sum
    gate: Optional[torch.Tensor] = None       # 16-bit [d_model]
    residual_scale: float = 1.0


class DecoderLayer:
    """One layer: its attention weights, its paged cache and its FFN layer (``ls.Layer``)."""

    def __init__(self, att: AttentionWeights, ffn: ls.Layer, heads: int, kv_heads: int, head_dim: int, n_pages: int, page_size: int, max_seqs: int,
                 rope: Optional[torch.Tensor], k_select: int, n_chunks: int = 8, eps: float = 1e-5, window: int = 0, kv_bits: int = 16, kv_group: int = 64):
        """``kv_bits`` = 4 keeps keys and values in 4 bits, ``kv_group`` components to a scale (``page_size`` a multiple of 16 then)."""
        if kv_bits not in (4, 16):
            raise ValueError("kv_bits: 4 or 16")
        dev, dt = att.w_qkv.device, att.w_qkv.dtype
        self.att, self.ffn = att, ffn
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.eps, self.window, self.k, self.n_chunks = eps, window, k_select, n_chunks
        self.kv_bits = kv_bits
        # zeros, not because the kernels need them (slots nobody sees may hold anything) but so that a dump is readable
        if kv_bits == 4:
            self.pages = torch.zeros(n_pages, kv_heads, ls.ls_paged_kv4_block_bytes(page_size, head_dim, kv_group), dtype=torch.uint8, device=dev)
            self.kv = ls.ls_paged_kv4_create(self.pages, heads, head_dim, page_size, dtype=dt, group=kv_group, max_seqs=max_seqs, max_q_len=1, rope=rope)
        else:
            self.k_pages = torch.zeros(n_pages, page_size, kv_heads, head_dim, dtype=dt, device=dev)
            self.v_pages = torch.zeros_like(self.k_pages)
            self.kv = ls.ls_paged_kv_create(self.k_pages, self.v_pages, heads, max_seqs=max_seqs, max_q_len=1, rope=rope)
        d = ffn.d_model
        self.h = torch.empty(max_seqs, d, dtype=dt, device=dev)
        self.q = torch.empty(max_seqs, heads, head_dim, dtype=dt, device=dev)
        self.o = torch.empty_like(self.q)
        self.sel = ls.Selection(ffn.d_ff, min(max_seqs * k_select, ffn.d_ff), ffn.device)

    def qkv(self, x: torch.Tensor):
        """Pre-norm and projection of residual rows x [n, d]: views q, k, v of one product."""
        n = x.shape[0]
        h = self.h[:n] if n <= self.h.shape[0] else torch.empty(n, x.shape[1], dtype=self.h.dtype, device=x.device)
        ls.ls_block_norm(x, None, None, h, w_pre=self.att.gain_pre, eps=self.eps)
        y = (h @ self.att.w_qkv).view(n, self.heads + 2 * self.kv_heads, self.head_dim)
        return y.split([self.heads, self.kv_heads, self.kv_heads], 1)

    def decode(self, x: torch.Tensor, seq: torch.Tensor, pos: torch.Tensor, seq_len: torch.Tensor, table: torch.Tensor,
               prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0) -> torch.Tensor:
        """One token for each of n sequences: x [n, d] fp32 is replaced by the layer's output."""
        n = x.shape[0]
        q, k, v = self.qkv(x)
        if self.kv_bits == 4:  # (the prefix stands in the table like any other pages)
            ls.ls_paged_kv4_append(self.kv, q, k, v, self.q[:n], seq, pos, table)
            ls.ls_paged_kv4_attend(self.kv, self.q[:n], self.o[:n], seq_len, table, window=self.window)
        else:
            ls.ls_paged_kv_append(self.kv, q, k, v, self.q[:n], seq, pos, table)
            ls.ls_paged_kv_attend(self.kv, self.q[:n], self.o[:n], seq_len, table, prefix_pages, prefix_len, window=self.window)
        y = self.o[:n].view(n, -1) @ self.att.w_out
        a = self.att
        ls.ls_block_norm(x, y, x, None, post_norm=a.gain_post is not None, w_post=a.gain_post, gate=a.gate, scale=a.residual_scale, eps=self.eps)
        ls.ls_predict(self.ffn, x, self.k, self.sel)
        ls.ls_sparse_ffn_step(self.ffn, None, x, x, self.sel, self.n_chunks)
        return x

    def cached(self, seq: torch.Tensor, pos: torch.Tensor, table: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """Keys (turned) and values, 16-bit [tokens, kv_heads, head_dim], that the cache holds at positions ``pos`` of sequences ``seq`` (int32)."""
        if self.kv_bits == 4:
            k, v = (torch.empty(seq.numel(), self.kv_heads, self.head_dim, dtype=self.kv.dtype, device=table.device) for _ in range(2))
            ls.ls_paged_kv4_read(self.kv, k, v, seq, pos, table)
            return k, v
        page = self.k_pages.shape[1]
        at = table[seq.long(), torch.div(pos, page, rounding_mode="floor").long()].long()
        return self.k_pages[at, (pos % page).long()], self.v_pages[at, (pos % page).long()]

    def status(self) -> int:
        return ls.ls_paged_kv4_status(self.kv) if self.kv_bits == 4 else ls.ls_paged_kv_status(self.kv)

    def close(self) -> None:
        self.kv.close()


class Decoder:
    """A stack of layers over one page pool, decoding a batch whose sequences share a prompt."""

    def __init__(self, layers: List[DecoderLayer], pool: PagePool, max_seqs: int):
        self.layers, self.pool = layers, pool
        dev = pool.table.device
        self.max_seqs = max_seqs
        self.lens = [0] * max_seqs
        self.prefix_len = 0
        self.prefix_held: List[int] = []  # pages of the prefix, and the same on the device
        self.prefix_pages: Optional[torch.Tensor] = None
        self.seq = torch.arange(max_seqs, dtype=torch.int32, device=dev)

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """The next token of every sequence: x [max_seqs, d] fp32 in place through all layers.  Nothing has happened if there is no room
        for one of them."""
        self.pool.reserve_all([(b, self.lens[b] + 1) for b in range(self.max_seqs)], self.prefix_len)
        self.lens = [n + 1 for n in self.lens]
        seq_len = torch.tensor(self.lens, dtype=torch.int32).to(x.device)
        for layer in self.layers:
            layer.decode(x, self.seq, seq_len - 1, seq_len, self.pool.table[:self.max_seqs], self.prefix_pages, self.prefix_len)
        return x

    def share_prefix(self, seq: int = 0) -> None:
        """Makes what sequence ``seq`` has decoded so far (a whole number of pages of it, a prefix that it stands on among them) the
        prefix of all sequences; the others must have nothing of their own.  The rest of the sequence is dropped."""
        ps = self.pool.page_size
        n = self.lens[seq] // ps * ps
        if any(self.lens[b] > self.prefix_len for b in range(self.max_seqs) if b != seq):
            raise ls.LeanStreamError(ls.LS_ERR_STATE, "the other sequences must have nothing of their own")
        held = self.pool.held[seq]
        kept = (n - self.prefix_len) // ps
        self.prefix_held += held[:kept]
        self.pool.held[seq] = held[kept:]
        self.pool.release(seq)
        self.prefix_len = n
        self.prefix_pages = torch.tensor(self.prefix_held, dtype=torch.int32, device=self.pool.table.device)
        self.pool.table[:self.max_seqs, :len(self.prefix_held)] = self.prefix_pages
        self.lens = [n] * self.max_seqs

    def cached(self, seq: int) -> List[Tuple[torch.Tensor, torch.Tensor]]:
        """Keys and values of every layer for all positions of a sequence (its prefix among them), in 16 bits: to be looked at, moved to
        another machine or kept."""
        seq = range(self.max_seqs)[seq]
        n = self.lens[seq]
        pos = torch.arange(n, dtype=torch.int32, device=self.pool.table.device)
        return [layer.cached(torch.full_like(pos, seq), pos, self.pool.table) for layer in self.layers]

    def close(self) -> None:
        for layer in self.layers:
            layer.close()


def make_attention(spec: wl.StackSpec, layer: int, heads: int, kv_heads: int, head_dim: int, device, post: bool = False) -> AttentionWeights:
    """Seeded synthetic attention weights of a stack's shape."""
    gen = torch.Generator().manual_seed(1000 * spec.seed + layer)
    dt = torch.bfloat16 if spec.wdtype == "bf16" else torch.float16
    d = spec.d_model
    rnd = lambda *s: torch.randn(*s, generator=gen)
    w_qkv = (rnd(d, (heads + 2 * kv_heads) * head_dim) * d ** -0.5).to(dt).to(device)
    w_out = (rnd(heads * head_dim, d) * (heads * head_dim) ** -0.5).to(dt).to(device)
    gain = (1 + 0.1 * rnd(d)).to(device)
    if not post:
        return AttentionWeights(w_qkv, w_out, gain_pre=gain)
    return AttentionWeights(w_qkv, w_out, gain, (1 + 0.1 * rnd(d)).to(device), (0.5 + 0.1 * rnd(d)).to(dt).to(device), 0.5)


def build(spec: wl.StackSpec, n_layers: int, heads: int, kv_heads: int, head_dim: int, max_seqs: int, max_positions: int, page_size: int = 16, device: int = 0,
          post: bool = False, kv_bits: int = 16, kv_group: int = 64) -> Decoder:
    dev = torch.device("cuda", device)
    n_pages = (max_seqs + 1) * -(-max_positions // page_size)
    pool = PagePool(n_pages, page_size, max_seqs, max_positions, dev)
    rope = rope_table(max_positions, head_dim, device=dev)
    layers = []
    for i, arrays in enumerate(wl.make_stack(spec, n_layers)):
        ffn = ls.ls_layer_create(arrays, device, max_batch=max_seqs)
        layers.append(DecoderLayer(make_attention(spec, i, heads, kv_heads, head_dim, dev, post), ffn, heads, kv_heads, head_dim, n_pages, page_size, max_seqs, rope,
                                   spec.k, kv_bits=kv_bits, kv_group=kv_group))
    return Decoder(layers, pool, max_seqs)


def main(kv_bits: int = 16) -> None:
    torch.manual_seed(0)
    spec, batch, prompt, steps = wl.SPECS["tiny4"], 4, 40, 8
    dec = build(spec, spec.n_layers, heads=4, kv_heads=2, head_dim=64, max_seqs=batch, max_positions=256, post=True, kv_bits=kv_bits)
    dev = torch.device("cuda", 0)
    tokens = torch.from_numpy(wl.make_tokens(spec, prompt)).to(dev)
    one = Decoder(dec.layers, dec.pool, 1)  # sequence 0 alone, through the same layers and pool
    for t in range(prompt):
        one.step(tokens[t:t + 1].clone())
    dec.lens[0] = one.lens[0]
    dec.share_prefix(0)
    print(f"prompt of {prompt} tokens; {dec.prefix_len} of them shared by {batch} sequences")
    x = torch.randn(batch, spec.d_model, device=dev)
    for t in range(steps):
        x = dec.step(x)
        x = x / x.square().mean(1, keepdim=True).sqrt()
        print(f"step {t}: lengths {dec.lens}, residual rms {x.square().mean().sqrt().item():.3f}, first values {[round(v, 4) for v in x[0, :3].tolist()]}")
    k, v = dec.cached(0)[0]
    print(f"layer 0 keeps {k.shape[0]} positions of sequence 0 in {kv_bits} bits; rms of its keys {k.float().square().mean().sqrt().item():.3f}, of its values {v.float().square().mean().sqrt().item():.3f}")
    bad = [layer.status() for layer in dec.layers]
    assert not any(bad), bad
    dec.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 16)
