"""Plain 64-bit NumPy forms of the 4-bit paged cache, written from the definitions in the public header: quantisation of tokens, where a
block keeps them, and attention over what it holds (with the parts that error bounds are made of).  Test infrastructure only."""
from __future__ import annotations

import numpy as np
import torch

from oracle import decoder_oracle as dorc

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def to16(x, dtype):
    """x (float64) rounded to 32 bits and then to the type, as float64."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).float().to(DT[dtype]).double().numpy()


def bits16(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(DT[dtype]).view(torch.int16).numpy().view(np.uint16)


def from_bits(b, dtype):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).view(DT[dtype]).double().numpy()


def quantise(x, group, dtype):
    """(codes [..., D], scale, zero [..., D / group]) of components that the type holds; a range that is not finite: NaN."""
    y = x.reshape(*x.shape[:-1], -1, group)
    with np.errstate(all="ignore"):
        low, high = y.min(-1), y.max(-1)
        fine = np.isfinite(y).all(-1) & np.isfinite((high - low).astype(np.float32))
        scale = np.where(fine, to16(np.where(fine, high - low, 0) / 15, dtype), np.nan)
        zero = np.where(fine, low, np.nan)
        level = np.where((scale > 0)[..., None], (y - zero[..., None]) / np.where(scale > 0, scale, 1)[..., None], 0.0)
        codes = np.minimum(15, np.rint(np.nan_to_num(level))).astype(np.int64)
    return codes.reshape(x.shape), scale, zero


def block_bytes(page, D, group):
    return page * (D + 8 * (D // group))


def place(D, value, row):
    """For each component of a code row: its byte and its shift."""
    byte, shift = np.zeros(D, np.int64), np.zeros(D, np.int64)
    for c in range(D):
        if value:
            m, j, i = D // 64, c // 64, c % 32 // 4
            word = i * m + j
            s = {64: 0, 128: row // 2 % 2, 256: row % 4}[D]
            word = (word // 8 ^ s) * 8 + word % 8
            nibble = c % 64 // 32 * 4 + c % 4
        else:
            n, w = min(4, D // 32), c // 8
            part = w // 16 ^ row % 2 if D == 256 else 0
            word = part * 4 * n + w % 4 * n + w // 4 % n
            nibble = c % 8
        byte[c], shift[c] = word * 4 + nibble // 2, nibble % 2 * 4
    return byte, shift


def put(block, slot, k, v, group, dtype):
    """Stores one token's key and value (components as the type holds them) of one head in a block (uint8 array), in place."""
    D = k.shape[0]
    ng, tile, row = D // group, slot // 16 * 16 * (D + 8 * (D // group)), slot % 16
    for value, x in ((0, k), (1, v)):
        codes, scale, zero = quantise(x, group, dtype)
        byte, shift = place(D, value, row)
        out = np.zeros(D // 2, np.uint8)
        np.bitwise_or.at(out, byte, (codes << shift).astype(np.uint8))
        at = tile + (16 * value + row) * (D // 2)
        block[at:at + D // 2] = out
        meta = np.stack([bits16(scale, dtype), bits16(zero, dtype)], -1).reshape(-1).view(np.uint8)
        at = tile + 16 * D + (16 * value + row) * 4 * ng
        block[at:at + 4 * ng] = meta


def held(pages, page, D, group, dtype):
    """(codes, scale, zero) for keys and for values: [n_pages, page, heads, D] of pages [n_pages, heads, block]; scale and zero repeated."""
    n, H, _ = pages.shape
    ng = D // group
    t = pages.reshape(n, H, page // 16, -1)
    out = []
    for value in (0, 1):
        rows = t[..., 16 * value * (D // 2):16 * (value + 1) * (D // 2)].reshape(n, H, page // 16, 16, D // 2)
        codes = np.zeros((n, H, page // 16, 16, D), np.int64)
        for r in range(16):
            byte, shift = place(D, value, r)
            codes[..., r, :] = rows[..., r, byte] >> shift & 15
        at = 16 * D + 64 * ng * value
        meta = np.ascontiguousarray(t[..., at:at + 64 * ng]).view(np.uint16).reshape(n, H, page // 16, 16, ng, 2)
        x = [codes] + [np.repeat(from_bits(meta[..., i], dtype).reshape(meta.shape[:-1]), group, -1) for i in (0, 1)]
        out.append([a.reshape(n, H, page, D).transpose(0, 2, 1, 3) for a in x])
    return out


def values(parts):
    codes, scale, zero = parts
    with np.errstate(invalid="ignore"):
        return codes * scale + zero


def attend(q, pages, page, group, dtype, seq_len, table, window, scale):
    """q [seqs, q_len, heads, D] -> (out, lse, bounds): bounds are absout = sum w |v|, absqk = max sum |q| (s u + |z|), rounded = sum w s |u - 8|,
    parts = sum w (16 s + |z|), top = max w s."""
    B, m, H, D = q.shape
    K, V = held(pages, page, D, group, dtype)
    kv, vv = values(K), values(V)
    G = H // kv.shape[2]
    out, lse = np.zeros(q.shape), np.full((B, m, H), -np.inf)
    bound = {n: np.zeros(q.shape) for n in ("absout", "rounded", "parts", "top")}
    absqk = np.zeros((B, m, H))
    for b in range(B):
        n = int(seq_len[b])
        for i in range(m):
            hi = n - m + i + 1
            if hi <= 0:
                continue
            pos = np.arange(max(0, hi - window) if window else 0, hi)
            ids = np.asarray(table[b])[pos // page], pos % page
            for j in range(kv.shape[2]):
                h = slice(j * G, (j + 1) * G)
                s = q[b, i, h] @ kv[ids][:, j].T * scale
                top = s.max(1, keepdims=True)
                e = np.exp(s - top)
                w = e / e.sum(1, keepdims=True)
                u, sc, z = (x[ids][:, j] for x in V)
                out[b, i, h] = w @ vv[ids][:, j]
                lse[b, i, h] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
                bound["absout"][b, i, h] = w @ np.abs(vv[ids][:, j])
                bound["rounded"][b, i, h] = w @ (sc * np.abs(u - 8))
                bound["parts"][b, i, h] = w @ (16 * sc + np.abs(z))
                bound["top"][b, i, h] = (w[:, :, None] * sc[None]).max(1)
                ku, ks, kz = (x[ids][:, j] for x in K)
                absqk[b, i, h] = (np.abs(q[b, i, h]) @ (ks * ku + np.abs(kz)).T).max(1)
    return out, lse, bound, absqk


rotate = dorc.rotate
