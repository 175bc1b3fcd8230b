"""Scales and codes of ls_paged_kv4_append where a rounding is close, against the definition bit by bit: quotients by 15 of every size, components
halfway between two codes, distances from the zero that fp32 does not hold."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from paper_2609_03079_b200 import binding as ls
from test_gpu_kv4_attend import DEV

pytestmark = pytest.mark.gpu


def stored(values, dtype):
    """Appends [n, 32] values as one token each (a head of 64: the 32 twice) and returns (codes, scale bits, zero bits) of the values' first group."""
    n = values.shape[0]
    x = torch.cat([values, values], 1).view(n, 1, 64).to(DEV)
    pages = torch.zeros(-(-n // 16), 1, ls.ls_paged_kv4_block_bytes(16, 64, 32), dtype=torch.uint8, device=DEV)
    kv = ls.ls_paged_kv4_create(pages, 1, 64, 16, dtype=orc.DT[dtype], group=32)
    table = torch.arange(pages.shape[0], dtype=torch.int32, device=DEV)[None]
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    ls.ls_paged_kv4_append(kv, None, x, x, None, torch.zeros_like(pos), pos, table)
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()
    raw = pages.cpu().numpy()
    meta = np.ascontiguousarray(raw[:, 0, 16 * 64 + 16 * 8:]).view(np.uint16).reshape(-1, 2, 2)[:n]  # [token, group, (scale, zero)] of values
    keys = np.ascontiguousarray(raw[:, 0, 16 * 64:16 * 64 + 16 * 8]).view(np.uint16).reshape(-1, 2, 2)[:n]
    assert (meta == keys).all() and (meta[:, 0] == meta[:, 1]).all()
    held = orc.held(raw, 16, 64, 32, dtype)
    codes = [h[0].reshape(-1, 64)[:n, :32] for h in held]
    assert (codes[0] == codes[1]).all()
    return codes[1], meta[:, 0, 0], meta[:, 0, 1]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scales_of_every_range(dtype):
    """Zero 0 and each positive finite number of the type as the largest component; then 2^17 pairs of any two finite numbers."""
    dt = orc.DT[dtype]
    every = torch.arange(1, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dt)
    every = every[torch.isfinite(every)]
    lo, hi = torch.zeros_like(every), every
    g = torch.Generator().manual_seed(0)
    any_ = torch.randint(0, 2 ** 16, (2, 2 ** 17), generator=g).to(torch.int32).to(torch.int16).view(dt)
    any_ = any_[:, torch.isfinite(any_).all(0) & torch.isfinite(any_[0].float() - any_[1].float())]
    lo, hi = torch.cat([lo, torch.minimum(any_[0], any_[1])]), torch.cat([hi, torch.maximum(any_[0], any_[1])])
    x = lo[:, None].repeat(1, 32)
    x[:, 5] = hi
    codes, scale, zero = stored(x, dtype)
    want = ((hi.float() - lo.float()) / 15).to(dt)
    assert (scale == want.view(torch.int16).numpy().view(np.uint16)).all()
    assert (torch.from_numpy(zero.view(np.int16)).view(dt) == lo).all()  # (0 and -0 are the same)
    top = np.where(want.double().numpy() > 0, np.minimum(15, np.rint((hi.double() - lo.double()).numpy() / np.where(want.double().numpy() > 0, want.double().numpy(), 1))), 0)
    assert (codes[:, 5] == top).all() and (np.delete(codes, 5, 1) == 0).all()


@pytest.mark.parametrize("dtype,tiny", [("bf16", 1e-9), ("bf16", 1e-30), ("fp16", 2.0 ** -24)])
@pytest.mark.parametrize("scale", [2.0, 0.125, 3.0])
def test_distances_that_32_bits_do_not_hold(dtype, tiny, scale):
    """Components halfway between two codes, but for a zero so small that their difference from it, rounded to fp32, is (nearly always) the half: ties go
    to even codes."""
    if dtype == "fp16":
        scale *= 8
    dt = orc.DT[dtype]
    half = torch.arange(15, dtype=torch.float64) * scale + scale / 2
    x = torch.stack([torch.full((32,), sign * tiny, dtype=torch.float64) for sign in (-1.0, 1.0)])
    x[:, 1:16], x[:, 16] = half, 15 * scale
    assert (x[:, 1:17].to(dt).double() == x[:, 1:17]).all()
    codes, s, _ = stored(x.to(dt), dtype)
    assert (orc.from_bits(s, dtype) == scale).all()
    level = (x.to(dt).float() - x[:, :1].to(dt).float()).double().numpy()[:, 1:16] / scale
    assert (level == np.arange(15) + 0.5).mean() > 0.9 and (codes[:, 1:16] == np.rint(level)).all(), codes[:, :17]
    assert (codes[:, 16] == 15).all() and (codes[:, 17:] == 0).all() and (codes[:, 0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_codes_at_every_half(dtype):
    """Components at (k + 1/2) scale, one step of the type below and one above, for many scales down to the smallest: ties go to even codes."""
    dt = orc.DT[dtype]
    bits = np.concatenate([np.arange(1, 200), np.random.RandomState(0).randint(200, 0x7000 if dtype == "bf16" else 0x6000, 3000)])
    scale = orc.from_bits(bits.astype(np.uint16), dtype)
    rows = []
    for s in scale:
        at = torch.from_numpy((np.arange(10) + 0.5) * s).to(dt)
        near = torch.cat([at, (at.view(torch.int16) - 1).clamp(min=0).view(dt), (at.view(torch.int16) + 1).view(dt)])
        rows.append(torch.cat([torch.zeros(1, dtype=dt), torch.tensor([15 * s], dtype=torch.float64).to(dt), near]))
    x = torch.stack(rows)
    x = torch.where(x.double() <= x[:, 1:2].double(), x, torch.zeros_like(x))
    x = x[torch.isfinite(x.float()).all(1)]
    codes, s, _ = stored(x, dtype)
    want, ws, _ = orc.quantise(x.double().numpy(), 32, dtype)
    assert (orc.from_bits(s, dtype) == ws[:, 0]).all()
    assert (codes == want).all()
