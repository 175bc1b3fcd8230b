"""ls_block_norm against its plain 64-bit form.  Tolerances come from the formats: a sum of d squares in fp32 is off by at most
d 2^-24 of itself (all terms are positive), its root by half of that; u is the rounding to the output's type."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc
from paper_2609_03079_b200 import binding as ls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 1e-38, "fp16": 2.0 ** -24, "f32": 1e-38}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def case(n=3, d=256, xt="f32", bt="bf16", post=True, gain=True, gate="channel", scale=0.5, pre=True, want=("x", "h"), block=True, pad=0, off=0,
         alias=False, seed=0, zero_row=False):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def rnd(dt, std, rows=n):
        buf = torch.zeros(off + rows * (d + pad) + 8, dtype=DT[dt], device=DEV)
        v = buf[off:off + rows * (d + pad)].view(rows, d + pad)[:, :d]
        v.copy_(torch.randn(rows, d, generator=gen, device=DEV) * std)
        return v

    x, y = rnd(xt, 2.0), rnd(bt, 0.7) if block else None
    if zero_row:
        x[0] = 0
        if block:
            y[0] = 0
    wp = 1 + 0.1 * torch.randn(d, generator=gen, device=DEV) if gain and block else None
    wn = 1 + 0.1 * torch.randn(d, generator=gen, device=DEV) if gain else None
    g = None if gate == "none" or not block else rnd(bt, 0.7, 1)[0] if gate == "channel" else rnd(bt, 0.7)
    ref_x, ref_h, mag = orc.block_norm(f64(x), f64(y), post, f64(wp), f64(g), float(np.float32(scale)), pre, f64(wn), float(np.float32(1e-5)))
    xo = (x if alias else rnd(xt, 0.0)) if "x" in want else None
    h = (y if alias and block else rnd(bt, 0.0)) if "h" in want else None
    ls.ls_block_norm(x, y, xo, h, post_norm=post, w_post=wp, gate=g, scale=scale, pre_norm=pre, w_pre=wn, eps=1e-5)
    torch.cuda.synchronize()
    e = 2.0 ** -24
    ex = mag * (d * e / 2 + 8 * e) + np.abs(ref_x) * e            # x' before its rounding
    if xo is not None:
        assert (np.abs(f64(xo) - ref_x) <= ex + np.abs(ref_x) * U[xt] * 1.001 + TINY[xt]).all(), np.abs(f64(xo) - ref_x).max()
    if h is not None:
        r = (1 / np.sqrt((ref_x ** 2).mean(1, keepdims=True) + 1e-5)) if pre else 1.0
        w = 1.0 if wn is None else np.abs(f64(wn))
        norm_err = np.sqrt((ex ** 2).mean(1, keepdims=True)) * r if pre else 0.0   # the root mean square moves by no more than ex's
        eh = ex * r * w + np.abs(ref_h) * (norm_err + d * e / 2 + 8 * e + U[bt] * 1.001) + TINY[bt]
        assert (np.abs(f64(h) - ref_h) <= eh).all(), np.abs(f64(h) - ref_h).max()


@pytest.mark.parametrize("xt,bt", [("f32", "bf16"), ("f32", "fp16"), ("f32", "f32"), ("bf16", "bf16"), ("fp16", "fp16")])
@pytest.mark.parametrize("d", [1, 2, 7, 8, 31, 64, 96, 100, 255, 256, 257, 1000, 1024, 2040, 2048, 4096, 4099, 5120, 5121, 8192, 11008, 16384])
def test_widths_and_types(xt, bt, d):
    case(d=d, xt=xt, bt=bt, seed=d)
    case(d=d, xt=xt, bt=bt, n=1, post=False, gain=False, gate="none", scale=1.0, seed=d + 1)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gain", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("d", [48, 127])
def test_every_combination(post, pre, gain, gate, d):
    case(n=5, d=d, post=post, pre=pre, gain=gain, gate=gate)


@pytest.mark.parametrize("want", [("x",), ("h",), ("x", "h")])
@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("d", [512, 513])
def test_outputs_that_are_not_wanted(want, block, d):
    case(n=4, d=d, want=want, block=block)


@pytest.mark.parametrize("n", [1, 2, 147, 148, 149, 1000])
@pytest.mark.parametrize("d", [64, 4096])
def test_row_counts(n, d):
    case(n=n, d=d, gate="token")


@pytest.mark.parametrize("d", [40, 255, 264, 500, 1001, 4097, 5121, 16383])
def test_many_rows(d):
    case(n=700, d=d, gate="token")
    case(n=601, d=d, xt="fp16", bt="fp16", pad=5, gate="channel")


@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (0, 1), (8, 8), (5, 3)])
@pytest.mark.parametrize("xt,bt", [("f32", "bf16"), ("fp16", "fp16")])
def test_strides_and_alignment(pad, off, xt, bt):
    case(n=6, d=1024, pad=pad, off=off, xt=xt, bt=bt, gate="token")


@pytest.mark.parametrize("d", [640, 641])
def test_in_place(d):
    case(n=9, d=d, alias=True)
    case(n=9, d=d, alias=True, xt="bf16", gate="token")


def test_a_row_of_zeros():
    case(zero_row=True)
    case(zero_row=True, d=33, gate="none")


def test_rows_do_not_touch_what_lies_between_them():
    x = torch.full((4, 80), 7.0, device=DEV)
    y = torch.full((4, 80), 7.0, device=DEV, dtype=torch.bfloat16)
    ls.ls_block_norm(x[:, :64], y[:, :64], x[:, :64], y[:, :64])
    torch.cuda.synchronize()
    assert (x[:, 64:] == 7).all() and (y[:, 64:] == 7).all() and (x[:, :64] == 14).all()


def test_infinite_and_nan_rows_stay_in_their_row():
    x, y = torch.ones(3, 256, device=DEV), torch.ones(3, 256, device=DEV).half()
    y[1, 5] = float("inf")
    x[2, 9] = float("nan")
    xo, h = torch.empty_like(x), torch.empty_like(y)
    ls.ls_block_norm(x, y, xo, h, post_norm=True)
    torch.cuda.synchronize()
    assert torch.isfinite(h[0]).all() and torch.isfinite(xo[0]).all() and torch.isnan(xo[1, 5]) and torch.isnan(h[2]).all()


def test_on_another_stream_and_in_a_graph():
    x, y = torch.randn(2, 512, device=DEV), torch.randn(2, 512, device=DEV).bfloat16()
    xo, h, h2 = torch.empty_like(x), torch.empty_like(y), torch.empty_like(y)
    ls.ls_block_norm(x, y, xo, h)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ls.ls_block_norm(x, y, xo, h2, stream=s)
    s.synchronize()
    assert torch.equal(h, h2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ls.ls_block_norm(x, y, xo, h2)
    h2.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, h2)
