"""Calls of the 4-bit cache one behind the other and side by side: every call's own outputs are looked at, as it left them."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls
from test_gpu_kv4_attend import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,hk", [(4, 2), (16, 2)])
def test_every_step_of_calls_back_to_back(heads, hk):
    """Append, attention, append ... without a wait between: what each left behind is looked at, with no second call."""
    B, steps = 3, 40
    b = Batch(lens=[steps] * B, heads=heads, hk=hk)
    kv = b.handle()
    b.pages.fill_(255)
    gen = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(steps, B, hk, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    seq = torch.arange(B, dtype=torch.int32, device=DEV)
    lens = [torch.full((B,), t + 1, dtype=torch.int32, device=DEV) for t in range(steps)]
    pos = [n - 1 for n in lens]
    outs = torch.full((steps, B, 1, heads, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    lses = torch.full((steps, B, 1, heads), float("nan"), device=DEV)
    torch.cuda.synchronize()
    for t in range(steps):
        ls.ls_paged_kv4_append(kv, None, k[t], v[t], None, seq, pos[t], b.table)
        ls.ls_paged_kv4_attend(kv, b.q, outs[t], lens[t], b.table, lse=lses[t])
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()
    for t in range(steps):
        b.lens, b.out, b.lse = [t + 1] * B, outs[t], lses[t]
        b.check()


def test_every_call_of_two_handles_at_once():
    """Two caches' calls on two streams: all outputs of all calls, none written over by the next."""
    batches = [Batch(lens=[900, 30, 0, 2000], heads=16, hk=2, seed=s) for s in (3, 4)]
    handles, streams = [b.handle() for b in batches], [torch.cuda.Stream() for _ in batches]
    outs = [torch.full((50, *b.out.shape), float("nan"), dtype=b.out.dtype, device=DEV) for b in batches]
    lses = [torch.full((50, *b.lse.shape), float("nan"), device=DEV) for b in batches]
    torch.cuda.synchronize()
    for i in range(50):
        for b, kv, st, o, l in zip(batches, handles, streams, outs, lses):
            with torch.cuda.stream(st):
                ls.ls_paged_kv4_attend(kv, b.q, o[i], b.seq_len, b.table, lse=l[i])
    torch.cuda.synchronize()
    for b, kv, o, l in zip(batches, handles, outs, lses):
        assert ls.ls_paged_kv4_status(kv) == 0
        b.out, b.lse = o[0], l[0]
        b.check()
        assert all(torch.equal(o[i], o[0]) and torch.equal(l[i], l[0]) for i in range(50))
        kv.close()


def test_append_attention_and_read_of_every_step():
    """A token is stored, attended to and read back, step by step on one stream without a wait: each read brings what its own step stored, not what the
    next one puts in the same place."""
    b = Batch(lens=[1], heads=4, hk=2)
    kv = b.handle()
    steps = 60
    gen = torch.Generator(device=DEV).manual_seed(2)
    k, v = (torch.randn(steps, 1, 2, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    ko, vo = (torch.full_like(k, float("nan")) for _ in range(2))
    outs = torch.full((steps, 1, 1, 4, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    for t in range(steps):
        ls.ls_paged_kv4_append(kv, None, k[t], v[t], None, zero, zero, b.table)
        ls.ls_paged_kv4_attend(kv, b.q, outs[t], b.seq_len, b.table)
        ls.ls_paged_kv4_read(kv, ko[t], vo[t], zero, zero, b.table)
    assert ls.ls_paged_kv4_status(kv) == 0
    kv.close()
    for x, y in ((k, ko), (v, vo)):  # half a step of 15, the scale's rounding 15 times, the last rounding
        x, y = x.float().view(steps, 2, 2, 64), y.float().view(steps, 2, 2, 64)
        step = (x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)) / 15
        assert ((x - y).abs() <= step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -8 * y.abs()).all()
    # one key: the value that the cache holds of it, rounded once, as read (a weight times a scale is rounded to 2^-11, and counts up to 8 of it)
    seen = vo.repeat_interleave(2, 2).float()
    room = (vo.float().view(steps, 1, 2, 2, 64).amax(-1) - vo.float().view(steps, 1, 2, 2, 64).amin(-1)).repeat_interleave(64, -1).repeat_interleave(2, 2)
    assert ((outs[:, 0].float() - seen).abs() <= 2 * 2.0 ** -8 * seen.abs() + 2.0 ** -11 * 8 / 15 * 1.1 * room + 2.0 ** -20).all()
