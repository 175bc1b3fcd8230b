"""A prompt kept in a 16-bit cache moved into a 4-bit one: its keys are turned already, so the 4-bit handle that takes them has no rotation table."""
import pytest
import torch

from paper_2609_03079_b200 import binding as ls
from paper_2609_03079_b200.decoder import rope_table

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_16_bit_prompt_goes_on_in_4_bits(dtype):
    """Keys and values read back are those of the 16-bit cache to half a step (and the roundings of 15 scales and of the result); the next token is
    appended through a handle with the rotation, over the same pages, and stands where one that never moved does."""
    H, HK, D, page, n, group = 8, 2, 64, 16, 70, 32
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    gen = torch.Generator(device=DEV).manual_seed(0)
    rope = rope_table(128, D, device=DEV)
    k, v = (torch.randn(n + 1, HK, D, generator=gen, device=DEV).to(dtype) for _ in range(2))
    pages = -(-(n + 1) // page)
    table = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)[None]
    pos, zero = torch.arange(n + 1, dtype=torch.int32, device=DEV), torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    kp, vp = (torch.zeros(pages, page, HK, D, dtype=dtype, device=DEV) for _ in range(2))
    k16 = ls.ls_paged_kv_create(kp, vp, H, rope=rope)
    ls.ls_paged_kv_append(k16, None, k[:n], v[:n], None, zero[:n], pos[:n], table)
    at = table[0, (pos[:n] // page).long()].long()
    turned, values = kp[at, (pos[:n] % page).long()], vp[at, (pos[:n] % page).long()]

    def cache(rope_, raw):
        return ls.ls_paged_kv4_create(raw, H, D, page, dtype=dtype, group=group, rope=rope_)

    raw, direct = (torch.zeros(pages, HK, ls.ls_paged_kv4_block_bytes(page, D, group), dtype=torch.uint8, device=DEV) for _ in range(2))
    plain, rotating, other = cache(None, raw), cache(rope, raw), cache(rope, direct)
    ls.ls_paged_kv4_append(plain, None, turned, values, None, zero[:n], pos[:n], table)
    ko, vo = torch.empty_like(turned), torch.empty_like(values)
    ls.ls_paged_kv4_read(plain, ko, vo, zero[:n], pos[:n], table)
    for x, y in ((turned, ko), (values, vo)):
        x, y = x.float().unflatten(-1, (-1, group)), y.float().unflatten(-1, (-1, group))
        step = (x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)) / 15
        assert ((x - y).abs() <= step * (0.5 + 15 * u) + u * y.abs() + 2.0 ** -24).all()
    last = []
    for c in (rotating, other):
        ls.ls_paged_kv4_append(c, None, k[n:], v[n:], None, zero[n:], pos[n:], table)
        a, b = torch.empty_like(k[n:]), torch.empty_like(k[n:])
        ls.ls_paged_kv4_read(c, a, b, zero[n:], pos[n:], table)
        last.append((a, b))
    assert torch.equal(last[0][0], last[1][0]) and torch.equal(last[0][1], last[1][1])
    assert [ls.ls_paged_kv4_status(c) for c in (plain, rotating, other)] == [0] * 3 and ls.ls_paged_kv_status(k16) == 0
    for c in (plain, rotating, other, k16):
        c.close()
