"""What ls_paged_kv_append says of padding and of tokens that share a slot, on both of its kernels."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc
from paper_2609_03079_b200 import binding as ls
from test_gpu_paged_kv import DEV, f64, rope_table

pytestmark = pytest.mark.gpu


def setup(D, heads, hk, T, positions):
    gen = torch.Generator(device=DEV).manual_seed(D + heads)
    kp, vp = (torch.zeros(6, 16, hk, D, dtype=torch.float16, device=DEV) for _ in range(2))
    rope = rope_table(positions, D)
    q, k, v = torch.randn(T, heads + 2 * hk, D, generator=gen, device=DEV).half().split([heads, hk, hk], 1)
    return kp, vp, rope, q, k, v, ls.ls_paged_kv_create(kp, vp, heads, rope=rope)


@pytest.mark.parametrize("D,heads,hk", [(64, 4, 2), (128, 40, 8), (24, 4, 2)])
def test_queries_of_padding(D, heads, hk):
    """Turned by the position whatever the sequence; copied where the position is negative or beyond the rotation table."""
    seq, pos = [0, -1, -7, 0, -1, 0], [3, 7, 0, -1, -2, 45]
    kp, vp, rope, q, k, v, kv = setup(D, heads, hk, len(seq), 40)
    out = torch.full((len(seq), heads, D), float("nan"), dtype=torch.float16, device=DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    ls.ls_paged_kv_append(kv, q, k, v, out, i32(seq), i32(pos), i32([[0, 1, 2]]))
    assert ls.ls_paged_kv_status(kv) == ls.LS_ERR_INVALID  # the last token's position
    for t in (3, 4, 5):
        assert torch.equal(out[t], q[t])
    ref = orc.rotate(f64(q)[:3], pos[:3], f64(rope), False)
    size = np.abs(f64(q)[:3])
    pair = np.concatenate([size[..., : D // 2] + size[..., D // 2:]] * 2, -1)
    assert (np.abs(f64(out)[:3] - ref) <= 2.0 ** -11 * np.abs(ref) + 3 * 2.0 ** -24 * pair + 2.0 ** -25).all()
    assert not torch.equal(out[1], q[1]) and torch.equal(out[2], q[2])  # (position 0 turns by nothing)
    stored = torch.zeros(6, 16, dtype=torch.bool, device=DEV)
    stored[0, 3] = True
    assert (kp[stored] != 0).any() and not kp[~stored].any() and not vp[~stored].any()
    kv.close()


@pytest.mark.parametrize("D,heads,hk", [(64, 4, 2), (128, 40, 8), (24, 4, 2)])
def test_tokens_that_share_a_slot(D, heads, hk):
    """Every component that is stored is one of theirs."""
    T = 64
    kp, vp, rope, q, k, v, kv = setup(D, heads, hk, T, 40)
    one = torch.empty(T, hk, D, dtype=torch.float16, device=DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = i32([[0, 1, 2]])
    for t in range(T):
        ls.ls_paged_kv_append(kv, None, k[t:t + 1], v[t:t + 1], None, i32([0]), i32([20]), table)
        one[t] = kp[1, 4]
    ls.ls_paged_kv_append(kv, None, k, v, None, i32([0] * T), i32([20] * T), table)
    assert ls.ls_paged_kv_status(kv) == 0
    assert (kp[1, 4][None] == one).any(0).all() and (vp[1, 4][None] == v).any(0).all()
    kp[1, 4], vp[1, 4] = 0, 0
    assert not kp.any() and not vp.any()
    kv.close()
