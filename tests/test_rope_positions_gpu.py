"""Calls of few tokens whose positions are the head of a longer tensor: what stands behind them changes nothing."""
import pytest
import torch

import paper_2512_10411_b200 as swaa
from test_qk_norm_rope_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 4, 2, 64), (1, 16, 4, 64), (3, 32, 8, 128), (17, 5, 1, 64), (37, 4, 2, 64), (2, 7, 7, 128)])
def test_positions_are_the_head_of_a_longer_tensor(T, Hq, Hkv, D):
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, D, 21)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, T], [T + 5]))
    got = []
    for behind in (0, 2 ** 31 - 1):
        longer = torch.full((T + 64,), behind, dtype=torch.int32, device="cuda")
        longer[:T] = pos
        out = [torch.zeros(T, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv, Hq)] + [torch.zeros(1, T + 7, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        swaa.swaa_qk_norm_rope(q, k, v, qw, kw, f, longer[:T], *out[:3])
        swaa.swaa_cache_append(q, k, v, qw, kw, f, cu, lens, *out[3:], positions=longer[:T])
        assert swaa.last_device_status() == 0
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    out = got[0]
    assert torch.equal(out[3], out[0]) and torch.equal(out[4][0, 5:T + 5], out[1]) and torch.equal(out[5][0, 5:T + 5], out[2])
    assert out[0].any() and not out[4][0, :5].any() and not out[4][0, T + 5:].any()
