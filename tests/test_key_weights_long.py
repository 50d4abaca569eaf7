"""Workspace of key weights for long prompts: chunks get longer instead of more (CPU), and what long chunks sum (GPU)."""
import numpy as np
import pytest
import torch

import paper_2512_10411_b200 as swaa
from paper_2512_10411_b200.build import build_library

SM = 148


@pytest.mark.parametrize("window,n_sink,full", [(1, 0, True), (2048, 4, False), (300, 100000, False), (100000, 4, False)])
@pytest.mark.parametrize("B,Hkv", [(1, 8), (8, 8), (64, 2), (1, 1)])
def test_workspace_is_bounded_and_grows(B, Hkv, window, n_sink, full):
    """One sequence of a million tokens and 8 key heads would have 512 chunks a key: 17 GB of sums for 33 MB of weights."""
    build_library()
    most = 64 * SM * 128 * 4 * (1 if not torch.cuda.is_available() else 2)  # 64 key tiles an SM, whatever the call
    last = 0
    for n in (1000, 2100, 9000, 32768, 70000, 131072, 300000, 2 ** 20, 2 ** 24, 2 ** 30):
        now = swaa.key_weights_workspace_size(B, n, n, 4 * Hkv, Hkv, window, n_sink, full)
        assert last <= now <= most
        assert swaa.key_weights_workspace_size(B, 64, n, 4 * Hkv, Hkv, window, n_sink, full) <= now
        assert swaa.key_weights_workspace_size(B, n, n, 4 * Hkv, Hkv, window, n_sink, full, last=500) <= now
        last = now


def test_prompts_that_fit_are_cut_as_before():
    """A 16k prompt of 8 key heads under full attention: 8 chunks of 16 query tiles."""
    build_library()
    assert swaa.key_weights_workspace_size(1, 16384, 16384, 32, 8, 1, 0, True) == 8 * 128 * 8 * 128 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("D,mask", [(64, (9, 9, True)), (128, (9, 9, True)), (64, (300, 2 ** 19, False))])
def test_long_chunks(D, mask, paged):
    """The stated longest sequence decides how long a chunk is: with a million tokens the ten query tiles of the first are one chunk of 640
    steps, more than 256 for either group of warps."""
    from test_key_weights_gpu import call, check, make

    lens, most, Hq, Hkv = (1200, 300, 1), 2 ** 20, 64, 1
    s = {**make(lens, lens, Hq, Hkv, D, 17, paged), "max_q": most, "max_k": most}
    if paged:
        s["table"] = torch.nn.functional.pad(s["table"], (0, most // 128 - s["table"].shape[1]), value=-1)
    w = torch.full((3, Hkv, most if paged else 1200), 9.0, device="cuda")
    call(s, None, w, mask)
    assert swaa.last_device_status() == 0
    check(s, lens, lens, None, w, mask, 0, D ** -0.5)
    again = torch.full_like(w, 9.0)
    call(s, None, again, mask)
    assert torch.equal(again, w)
    # the sums of short chunks, joined: the same terms in another order
    short = torch.full((3, Hkv, 1200), 9.0, device="cuda")
    few = {**s, "max_q": 1200, "max_k": 1200}
    if paged:
        few["table"] = s["table"][:, :10].contiguous()
    call(few, None, short, mask)
    assert swaa.last_device_status() == 0
    a, b = w[0, :, :1200].double().cpu().numpy(), short[0].double().cpu().numpy()
    assert (np.abs(a - b) <= 2 * (1200 * Hq // Hkv + 16) * 2.0 ** -24 * b + 1e-30).all()
