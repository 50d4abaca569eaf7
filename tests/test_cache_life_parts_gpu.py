"""A training step through norm, rotation and attention part by part, and the weights of a long decode against the roundings of the sums
that a lane really takes."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa
from test_cache_life_gpu import BF, D, EPS, HKV, HQ, Layer, f64, int32, split

pytestmark = pytest.mark.gpu
W, S = 16, 2


def step(layer, n):
    """Forward and backward through the library: projection, gradient of its output and what stood between, float64."""
    qkv = layer.project(n)
    pos, cu = torch.arange(n, dtype=torch.int32, device="cuda"), int32([0, n])
    q, k, v = (torch.empty(n, h, D, dtype=BF, device="cuda") for h in (HQ, HKV, HKV))
    swaa.swaa_qk_norm_rope(*split(qkv), layer.qw, layer.kw, layer.f, pos, q, k, v, eps=EPS)
    out, lse = torch.empty_like(q), torch.empty(HQ, n, device="cuda")
    swaa.swaa_prefill(q, k, v, out, cu, n, W, S, False, lse=lse)
    dout = torch.randn(n, HQ, D, generator=layer.g, device="cuda").to(BF)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(swaa.prefill_backward_workspace_size(1, n, HQ, HKV, D, S), dtype=torch.uint8, device="cuda")
    swaa.swaa_prefill_backward(q, k, v, out, dout, lse, cu, n, W, S, False, dq, dk, dv, ws)
    dqkv, dqw, dkw = torch.empty_like(qkv), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(swaa.qk_norm_rope_backward_workspace_size(n, HQ, HKV, D), dtype=torch.uint8, device="cuda")
    swaa.swaa_qk_norm_rope_backward(*split(qkv)[:2], dq, dk, dv, layer.qw, layer.kw, layer.f, pos, *split(dqkv), dqw, dkw, ws, eps=EPS)
    assert swaa.last_device_status() == 0
    return {name: f64(x) for name, x in dict(x=qkv, dx=dqkv, dout=dout, dq=dq, dk=dk, dv=dv, dqw=dqw, dkw=dkw, qw=layer.qw, kw=layer.kw, f=layer.f).items()}


def parts(x):
    return dict(q=x[:, :HQ], k=x[:, HQ:HQ + HKV], v=x[:, HQ + HKV:])


def gradients(s, n):
    """Gradients of the whole chain, by torch's differentiation of it in float64."""
    x, qw, kw = (torch.tensor(s[name], requires_grad=True) for name in ("x", "qw", "kw"))
    t = torch.arange(n, dtype=torch.float64)[:, None, None] * torch.tensor(s["f"])
    c, si = torch.cos(t), torch.sin(t)

    def turned(y, w):
        y = w * y / (y.square().mean(-1, keepdim=True) + EPS).sqrt()
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * c - b * si, b * c + a * si], -1)

    q, k, v = x.split((HQ, HKV, HKV), 1)
    k, v = (y.repeat_interleave(HQ // HKV, 1) for y in (turned(k, kw), v))
    scores = torch.einsum("ihd,jhd->hij", turned(q, qw), k) * D ** -0.5
    i = np.arange(n)
    seen = torch.tensor(ref.visible(i[:, None], i[None], W, S, False))
    p = torch.softmax(scores.masked_fill(~seen, -torch.inf), -1)
    (torch.einsum("hij,jhd->ihd", p, v) * torch.tensor(s["dout"])).sum().backward()
    return parts(x.grad.numpy()), qw.grad.numpy(), kw.grad.numpy()


@pytest.mark.parametrize("n", [1, 40, 130])
def test_parts_of_a_training_step(n):
    layer = Layer(14)
    s = step(layer, n)
    got, x = parts(s["dx"]), parts(s["x"])
    want, want_qw, want_kw = gradients(s, n)
    assert np.array_equal(got["v"], s["dv"])
    # q, k, v, P, the attention's output, dS, dq or dk and the result are rounded to bf16 on the way: eight half steps, each relative to
    # what it rounds.  The term of the norm's gradient along the input is about 1/8 of the norm of the q and k parts (one of 64 channels).
    for name in "qkv":
        size = np.linalg.norm(want[name])
        if n == 1 and name != "v":  # the only key has weight 1 whatever the scores: 0 but for the rounding of dS
            size = np.linalg.norm(s["dout"])
        assert np.linalg.norm(got[name] - want[name]) <= 8 * ref.HALF_BF16 * size, name
    for name, w in (("dqw", want_qw), ("dkw", want_kw)):
        size = np.linalg.norm(w) if n > 1 else np.linalg.norm(s["dout"])
        assert np.linalg.norm(s[name] - w) <= 8 * ref.HALF_BF16 * size, name
    # A head's norm does not change along its input x, so neither does the loss: x . dx is 0 but for eps, (x . w g) r eps / (m + eps), for
    # half a step of bf16 of every channel of dx and for what fp32 adds to it.
    for name, w, dy in (("q", s["qw"], s["dq"]), ("k", s["kw"], s["dk"])):
        wg = w * ref.rotate(dy, np.arange(n), s["f"], False, back=True)
        m = (x[name] ** 2).mean(-1, keepdims=True)
        r = (m + EPS) ** -0.5
        _, bound, _, _ = ref.qk_rope_backward(x[name], w, EPS, np.arange(n), s["f"], False, dy)
        rest = (x[name] * wg).sum(-1) * (r * EPS / (m + EPS))[..., 0]
        assert (np.abs((x[name] * got[name]).sum(-1) - rest) <= (np.abs(x[name]) * bound).sum(-1)).all(), name
        if n > 1:  # without that term it would be (x . w g) r, far outside of the bound
            lost = np.abs((x[name] * wg).sum(-1) * r[..., 0])
            assert (lost[1:] > (np.abs(x[name]) * bound).sum(-1)[1:]).mean() > 0.5


@pytest.mark.parametrize("L,Hq,Hkv", [(500_000, 2, 2), (300_001, 8, 2), (64 * 148 * 3, 1, 1)])
def test_weights_of_a_long_row(L, Hq, Hkv):
    """Every key but the last scores 0.  A lane adds two terms per tile of 64 entries, one after another, and a block takes tiles /
    blocks of them; the lanes, warps and blocks of a row are added at the end."""
    g = torch.Generator(device="cuda").manual_seed(15)
    kc, vc = (torch.zeros(1, L, Hkv, D, dtype=BF, device="cuda") for _ in range(2))
    kc[0, L - 1] = torch.randn(Hkv, D, generator=g, device="cuda").to(BF)
    q = torch.randn(1, Hq, D, generator=g, device="cuda").to(BF)
    out, w = torch.empty_like(q), torch.full((1, Hkv, L), float("nan"), device="cuda")
    ws = torch.empty(swaa.decode_weighted_workspace_size(1, Hq, Hkv, D, L, 1, 0, True), dtype=torch.uint8, device="cuda")
    swaa.swaa_decode_weighted(q, kc, vc, out, None, w, int32([L]), 1, 0, True, ws)
    assert swaa.last_device_status() == 0
    blocks = swaa.decode_num_blocks(1, Hq, Hkv, D, L, 1, 0, True)
    tiles = -(-Hkv * -(-L // 64) // blocks) + 1
    x = np.einsum("hgd,hd->hg", f64(q[0]).reshape(Hkv, -1, D), f64(kc[0, L - 1])) * D ** -0.5
    rest = 1 / (L - 1 + np.exp(x))
    # half steps of fp32: a lane's additions, 32 lanes, 4 warps, the blocks; an exponent up to its size in powers of two, rounded four times
    # (see the softmax weights of the reference); the scores of the last key, D products; the sum over the group
    steps = 2 * tiles + 5 + 4 + blocks + 4 * 1.45 * (np.abs(x).max() + np.log(L) + 4) + 16 + Hq // Hkv
    score = 2 * (D + 2) * 2 * np.einsum("hgd,hd->hg", np.abs(f64(q[0])).reshape(Hkv, -1, D), np.abs(f64(kc[0, L - 1]))).max() * D ** -0.5
    bound = (steps + score * np.exp(x).max() / L) * ref.U32  # of the other keys: the last one is a small part of the row's sum
    assert bound < 5e-5  # (500000 entries of 2 heads: 106 tiles a block)
    np.testing.assert_allclose(f64(w[0, :, L - 1]), (np.exp(x) * rest).sum(1), rtol=bound + score * ref.U32)
    np.testing.assert_allclose(f64(w[0, :, :L - 1]), np.broadcast_to(rest.sum(1)[:, None], (Hkv, L - 1)), rtol=bound)
    np.testing.assert_allclose(f64(w[0].double().sum(-1)), Hq // Hkv, rtol=bound)
