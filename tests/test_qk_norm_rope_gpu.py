"""Norm and rotation of queries and keys, and their gradient, against the float64 definition."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa

pytestmark = pytest.mark.gpu
EPS = 1e-6


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def make(T, Hq, Hkv, D, rot, seed, norm="qk", spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (spread * torch.randn(T, Hq + 2 * Hkv, D, generator=g, device="cuda")).bfloat16()
    w = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") if c in norm else None for c in "qk"]
    f = (1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda() if rot else None
    pos = torch.randint(0, 200000, (T,), generator=g, device="cuda", dtype=torch.int32)
    return qkv, w, f, pos


def check(got, want, bound, what):
    err = np.abs(f64(got) - want)
    assert (err <= bound).all(), f"{what}: {err.max()} at {np.unravel_index((err - bound).argmax(), err.shape)}, worst {np.max(err / bound)} of its bound"


def freqs(f):
    return np.zeros(0) if f is None else f64(f)


SHAPES = [(1, 4, 2, 64, 64), (37, 4, 2, 64, 32), (300, 16, 4, 64, 16), (5, 1, 1, 64, 64), (2, 28, 4, 128, 128), (37, 32, 8, 128, 64), (130, 64, 8, 128, 128),
          (3, 7, 7, 128, 16), (65, 5, 1, 128, 112), (9, 28, 4, 64, 48), (4, 4, 2, 128, 0), (2500, 4, 2, 64, 64)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["qk", "", "q"])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
def test_forward(T, Hq, Hkv, D, rot, norm, interleaved):
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, rot, 5, norm)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    outs = [torch.full((T + 2, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    qo, ko, vo = (o[1:-1] for o in outs)
    swaa.swaa_qk_norm_rope(q, k, v, qw, kw, f, pos, qo, ko, vo, eps=EPS, interleaved=interleaved)
    assert swaa.last_device_status() == 0
    for got, x, w, what in ((qo, q, qw, "q"), (ko, k, kw, "k")):
        want, bound = ref.qk_rope(f64(x), f64(w), EPS, f64(pos), freqs(f), interleaved)
        check(got, want, bound, what)
    assert torch.equal(vo, v)
    for o in outs:
        assert (o[0] == 7).all() and (o[-1] == 7).all(), "store outside the output"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["qk", "", "k"])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
def test_backward(T, Hq, Hkv, D, rot, norm, interleaved):
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, rot, 6, norm)
    q, k, _ = qkv.split((Hq, Hkv, Hkv), 1)
    g = torch.Generator(device="cuda").manual_seed(8)
    d = [torch.randn(T, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    dqkv = torch.full((T + 2, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    dq, dk, dv = dqkv[1:-1].split((Hq, Hkv, Hkv), 1)
    dw = [torch.full((D,), 9.0, device="cuda") if w is not None else None for w in (qw, kw)]
    n = swaa.qk_norm_rope_backward_workspace_size(T, Hq, Hkv, D)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")

    def call():
        swaa.swaa_qk_norm_rope_backward(q if qw is not None else None, k if kw is not None else None, *d, qw, kw, f, pos, dq, dk, dv, *dw,
                                        ws[256:256 + n] if norm else None, eps=EPS, interleaved=interleaved)
        assert swaa.last_device_status() == 0

    call()
    for got, x, w, dy, gw, what in ((dq, q, qw, d[0], dw[0], "dq"), (dk, k, kw, d[1], dw[1], "dk")):
        want, bound, want_w, bound_w = ref.qk_rope_backward(f64(x), f64(w), EPS, f64(pos), freqs(f), interleaved, f64(dy))
        check(got, want, bound, what)
        if w is not None:
            check(gw, want_w, bound_w, what + " weight")
    assert torch.equal(dv, d[2])
    assert (dqkv[0] == 7).all() and (dqkv[-1] == 7).all() and (ws[:256] == 0xA5).all() and (ws[-256:] == 0xA5).all()
    first = [x.clone() for x in (dqkv, *dw) if x is not None]
    ws.fill_(0xFF)
    call()
    for a, b in zip(first, (x for x in (dqkv, *dw) if x is not None)):
        assert torch.equal(a, b), "a repeated call has other bits"


def test_far_and_negative_positions():
    T, Hq, Hkv, D = 8, 4, 2, 128
    qkv, (qw, kw), f, _ = make(T, Hq, Hkv, D, D, 7)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    pos = torch.tensor([0, -1, 1, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 999983], dtype=torch.int32, device="cuda")
    qo, ko = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, Hkv, D, dtype=torch.bfloat16, device="cuda")
    swaa.swaa_qk_norm_rope(q, k, None, qw, kw, f, pos, qo, ko, None, eps=EPS)
    # float64 angles of the reference: 2^31 * 2^-53 radians, far below the bound
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        check(got, *ref.qk_rope(f64(x), f64(w), EPS, f64(pos), f64(f), False), "far")
    assert swaa.last_device_status() == 0


@pytest.mark.parametrize("T", [1, 40])
def test_in_place(T):
    Hq, Hkv, D = 16, 4, 64
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, 32, 9)
    q, k, v = (x.contiguous() for x in qkv.split((Hq, Hkv, Hkv), 1))
    want = [torch.empty_like(x) for x in (q, k)]
    swaa.swaa_qk_norm_rope(q, k, None, qw, kw, f, pos, *want, None)
    x = [q.clone(), k.clone()]
    swaa.swaa_qk_norm_rope(*x, None, qw, kw, f, pos, *x, None)
    assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])
    ws = torch.empty(swaa.qk_norm_rope_backward_workspace_size(T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    d = [torch.randn(T, h, D, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    dx, dw = [torch.empty_like(t) for t in d], [torch.empty(D, device="cuda") for _ in range(4)]
    swaa.swaa_qk_norm_rope_backward(q, k, *d, qw, kw, f, pos, *dx, *dw[:2], ws)
    y = [t.clone() for t in d]
    swaa.swaa_qk_norm_rope_backward(q, k, *y, qw, kw, f, pos, *y, *dw[2:], ws)  # over the incoming gradients
    for a, b in zip(dx + dw[:2], y + dw[2:]):
        assert torch.equal(a, b)
    swaa.swaa_qk_norm_rope_backward(q, k, *d, qw, kw, f, pos, q, k, y[2], *dw[2:], ws)  # over the inputs
    for a, b in zip(dx[:2] + dw[:2], [q, k] + dw[2:]):
        assert torch.equal(a, b)


def test_rows_of_zeros_and_infinities():
    """A zero head stays zero (eps); without a norm, channels that are not rotated pass infinities and NaN as they are, and the
    pairs around them are untouched."""
    T, Hq, Hkv, D, rot = 3, 4, 2, 64, 32
    for interleaved in (False, True):
        qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, rot, 10)
        q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
        q[1, 2] = 0
        q[0, 1, 40], q[0, 1, 63], q[2, 3, 33] = float("inf"), float("nan"), float("-inf")
        qo, ko = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, Hkv, D, dtype=torch.bfloat16, device="cuda")
        swaa.swaa_qk_norm_rope(q, k, None, qw, kw, f, pos, qo, ko, None, eps=EPS, interleaved=interleaved)
        assert (qo[1, 2] == 0).all() and torch.isfinite(ko.float()).all()
        swaa.swaa_qk_norm_rope(q, k, None, None, None, f, pos, qo, ko, None, interleaved=interleaved)
        assert torch.equal(qo[..., rot:].nan_to_num(3.0), q[..., rot:].nan_to_num(3.0))
        want, bound = ref.qk_rope(f64(q)[..., :rot], None, EPS, f64(pos), f64(f), interleaved)
        check(qo[..., :rot], want, bound, "rotated channels")


def test_no_tokens():
    z = torch.empty(0, 6, 64, dtype=torch.bfloat16, device="cuda")
    q, k = z[:, :4], z[:, 4:]
    f, pos, w = torch.ones(32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    swaa.swaa_qk_norm_rope(q, k, k, w, w, f, pos, q.contiguous(), k.contiguous(), k.contiguous())
    dw = [torch.full((64,), 5.0, device="cuda") for _ in range(2)]
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    swaa.swaa_qk_norm_rope_backward(q, k, q.contiguous(), k.contiguous(), k.contiguous(), w, w, f, pos, q, k, k, *dw, ws)
    assert (dw[0] == 0).all() and (dw[1] == 0).all() and swaa.last_device_status() == 0


def test_other_stream_and_graph():
    T, Hq, Hkv, D = 50, 32, 8, 128
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, D, 11)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    d = [torch.randn(T, h, D, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    ws = torch.empty(swaa.qk_norm_rope_backward_workspace_size(T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    out = [torch.empty(T, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv) * 2] + [torch.empty(D, device="cuda") for _ in range(2)]

    def call(stream=None):
        swaa.swaa_qk_norm_rope(q, k, v, qw, kw, f, pos, *out[:3], stream=stream)
        swaa.swaa_qk_norm_rope_backward(q, k, *d, qw, kw, f, pos, *out[3:6], *out[6:], ws, stream=stream)

    call()
    want = [x.clone() for x in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x in out:
        x.zero_()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(2):
        for x in out:
            x.zero_()
        graph.replay()
        assert swaa.last_device_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refused_tensors():
    T, Hq, Hkv, D = 3, 4, 2, 64
    qkv, (qw, kw), f, pos = make(T, Hq, Hkv, D, D, 12)
    good = dict(zip(("q", "k", "v"), qkv.split((Hq, Hkv, Hkv), 1)))
    good.update(q_weight=qw, k_weight=kw, inv_freq=f, positions=pos)
    good.update({n: torch.empty(T, h, D, dtype=torch.bfloat16, device="cuda") for n, h in (("q_out", Hq), ("k_out", Hkv), ("v_out", Hkv))})
    swaa.swaa_qk_norm_rope(**good)
    bad = [(dict(k=good["k"][:2]), ValueError), (dict(v=good["v"][:, :1]), ValueError), (dict(positions=pos[:2]), ValueError), (dict(positions=pos.long()), TypeError),
           (dict(q=good["q"].float()), TypeError), (dict(q=good["q"].cpu()), TypeError), (dict(q=good["q"].transpose(0, 1).contiguous().transpose(0, 1)), ValueError),
           (dict(k_out=good["v_out"][:, :1]), ValueError), (dict(q_out=torch.empty(T, Hq, 2 * D, dtype=torch.bfloat16, device="cuda")[..., :D]), ValueError),
           (dict(q_weight=qw.bfloat16()), TypeError), (dict(k_weight=kw[:32]), ValueError), (dict(v_out=None), swaa.SwaaError), (dict(inv_freq=f[:5]), swaa.SwaaError),
           (dict(q=torch.empty(T, Hq * D + 4, dtype=torch.bfloat16, device="cuda")[:, :Hq * D].view(T, Hq, D)), swaa.SwaaError)]
    for change, error in bad:
        with pytest.raises(error):
            swaa.swaa_qk_norm_rope(**{**good, **change})
    assert swaa.last_device_status() == 0
