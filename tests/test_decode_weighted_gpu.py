"""Decode that gathers attention weights: the output is swaa_decode's, bit for bit; the weights are those of the float64 softmax."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def make(lens, Hq, Hkv, D, form, seed, page=64):
    B, g, rng = len(lens), torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    q = torch.randn(B, Hq, D, generator=g, device="cuda").bfloat16()
    L = max(lens) + 3
    kd = torch.randn(B, L, Hkv, D, generator=g, device="cuda").bfloat16()
    vd = torch.randn(B, L, Hkv, D, generator=g, device="cuda").bfloat16()
    for b, n in enumerate(lens):  # what lies behind a sequence is never used
        kd[b, n:], vd[b, n:] = float("nan"), float("nan")
    if form == "dense":
        return q, kd, vd, None, kd
    used = [-(-n // page) for n in lens]
    order = rng.permutation(sum(used) + 2)
    table = np.full((B, max(used) + 1), -1, dtype=np.int32)
    k, v = (torch.full((len(order), page, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = 0
    for b, n in enumerate(lens):
        for i in range(used[b]):
            table[b, i] = order[at]
            m = min(page, n - i * page)
            k[order[at], :m], v[order[at], :m] = kd[b, i * page:i * page + m], vd[b, i * page:i * page + m]
            at += 1
    return q, k, v, torch.tensor(table, device="cuda"), kd


def calls(q, k, v, table, lens_t, mask, w_in, w_out, scale=0.0):
    """(weighted call, its output, plain output, guards of the workspace)"""
    B, Hq, D = q.shape
    Hkv = k.shape[2]
    L = k.shape[1] if table is None else table.shape[1] * k.shape[1]
    out, plain = torch.full_like(q, 7.0), torch.full_like(q, 5.0)
    n = swaa.decode_weighted_workspace_size(B, Hq, Hkv, D, L, *mask)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")

    def call():
        if table is None:
            swaa.swaa_decode_weighted(q, k, v, out, w_in, w_out, lens_t, *mask, ws[256:256 + n], scale=scale)
        else:
            swaa.swaa_decode_weighted_paged(q, k, v, out, w_in, w_out, table, lens_t, *mask, ws[256:256 + n], scale=scale)

    if table is None:
        wp = torch.empty(swaa.decode_workspace_size(B, Hq, Hkv, D, L, *mask), dtype=torch.uint8, device="cuda")
        swaa.swaa_decode(q, k, v, plain, lens_t, *mask, wp, scale=scale)
    else:
        wp = torch.empty(swaa.decode_paged_workspace_size(B, Hq, Hkv, D, table.shape[1], k.shape[1], *mask), dtype=torch.uint8, device="cuda")
        swaa.swaa_decode_paged(q, k, v, plain, table, lens_t, *mask, wp, scale=scale)
    return call, out, plain, ws


def check_weights(w_out, w_in, q, kd, lens, mask, scale, G):
    got = f64(w_out)
    for b, n in enumerate(lens):
        want, bound = ref.decode_weights(f64(q[b]), f64(kd[b, :n]), n, *mask, scale)
        old = np.zeros_like(want)
        if w_in is not None:
            old[:, :n - 1] = f64(w_in)[b, :, :n - 1]
        err = np.abs(got[b, :, :n] - (old + want))
        bound = bound + 2 * ref.U32 * (old + want)
        assert (err <= bound).all(), (b, err.max(), np.max(err / bound))
        if mask[2]:
            assert abs(want.sum() - q.shape[1]) < 1e-9


@pytest.mark.parametrize("form", ["dense", "paged"])
@pytest.mark.parametrize("window,n_sink,full", [(2048, 4, True), (100, 4, False), (1, 0, False), (64, 70, False), (300, 0, False)])
@pytest.mark.parametrize("lens,Hq,Hkv,D", [((1,), 4, 2, 64), ((300, 1, 17, 64, 65, 1000), 8, 2, 128), ((515, 130), 28, 4, 64), ((700, 3), 64, 8, 128),
                                           ((333,), 9, 1, 128), ((200, 90), 20, 1, 64), ((129,), 3, 3, 128), ((5000, 20), 16, 4, 64)])
def test_weights(lens, Hq, Hkv, D, window, n_sink, full, form):
    q, k, v, table, kd = make(lens, Hq, Hkv, D, form, 3)
    lens_t, mask = torch.tensor(lens, dtype=torch.int32, device="cuda"), (window, n_sink, full)
    rows = max(lens) + 5
    w_in = torch.rand(len(lens), Hkv, rows, device="cuda")
    for b, n in enumerate(lens):
        w_in[b, :, n - 1] = float("nan")  # the new token's own entry may hold anything
    w_out = torch.full_like(w_in, 9.0)
    call, out, plain, ws = calls(q, k, v, table, lens_t, mask, w_in, w_out)
    call()
    assert swaa.last_device_status() == 0
    assert torch.equal(out, plain)
    assert (ws[:256] == 0xA5).all() and (ws[-256:] == 0xA5).all(), "store outside the workspace"
    for b, n in enumerate(lens):
        assert (w_out[b, :, n:] == 9).all(), "entries behind the sequence were written"
    check_weights(w_out, w_in, q, kd, lens, mask, D ** -0.5, Hq // Hkv)
    first = w_out.clone()
    same = w_in.clone()
    call, out, plain, ws = calls(q, k, v, table, lens_t, mask, same, same)  # in place
    call()
    fresh = torch.full_like(w_in, 9.0)
    call2, *_ = calls(q, k, v, table, lens_t, mask, None, fresh)
    call2()
    for b, n in enumerate(lens):
        assert torch.equal(same[b, :, :n], first[b, :, :n]) and torch.equal(same[b, :, n:], w_in[b, :, n:])
    check_weights(fresh, None, q, kd, lens, mask, D ** -0.5, Hq // Hkv)


def test_scale_wide_scores_and_many_sequences():
    lens = [1 + (37 * i) % 400 for i in range(70)]
    q, k, v, table, kd = make(lens, 8, 2, 64, "dense", 8)
    q *= 6  # scores of standard deviation 20: weights from 1 down to 0
    lens_t, mask = torch.tensor(lens, dtype=torch.int32, device="cuda"), (50, 3, True)
    w_out = torch.zeros(70, 2, 400, device="cuda")
    call, out, plain, _ = calls(q, k, v, table, lens_t, mask, None, w_out, scale=0.4)
    call()
    assert swaa.last_device_status() == 0 and torch.equal(out, plain)
    check_weights(w_out, None, q, kd, lens, mask, np.float64(np.float32(0.4)), 4)


def test_bad_lengths_and_short_weights():
    lens = (40, 40, 40)
    q, k, v, _, kd = make(lens, 4, 2, 64, "dense", 9)
    for bad in (0, 44, -3):
        lens_t = torch.tensor([40, bad, 7], dtype=torch.int32, device="cuda")
        w = torch.full((3, 2, 60), 9.0, device="cuda")
        call, out, _, _ = calls(q, k, v, None, lens_t, (8, 2, True), None, w)
        swaa.last_device_status()
        call()
        assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
        assert (w[1] == 9).all() and (out[1] == 0).all() and abs(w[0, :, :40].sum().item() - 4) < 1e-4 and abs(w[2, :, :7].sum().item() - 4) < 1e-4
    w = torch.full((3, 2, 20), 9.0, device="cuda")  # 40 entries do not fit
    lens_t = torch.tensor([40, 20, 7], dtype=torch.int32, device="cuda")
    call, out, plain, _ = calls(q, k, v, None, lens_t, (8, 2, True), None, w)
    call()
    assert swaa.last_device_status() == -5 and (w[0] == 9).all() and torch.equal(out, plain) and abs(w[1].sum().item() - 4) < 1e-4


@pytest.mark.parametrize("form", ["dense", "paged"])
def test_captured_steps_accumulate(form):
    """A captured step replayed with growing lengths gathers what plain calls gather, in place."""
    lens = (640, 30, 9000)
    q, k, v, table, kd = make(lens, 16, 4, 64, form, 10)
    k.nan_to_num_(0.5), v.nan_to_num_(0.5)
    lens_t = torch.tensor([600, 5, 8000], dtype=torch.int32, device="cuda")
    w = [torch.zeros(3, 4, 9010, device="cuda") for _ in range(2)]
    (c0, o0, *_), (c1, o1, *_) = (calls(q, k, v, table, lens_t, (128, 4, True), x, x) for x in w)
    c0()
    w[0].zero_()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c0()
    for step in range(5):
        q.copy_(torch.randn(q.shape, device="cuda"))
        graph.replay()
        c1()
        assert torch.equal(w[0], w[1]) and torch.equal(o0, o1)
        lens_t += torch.tensor([8, 5, 200], dtype=torch.int32, device="cuda")
    assert swaa.last_device_status() == 0
