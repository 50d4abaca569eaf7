"""Attention weights that the keys of a prompt receive, against the float64 definition."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def make(new, ctx, Hq, Hkv, D, seed, paged=False, page=128, pad=0):
    """Packed queries and keys (or pages), random log-sum-exps near those of such scores; keys and log-sum-exps that no query of the
    sequence may use are NaN."""
    g, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    Tq = sum(new)
    q = torch.randn(Tq + pad, Hq, D, generator=g, device="cuda").bfloat16()
    lse = 3 + torch.randn(Hq, Tq + pad, generator=g, device="cuda")
    if pad:
        q[Tq:], lse[:, Tq:] = float("nan"), float("nan")
    ks = [torch.randn(n, Hkv, D, generator=g, device="cuda").bfloat16() for n in ctx]
    cu = lambda x: torch.tensor(np.concatenate([[0], np.cumsum(x)]).astype(np.int32), device="cuda")
    s = {"q": q, "lse": lse, "ks": ks, "cu_q": cu(new), "max_q": max(new), "max_k": max(ctx), "lens": torch.tensor(ctx, dtype=torch.int32, device="cuda")}
    if not paged:
        return {**s, "k": torch.cat([*ks, torch.full((pad, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")]), "cu_k": cu(ctx)}
    used = [-(-n // page) for n in ctx]
    order, at = rng.permutation(sum(used) + 2), 0
    table = np.full((len(ctx), max(used) + 1), -1, dtype=np.int32)
    k = torch.full((len(order), page, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    for b, n in enumerate(ctx):
        for i in range(used[b]):
            table[b, i] = order[at]
            k[order[at], :min(page, n - i * page)] = ks[b][i * page:(i + 1) * page]
            at += 1
    return {**s, "k": k, "table": torch.tensor(table, device="cuda")}


def call(s, w_in, w_out, mask, last=0, scale=0.0, workspace=None):
    B, Hkv, rows = w_out.shape
    Hq = s["q"].shape[1]
    max_k = s["max_k"] if "cu_k" in s else min(s["table"].shape[1] * s["k"].shape[1], rows)
    n = swaa.key_weights_workspace_size(B, s["max_q"], max_k, Hq, Hkv, *mask, last)
    ws = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device="cuda") if workspace is None else workspace  # NaN where it is not written
    if "cu_k" in s:
        swaa.swaa_key_weights(s["q"], s["k"], s["lse"], w_in, w_out, s["cu_q"], s["cu_k"], s["max_q"], s["max_k"], *mask, ws[256:256 + n], last=last, scale=scale)
    else:
        swaa.swaa_key_weights_paged(s["q"], s["k"], s["lse"], w_in, w_out, s["cu_q"], s["lens"], s["table"], s["max_q"], *mask, ws[256:256 + n], last=last, scale=scale)
    assert (ws[:256] == 0xFF).all() and (ws[256 + n:] == 0xFF).all(), "store outside the workspace"


def check(s, new, ctx, w_in, w_out, mask, last, scale):
    at, got = 0, f64(w_out)
    for b, (m, n) in enumerate(zip(new, ctx)):
        r = min(m, last) if last else m
        rows = slice(at + m - r, at + m)
        want, bound = ref.key_weights(f64(s["q"][rows]), f64(s["ks"][b]), f64(s["lse"][:, rows]), np.arange(n - r, n), *mask, scale)
        old = np.zeros_like(want)
        if w_in is not None:
            old[:, :n - m] = f64(w_in)[b, :, :n - m]
        err = np.abs(got[b, :, :n] - old - want)
        bound = bound + 2 * ref.U32 * (old + want)
        assert (err <= bound).all(), (b, np.unravel_index((err - bound).argmax(), err.shape), err.max(), np.nanmax(err / np.maximum(bound, 1e-300)))
        assert (got[b, :, n:] == 9).all(), "entries behind the sequence were written"
        at += m


MASKS = [(2048, 4, True), (100, 4, False), (1, 0, False), (64, 130, False), (300, 0, False), (200, 300, False)]
BATCHES = [((1,), (1,)), ((64,), (64,)), ((65, 1, 128), (65, 1, 128)), ((130, 0, 7), (700, 50, 7)), ((500,), (500,)), ((1, 1, 1), (300, 129, 128))]


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("new,ctx", BATCHES)
@pytest.mark.parametrize("Hq,Hkv,D,last", [(4, 2, 64, 0), (7, 1, 128, 64), (3, 3, 64, 1), (16, 4, 128, 0)])
def test_weights(new, ctx, Hq, Hkv, D, last, mask, paged):
    s = make(new, ctx, Hq, Hkv, D, 3, paged, pad=3)
    w_in = torch.rand(len(new), Hkv, max(ctx) + 5, device="cuda")
    for b, (m, n) in enumerate(zip(new, ctx)):
        w_in[b, :, n - m:n] = float("nan")  # entries of the call's own tokens may hold anything
    w_out = torch.full_like(w_in, 9.0)
    call(s, w_in, w_out, mask, last)
    assert swaa.last_device_status() == 0
    check(s, new, ctx, w_in, w_out, mask, last, D ** -0.5)
    same = w_in.clone()
    call(s, same, same, mask, last)
    fresh = torch.full_like(w_in, 9.0)
    call(s, None, fresh, mask, last)
    assert swaa.last_device_status() == 0
    for b, n in enumerate(ctx):
        assert torch.equal(same[b, :, :n], w_out[b, :, :n])
    check(s, new, ctx, None, fresh, mask, last, D ** -0.5)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("new,ctx,mask,last", [((2500,), (2500,), (9, 9, True), 0), ((2049, 300), (2049, 4000), (9, 9, True), 0), ((5000,), (5000,), (200, 4, False), 0),
                                               ((4200,), (4500,), (3000, 140, False), 0), ((4200,), (4200,), (4000, 4, False), 2100), ((6500,), (6500,), (9, 9, True), 0)])
def test_queries_cut_into_chunks(new, ctx, mask, last, paged):
    s = make(new, ctx, 2, 1, 64, 5, paged)
    w_out = torch.full((len(new), 1, max(ctx) + 1), 9.0, device="cuda")
    call(s, None, w_out, mask, last, scale=0.1)
    assert swaa.last_device_status() == 0
    check(s, new, ctx, None, w_out, mask, last, np.float64(np.float32(0.1)))
    again = torch.full_like(w_out, 9.0)
    call(s, None, again, mask, last, scale=0.1)
    assert torch.equal(again, w_out)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [(9, 9, True), (150, 4, False)])
def test_rows_of_the_prefill_sum_to_one(mask, D):
    """With the log-sum-exps of swaa_prefill every query hands out a weight of 1 per head."""
    lens, Hq, Hkv = (700, 33, 1, 400), 8, 2
    s = make(lens, lens, Hq, Hkv, D, 6)
    v, out = torch.randn_like(s["k"]), torch.empty_like(s["q"])
    swaa.swaa_prefill(s["q"], s["k"], v, out, s["cu_q"], max(lens), *mask, lse=s["lse"])
    w = torch.zeros(4, Hkv, max(lens), device="cuda")
    call(s, None, w, mask)
    assert swaa.last_device_status() == 0
    for b, n in enumerate(lens):
        # the prefill kernel's row sums may use exponentials of relative error 1.0e-4 (a share of them), hence 2e-4
        assert abs(f64(w[b]).sum() / (n * Hq) - 1) < 2e-4


def test_chunks_of_a_prompt_add_up():
    n, Hq, Hkv, D, mask = 900, 8, 2, 64, (200, 4, False)
    s = make((n,), (n,), Hq, Hkv, D, 7)
    whole = torch.full((1, Hkv, n), 9.0, device="cuda")
    call(s, None, whole, mask)
    parts = torch.full_like(whole, float("nan"))
    at = 0
    for m in (256, 1, 300, 343):
        q, lse = s["q"][at:at + m].contiguous(), s["lse"][:, at:at + m].contiguous()
        at += m
        cu = lambda x: torch.tensor([0, x], dtype=torch.int32, device="cuda")
        call({**s, "q": q, "lse": lse, "k": s["k"][:at], "cu_q": cu(m), "cu_k": cu(at), "max_q": m, "max_k": at}, parts, parts, mask)
    assert swaa.last_device_status() == 0
    a, b = f64(whole), f64(parts)
    assert (np.abs(a - b) <= 2 * (n * Hq // Hkv + 16) * ref.U32 * a + 1e-30).all()  # the same terms in another order


def test_scores_beyond_fp32_and_unfinite_keys():
    """A key that is not finite spoils its own weight only; weights below the smallest fp32 number are 0."""
    n, Hq, Hkv, D = 200, 4, 2, 64
    s = make((n,), (n,), Hq, Hkv, D, 8)
    clean = torch.zeros(1, Hkv, n, device="cuda")
    call(s, None, clean, (9, 9, True))
    s["k"][50, 0, 3], s["k"][130, 1, 7] = float("nan"), float("inf")
    w = torch.zeros(1, Hkv, n, device="cuda")
    call(s, None, w, (9, 9, True))
    left = torch.ones_like(w, dtype=torch.bool)
    left[0, 0, 50] = left[0, 1, 130] = False
    assert torch.equal(w[left], clean[left]) and torch.isnan(w[0, 0, 50])
    s["lse"] += 200
    call(s, None, w, (9, 9, True))
    assert (w[left] == 0).all()


def test_bad_lengths_and_pages_are_reported():
    s = make((10, 20, 5), (10, 200, 5), 4, 2, 64, 9)
    w = torch.full((3, 2, 200), 9.0, device="cuda")
    for cu_q, cu_k in (([0, 10, 30, 35], [0, 10, 20, 25]), ([0, 10, 31, 36], [0, 10, 210, 215]), ([0, 10, 5, 10], [0, 10, 210, 215]), ([0, 10, 30, 35], [0, 10, 300, 305])):
        t = {**s, "cu_q": torch.tensor(cu_q, dtype=torch.int32, device="cuda"), "cu_k": torch.tensor(cu_k, dtype=torch.int32, device="cuda")}
        w.fill_(9.0)
        call(t, None, w, (9, 9, True))
        assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
        assert (w[1] == 9).all() and (w[0, :, :10] != 9).any()
    for bounds in (dict(max_q=19), dict(max_k=199)):
        w.fill_(9.0)
        call({**s, **bounds}, None, w, (9, 9, True))
        assert swaa.last_device_status() == -5 and (w[1] == 9).all() and (w[2, :, :5] != 9).any()
    short = torch.full((3, 2, 199), 9.0, device="cuda")
    call(s, None, short, (9, 9, True))
    assert swaa.last_device_status() == -5 and (short[1] == 9).all() and (short[2, :, :5] != 9).any()
    s = make((10, 20), (10, 200), 4, 2, 64, 9, paged=True)
    for bad in (-1, s["k"].shape[0], 2 ** 31 - 1):
        t = s["table"].clone()
        t[1, 1] = bad
        w = torch.full((2, 2, 256), 9.0, device="cuda")
        call({**s, "table": t}, None, w, (9, 9, True))
        assert swaa.last_device_status() == -5
        assert (w[1, :, 128:] == 9).all() and (w[1, :, :128] != 9).any()


def test_no_queries():
    s = make((0, 0), (5, 200), 4, 2, 64, 10)
    w_in, w = torch.rand(2, 2, 201, device="cuda"), torch.full((2, 2, 201), 9.0, device="cuda")
    call(s, w_in, w, (9, 9, True))
    assert torch.equal(w[0, :, :5], w_in[0, :, :5]) and torch.equal(w[1, :, :200], w_in[1, :, :200]) and (w[1, :, 200] == 9).all()
    assert swaa.last_device_status() == 0


def test_graph_and_stream():
    new, ctx, mask = (2100, 60), (2100, 500), (9, 9, True)
    s = make(new, ctx, 4, 2, 128, 11)
    n = swaa.key_weights_workspace_size(2, 2100, 2100, 4, 2, *mask, 0)
    ws, w = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device="cuda"), [torch.zeros(2, 2, 2100, device="cuda") for _ in range(2)]
    run = lambda i: swaa.swaa_key_weights(s["q"], s["k"], s["lse"], w[i], w[i], s["cu_q"], s["cu_k"], 2100, 2100, *mask, ws[256:256 + n])
    run(0)
    w[0].zero_()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        run(0)
    for step in range(3):
        s["q"].copy_(torch.randn(s["q"].shape, device="cuda"))
        graph.replay()
        run(1)
        assert torch.equal(w[0], w[1])
    assert swaa.last_device_status() == 0


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("mask", [(9, 9, True), (300, 130, False), (1000, 0, False)])
@pytest.mark.parametrize("Hq,D,last", [(8, 64, 16), (16, 128, 64), (32, 128, 100), (4, 128, 0)])
def test_blocks_of_several_key_tiles(Hq, D, last, mask, paged):
    """Many sequences of which few queries count: a block goes through several tiles of keys, with its queries in place (up to two steps
    of 128 channels) or loaded again, and past tiles that no query sees."""
    Hkv, B = 4, 40
    ctx = [2000 + 7 * i % 140 for i in range(B)]
    ctx[3], ctx[17], ctx[18] = 1, 129, 1500
    new = list(ctx) if last else [min(n, 1 + i % 60) for i, n in enumerate(ctx)]
    s = make(new, ctx, Hq, Hkv, D, 12, paged)
    w_out = torch.full((B, Hkv, max(ctx) + 3), 9.0, device="cuda")
    call(s, None, w_out, mask, last)
    assert swaa.last_device_status() == 0
    check(s, new, ctx, None, w_out, mask, last, D ** -0.5)
    if paged:  # a bad page in the middle of a run: its keys stay as they are, the others have what they had
        t, before = s["table"].clone(), w_out.clone()
        t[5, 6] = -1
        w_out.fill_(9.0)
        call({**s, "table": t}, None, w_out, mask, last)
        if mask[2]:
            assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
            assert (w_out[5, :, 768:896] == 9).all()
            before[5, :, 768:896] = 9.0
        else:  # none of the last queries sees so far back, and 768 is past the sinks
            assert swaa.last_device_status() == 0
        assert torch.equal(w_out, before)


def test_pages_that_no_query_sees_may_be_gone():
    """Pages before the windows of a call (and without sinks) are not looked up: their keys keep what they had."""
    new, ctx, mask = (70, 9), (1000, 700), (200, 0, False)
    s = make(new, ctx, 8, 2, 64, 13, paged=True)
    w_in = torch.rand(2, 2, 1024, device="cuda")
    want, got = torch.full_like(w_in, 9.0), torch.full_like(w_in, 9.0)
    call(s, w_in, want, mask)
    t = s["table"].clone()
    t[0, :5], t[1, :3] = -1, 10 ** 6  # the first query of sequence 0 is at 930 and sees keys from 731 on, that of sequence 1 from 492 on
    call({**s, "table": t}, w_in, got, mask)
    assert swaa.last_device_status() == 0
    assert torch.equal(got, want) and torch.equal(got[0, :, :640], w_in[0, :, :640])
