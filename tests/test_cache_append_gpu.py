"""Norm, rotation and store into dense, ring and paged caches against the float64 definition."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa
from test_qk_norm_rope_gpu import check, f64, freqs, make

pytestmark = pytest.mark.gpu
EPS = 1e-6
FILL = 3.0


def run(new, ctx, Hq, Hkv, D, rot, form, interleaved=False, norm="qk", positions=False, pad=0, window=0, n_sink=0, seed=3, spare=2):
    new, ctx = list(new), list(ctx)
    T, B = sum(new) + pad, len(new)
    qkv, (qw, kw), f, far = make(T, Hq, Hkv, D, rot, seed, norm)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table = None
    if form == "paged":
        used = [-(-n // 64) for n in ctx]
        order = np.random.default_rng(seed).permutation(sum(used) + spare)
        table = np.full((B, max(max(used), 1) + 1), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = order[at:at + n]
            at += n
        shape = (len(order), 64, Hkv, D)
    else:
        shape = (B, n_sink + window if window else max(max(ctx), 1) + 1, Hkv, D)
    caches = [torch.full((shape[0] + 2, *shape[1:]), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kc, vc = caches[0][1:-1], caches[1][1:-1]
    qo = torch.full((T, Hq, D), FILL, dtype=torch.bfloat16, device="cuda")
    cu_t, lens_t = torch.tensor(cu, device="cuda"), torch.tensor(ctx, dtype=torch.int32, device="cuda")
    pos = far if positions else None
    kw_args = dict(positions=pos, eps=EPS, interleaved=interleaved)
    if form == "paged":
        swaa.swaa_cache_append_paged(q, k, v, qw, kw, f, cu_t, lens_t, torch.tensor(table, device="cuda"), qo, kc, vc, **kw_args)
    else:
        swaa.swaa_cache_append(q, k, v, qw, kw, f, cu_t, lens_t, qo, kc, vc, window=window, n_sink=n_sink, **kw_args)
    assert swaa.last_device_status() == 0
    want_q, bound_q, rows, want_k, bound_k = ref.append(f64(q), f64(k), f64(v), f64(qw), f64(kw), EPS, freqs(f), interleaved, cu, ctx, kc, vc,
                                                        None if pos is None else f64(pos), table, window, n_sink)
    n = int(cu[-1])
    if n:
        check(qo[:n], want_q[:n], bound_q[:n], "q")
    assert (qo[n:] == FILL).all(), "padding rows were written"
    left = torch.ones(shape[:2], dtype=torch.bool, device="cuda")
    if rows:
        outer, row, tok = (torch.tensor(x) for x in zip(*((a, b, t) for (a, b), t in rows.items())))
        check(kc[outer, row], want_k[tok], bound_k[tok], "k")
        assert torch.equal(vc[outer, row], v[tok.cuda()])
        left[outer, row] = False
    assert (kc[left] == FILL).all() and (vc[left] == FILL).all(), "other entries were written"
    for c in caches:
        assert (c[0] == FILL).all() and (c[-1] == FILL).all(), "store outside the cache"


BATCHES = [((1,), (1,)), ((1,) * 5, (1, 64, 65, 300, 17)), ((0, 3, 0, 70, 1, 0), (5, 3, 0, 200, 129, 64)), ((130, 1), (130, 1000)), ((1,) * 70, tuple(range(1, 71)))]


@pytest.mark.parametrize("form", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,D,rot,interleaved,norm", [(4, 2, 64, 64, False, "qk"), (32, 8, 128, 128, False, "qk"), (28, 4, 128, 32, True, "k"), (5, 1, 64, 16, False, "")])
@pytest.mark.parametrize("new,ctx", BATCHES)
def test_append(new, ctx, Hq, Hkv, D, rot, interleaved, norm, form):
    run(new, ctx, Hq, Hkv, D, rot, form, interleaved, norm)


@pytest.mark.parametrize("form", ["dense", "paged"])
def test_positions_padding_and_no_sequence_with_tokens(form):
    run((1, 4, 2), (7, 40, 2), 16, 4, 64, 64, form, positions=True, pad=5)
    run((0, 0), (3, 0), 4, 2, 64, 64, form, pad=3)


@pytest.mark.parametrize("B", [33, 1025, 1500])
def test_many_sequences(B):
    new = [(7 * i) % 3 for i in range(B)]
    run(new, [n + (11 * i) % 50 for i, n in enumerate(new)], 4, 2, 64, 64, "dense", pad=2)


@pytest.mark.parametrize("window,n_sink", [(8, 0), (8, 4), (1, 1), (64, 3)])
@pytest.mark.parametrize("new,ctx", [((1, 1, 1), (1, 5, 300)), ((30, 9, 4), (30, 100, 4)), ((200,), (1000,))])
def test_ring(new, ctx, window, n_sink):
    run(new, ctx, 4, 2, 64, 64, "dense", window=window, n_sink=n_sink)
    for b, n in enumerate(ctx):  # the reference's rows are those of the host function
        assert swaa.trimmed_cache_slot(n - 1, window, n_sink) == (n - 1 if n - 1 < n_sink else n_sink + (n - 1 - n_sink) % window)


def _small(B=2):
    qkv, (qw, kw), f, _ = make(4, 4, 2, 64, 64, 1)
    q, k, v = qkv.split((4, 2, 2), 1)
    return q, k, v, qw, kw, f, torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("lens", [(1, 4), (70, 4), (-1, 4)])
def test_inconsistent_lengths_are_reported(lens):
    """More new tokens than entries, or more entries than rows: nothing of that sequence is written, the other one is."""
    q, k, v, qw, kw, f, cu = _small()
    qo = torch.full((4, 4, 64), FILL, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.full((2, 64, 2, 64), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    swaa.swaa_cache_append(q, k, v, qw, kw, f, cu, torch.tensor(lens, dtype=torch.int32, device="cuda"), qo, kc, vc)
    assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
    assert (qo[:2] == FILL).all() and (kc[0] == FILL).all() and (vc[0] == FILL).all()
    assert (qo[2:] != FILL).any() and torch.equal(vc[1, 2:4], v[2:])


def test_bad_pages_are_reported():
    q, k, v, qw, kw, f, cu = _small()
    qo = torch.full((4, 4, 64), FILL, dtype=torch.bfloat16, device="cuda")
    kp, vp = (torch.full((3, 64, 2, 64), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for bad in (-1, 3, 2 ** 31 - 1):
        table = torch.tensor([[0, bad], [1, 2]], dtype=torch.int32, device="cuda")
        swaa.swaa_cache_append_paged(q, k, v, qw, kw, f, cu, torch.tensor([65, 2], dtype=torch.int32, device="cuda"), table, qo, kp, vp)
        assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
        assert torch.equal(vp[0, 63], v[0]) and (vp[0, :63] == FILL).all() and torch.equal(vp[1, :2], v[2:]) and (vp[2] == FILL).all()


def test_decreasing_cu_stays_in_bounds():
    q, k, v, qw, kw, f, _ = _small()
    qo = torch.full((4, 4, 64), FILL, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.full((3, 64, 2, 64), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for cu in ((0, 3, 1, 4), (2, 3, 4, 4), (0, 9, 9, 9), (-5, 4, 4, 4)):
        swaa.swaa_cache_append(q, k, v, qw, kw, f, torch.tensor(cu, dtype=torch.int32, device="cuda"),
                               torch.tensor([20, 20, 20], dtype=torch.int32, device="cuda"), qo, kc, vc)
        assert swaa.last_device_status() in (0, -5)


def test_graph_replay_follows_the_lengths():
    """One captured append serves every step: lengths and pages are read on the device."""
    B, Hq, Hkv, D = 3, 16, 4, 64
    qkv, (qw, kw), f, _ = make(B, Hq, Hkv, D, D, 4)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    cu, lens = torch.arange(B + 1, dtype=torch.int32, device="cuda"), torch.tensor([1, 63, 64], dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32, device="cuda")
    caches = [torch.zeros(6, 64, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    qo = torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda")
    call = lambda at: swaa.swaa_cache_append_paged(q, k, v, qw, kw, f, cu, lens, table, qo, *caches[at:at + 2])
    call(0)
    caches[0].zero_(), caches[1].zero_()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(0)
    for step in range(3):
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        graph.replay()
        call(2)
        assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
        lens += 1
    assert swaa.last_device_status() == 0
