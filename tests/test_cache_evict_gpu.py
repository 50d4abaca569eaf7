"""Eviction by weight: which entries stay, in which order, and that their rows and nothing else are copied."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa

pytestmark = pytest.mark.gpu
FILL = 3.0


def weights_of(kind, shape, rng):
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "sparse":  # most keys were never looked at
        w *= rng.random(shape) < 0.1
    elif kind == "ties":
        w = np.round(w)
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "any":  # what a caller may hand in: both signs, both zeros, infinities, NaN, denormals
        w = rng.standard_normal(shape).astype(np.float32)
        for value in (0.0, -0.0, np.inf, -np.inf, np.nan, 1e-42, -1e-42, np.float32(3.4e38)):
            w[rng.random(shape) < 0.03] = value
        w.view(np.uint32)[rng.random(shape) < 0.02] = 0xFFC00001  # a NaN with its sign set
    return w


def run(lens, Hkv, D, budget, n_sink, recent, form="dense", kind="plain", seed=1, extra=0):
    B, L = len(lens), max(max(lens), 1) + extra
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    tables = None
    if form == "paged":
        used, page_out = [-(-n // 64) for n in lens], 128
        blocks_out = -(-budget // page_out)
        order = rng.permutation(sum(used) + 3)
        table = np.full((B, max(max(used), 1) + 1), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = order[at:at + n]
            at += n
        table_out = rng.permutation(B * blocks_out + 2)[:B * blocks_out].reshape(B, blocks_out).astype(np.int32)
        tables = table, table_out
        shape, shape_out, L = (len(order), 64), (B * blocks_out + 2, page_out), table.shape[1] * 64
    else:
        shape, shape_out = (B, L), (B, budget + extra)
    k, v = (torch.randn(*shape, Hkv, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    ko, vo = (torch.full((*shape_out, Hkv, D), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = weights_of(kind, (B, Hkv, L), rng)
    wd = torch.tensor(w, device="cuda")
    wo = torch.full((B, Hkv, budget + extra), FILL, device="cuda")
    kept = torch.full((B, Hkv, budget), -7, dtype=torch.int32, device="cuda")
    n_in, n_out = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda")
    keep = (budget, n_sink, recent)

    def call():
        if form == "paged":
            t, to = (torch.tensor(x, device="cuda") for x in tables)
            swaa.swaa_cache_evict_paged(k, v, wd, n_in, t, *keep, ko, vo, to, wo, kept, n_out)
        else:
            swaa.swaa_cache_evict(k, v, wd, n_in, *keep, ko, vo, wo, kept, n_out)
        assert swaa.last_device_status() == 0

    call()
    assert n_out.tolist() == [min(n, budget) for n in lens]
    kept_h, wo_h = kept.cpu().numpy(), wo.cpu().numpy()
    place = lambda b, j, t, size: (b, j) if tables is None else (tables[t][b, j // size], j % size)
    left = torch.ones((*shape_out, Hkv), dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        m = min(n, budget)
        for h in range(Hkv):
            want = ref.evict(w[b, h], n, *keep)
            assert kept_h[b, h, :m].tolist() == want, (b, h)
            np.testing.assert_array_equal(wo_h[b, h, :m].view(np.uint32), w[b, h, want].view(np.uint32))
            if m:
                src = place(torch.full((m,), b), torch.tensor(want), 0, 64) if tables is None else tuple(torch.tensor(np.array(x)) for x in place(b, np.array(want), 0, 64))
                dst = place(torch.full((m,), b), torch.arange(m), 1, 128) if tables is None else tuple(torch.tensor(np.array(x)) for x in place(b, np.arange(m), 1, 128))
                src, dst = [x.long().cuda() for x in src], [x.long().cuda() for x in dst]
                assert torch.equal(k[src[0], src[1], h], ko[dst[0], dst[1], h]) and torch.equal(v[src[0], src[1], h], vo[dst[0], dst[1], h])
                left[dst[0], dst[1], h] = False
        assert (kept_h[b, :, m:] == -7).all() and (wo_h[b, :, m:] == FILL).all()
    assert (ko[left] == FILL).all() and (vo[left] == FILL).all(), "rows of other entries were written"
    return call


@pytest.mark.parametrize("form", ["dense", "paged"])
@pytest.mark.parametrize("kind", ["plain", "sparse", "ties", "equal", "any"])
@pytest.mark.parametrize("lens,Hkv,D,budget,n_sink,recent", [
    ((300, 17, 64), 2, 64, 64, 4, 16),
    ((1000, 999, 1), 4, 128, 129, 0, 0),
    ((5000,), 1, 64, 4096, 16, 1024),
    ((700, 64, 65), 8, 128, 65, 1, 64),   # nothing to choose between the sinks and the recent entries
])
def test_evict(lens, Hkv, D, budget, n_sink, recent, kind, form):
    run(lens, Hkv, D, budget, n_sink, recent, form, kind, extra=5)


@pytest.mark.parametrize("lens,budget,n_sink,recent", [((0, 1, 2), 1, 0, 0), ((0, 1, 2), 1, 1, 0), ((2, 3, 0), 2, 0, 1), ((40, 41), 40, 0, 40), ((9, 10), 9, 9, 0),
                                                       ((6, 7), 300, 100, 200)])
def test_smallest(lens, budget, n_sink, recent):
    run(lens, 2, 64, budget, n_sink, recent, kind="ties")


@pytest.mark.parametrize("lens,Hkv,budget", [((4097,), 1, 100), ((8193,), 1, 8192), ((33000,), 2, 1111), ((40001, 20), 2, 39999), ((65536,), 1, 5), ((4100,) * 10, 8, 512)])
@pytest.mark.parametrize("kind", ["plain", "sparse", "equal"])
def test_lengths_around_the_shares_of_a_cluster(lens, Hkv, budget, kind):
    run(lens, Hkv, 64, budget, 1 if budget > 5 else 0, 2 if budget > 5 else 0, kind=kind, seed=5)


def test_more_weights_than_shared_memory_holds():
    """150 rows of one block each, 60000 weights: the part beyond 48k is read again from memory."""
    run((60000,) * 3, 50, 64, 64, 4, 8, kind="ties", seed=6)


def test_bad_lengths_and_pages_are_reported():
    B, Hkv, D, N = 3, 2, 64, 8
    mk = lambda *s: torch.randn(*s, Hkv, D, device="cuda").bfloat16()
    k, v, w = mk(B, 64), mk(B, 64), torch.rand(B, Hkv, 64, device="cuda")
    out = lambda *s: torch.full((*s, Hkv, D), FILL, dtype=torch.bfloat16, device="cuda")
    wo, kept, n_out = torch.zeros(B, Hkv, N, device="cuda"), torch.zeros(B, Hkv, N, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    for bad in (-1, 65, 2 ** 31 - 1):
        ko, vo = out(B, N), out(B, N)
        swaa.swaa_cache_evict(k, v, w, torch.tensor([20, bad, 5], dtype=torch.int32, device="cuda"), N, 1, 2, ko, vo, wo, kept, n_out)
        assert swaa.status_str(swaa.last_device_status()) == "SWAA_ERR_BAD_SEQLENS"
        assert n_out.tolist() == [8, 0, 5] and (ko[1] == FILL).all() and torch.equal(ko[2, :5], k[2, :5])
    short = torch.rand(B, Hkv, 30, device="cuda")  # fewer weights than entries
    swaa.swaa_cache_evict(k, v, short, torch.tensor([30, 31, 5], dtype=torch.int32, device="cuda"), N, 1, 2, out(B, N), out(B, N), wo, kept, n_out)
    assert swaa.last_device_status() == -5 and n_out.tolist() == [8, 0, 5]
    table = torch.tensor([[0], [1], [2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([20, 20, 5], dtype=torch.int32, device="cuda")
    for bad in (-1, 3, 2 ** 31 - 1):
        for which in range(2):
            t = [table.clone(), table.clone()]
            t[which][1, 0] = bad
            ko, vo = out(3, 64), out(3, 64)
            swaa.swaa_cache_evict_paged(k, v, w, lens, t[0], N, 1, 2, ko, vo, t[1], wo, kept, n_out)
            assert swaa.last_device_status() == -5
            assert (ko[1] == FILL).all() and torch.equal(ko[2, :5], k[2, :5])


def test_repeats_and_graph():
    call = run((3000, 129), 4, 64, 128, 4, 32, kind="ties", seed=9)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    B, Hkv, D, N = 2, 4, 64, 100
    k, v, w = (torch.randn(B, 900, Hkv, D, device="cuda").bfloat16() for _ in range(2)), None, torch.rand(B, Hkv, 900, device="cuda")
    k, v = k
    lens = torch.tensor([900, 50], dtype=torch.int32, device="cuda")
    outs = [[torch.zeros(B, N, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, N, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hkv, N, device="cuda"),
             torch.zeros(B, Hkv, N, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")] for _ in range(2)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        swaa.swaa_cache_evict(k, v, w, lens, N, 2, 10, *outs[0])
    for step in range(3):
        w.copy_(torch.rand(w.shape, device="cuda"))
        lens.copy_(torch.tensor([900 - 300 * step, 50 + 200 * step], dtype=torch.int32))
        graph.replay()
        swaa.swaa_cache_evict(k, v, w, lens, N, 2, 10, *outs[1])
        for a, b in zip(*outs):
            assert torch.equal(a, b)
    assert swaa.last_device_status() == 0
    call()
