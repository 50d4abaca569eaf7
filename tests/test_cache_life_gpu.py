"""The operators together, as a generation loop uses them: prompt, generated tokens appended and decoded with weights, eviction,
more tokens; each stage against the float64 attention over the keys that are meant to be there."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2512_10411_b200 as swaa

pytestmark = pytest.mark.gpu
HQ, HKV, D, EPS = 8, 2, 64, 1e-6
PROMPTS = (150, 40)
BF = torch.bfloat16


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Layer:
    """One attention layer: norm weights and frequencies; a projection's output is drawn instead of computed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.qw, self.kw = (1 + 0.2 * torch.randn(D, generator=self.g, device="cuda") for _ in range(2))
        self.f = (1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()

    def project(self, T):
        return (torch.randn(T, HQ + 2 * HKV, D, generator=self.g, device="cuda") * 1.3).to(BF)


def split(qkv):
    return qkv.split((HQ, HKV, HKV), 1)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prefill(layer, qkv, lens, mask, last=0, rows=0):
    """(q, k, v of the packed prompts, attention, weights) through norm + rotation, swaa_prefill and swaa_key_weights."""
    T, B = sum(lens), len(lens)
    q, k, v = (torch.empty(T, h, D, dtype=BF, device="cuda") for h in (HQ, HKV, HKV))
    cu, pos = int32(np.concatenate([[0], np.cumsum(lens)]).tolist()), torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lens])
    swaa.swaa_qk_norm_rope(*split(qkv), layer.qw, layer.kw, layer.f, pos, q, k, v, eps=EPS)
    out, lse = torch.empty_like(q), torch.empty(HQ, T, device="cuda")
    swaa.swaa_prefill(q, k, v, out, cu, max(lens), *mask, lse=lse)
    w = torch.full((B, HKV, rows or max(lens)), float("nan"), device="cuda")
    ws = torch.empty(swaa.key_weights_workspace_size(B, max(lens), max(lens), HQ, HKV, *mask, last), dtype=torch.uint8, device="cuda")
    swaa.swaa_key_weights(q, k, lse, None, w, cu, cu, max(lens), max(lens), *mask, ws, last=last)
    assert swaa.last_device_status() == 0
    return q, k, v, out, w


def decode(q, kc, vc, lens, w):
    """swaa_decode_weighted over whole caches, weights gathered in place."""
    out = torch.empty_like(q)
    ws = torch.empty(swaa.decode_weighted_workspace_size(len(lens), HQ, HKV, D, kc.shape[1], 1, 0, True), dtype=torch.uint8, device="cuda")
    swaa.swaa_decode_weighted(q, kc, vc, out, w, w, int32(lens), 1, 0, True, ws)
    assert swaa.last_device_status() == 0
    return out


def attention(q, k, v):
    """float64 attention of one token, q [Hq, D], over k, v [n, Hkv, D], and the weights per kv head."""
    G = HQ // HKV
    x = np.einsum("hgd,nhd->hgn", q.reshape(HKV, G, D), k) * D ** -0.5
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return np.einsum("hgn,nhd->hgd", p, v).reshape(HQ, D), p.sum(1)


def test_generation_with_eviction():
    layer, steps, budget, n_sink, recent = Layer(1), 12, 64, 4, 16
    B, rows = len(PROMPTS), 200
    qkv = layer.project(sum(PROMPTS))
    _, k, v, _, w = prefill(layer, qkv, PROMPTS, (1, 0, True), last=32, rows=rows)
    kc, vc = (torch.full((B, rows, HKV, D), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    at = 0
    for b, n in enumerate(PROMPTS):
        kc[b, :n], vc[b, :n] = k[at:at + n], v[at:at + n]
        at += n
    # what the caches are meant to hold, per sequence and kv head: every key and value ever written, and which of them are left
    every = [[f64(kc[b, :n]), f64(vc[b, :n])] for b, n in enumerate(PROMPTS)]
    left = [[list(range(n)) for _ in range(HKV)] for n in PROMPTS]
    gathered = [[f64(w[b, h, :n]) for h in range(HKV)] for b, n in enumerate(PROMPTS)]
    lens, true = list(PROMPTS), list(PROMPTS)
    for step in range(steps):
        if step in (4, 9):  # over budget again
            new = [torch.full((B, rows, HKV, D), float("nan"), dtype=BF, device="cuda") for _ in range(2)]
            w2, kept, n2 = torch.full_like(w, float("nan")), torch.zeros(B, HKV, budget, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
            swaa.swaa_cache_evict(kc, vc, w, int32(lens), budget, n_sink, recent, *new, w2, kept, n2)
            assert swaa.last_device_status() == 0
            for b in range(B):
                for h in range(HKV):
                    keep = ref.evict(w[b, h].cpu().numpy(), lens[b], budget, n_sink, recent)
                    assert kept[b, h, :len(keep)].tolist() == keep
                    left[b][h] = [left[b][h][j] for j in keep]
                    gathered[b][h] = gathered[b][h][keep]
            (kc, vc), w, lens = new, w2, n2.tolist()
            assert lens == [min(n, budget) for n in (len(left[b][0]) for b in range(B))]
        qkv = layer.project(B)
        q1, k1, v1 = split(qkv)
        lens, true = [n + 1 for n in lens], [n + 1 for n in true]
        q = torch.empty(B, HQ, D, dtype=BF, device="cuda")
        swaa.swaa_cache_append(q1, k1, v1, layer.qw, layer.kw, layer.f, int32(list(range(B + 1))), int32(lens), q, kc, vc, positions=int32([n - 1 for n in true]), eps=EPS)
        out = decode(q, kc, vc, lens, w)
        pos = np.array(true) - 1
        for got, x, wt in ((q, q1, layer.qw), (kc[torch.arange(B), torch.tensor(lens) - 1], k1, layer.kw)):
            want, bound = ref.qk_rope(f64(x), f64(wt), EPS, pos, f64(layer.f), False)
            assert (np.abs(f64(got) - want) <= bound).all()
        for b in range(B):
            every[b] = [np.concatenate([every[b][0], f64(kc[b, lens[b] - 1])[None]]), np.concatenate([every[b][1], f64(v1[b])[None]])]
            for h in range(HKV):
                left[b][h].append(true[b] - 1)
                gathered[b][h] = np.append(gathered[b][h], 0.0)
            kk = np.stack([every[b][0][left[b][h], h] for h in range(HKV)], 1)
            vv = np.stack([every[b][1][left[b][h], h] for h in range(HKV)], 1)
            want, p = attention(f64(q[b]), kk, vv)
            # P in bf16 for the product with V: half a step each of P, the result and, over them, fp32 sums
            bound = 2 * ref.HALF_BF16 * np.einsum("hn,nhd->hd", p, np.abs(vv)).max() + 1e-5
            assert np.abs(f64(out[b]) - want).max() <= bound
            for h in range(HKV):
                gathered[b][h] = gathered[b][h] + p[h]
                # every step adds an error of a few 1e-6 of the weight (scores, exponentials, sum)
                np.testing.assert_allclose(f64(w[b, h, :lens[b]]), gathered[b][h], rtol=2e-4, atol=1e-9)


@pytest.mark.parametrize("paged", [False, True])
def test_generated_tokens_continue_the_prompt(paged):
    """Prompt in chunks and tokens one by one through the cache give what one prefill over everything gives; so do the weights."""
    layer, n, mask = Layer(2), 300, (1, 0, True)
    qkv = layer.project(n)
    q, k, v, want, w_want = prefill(layer, qkv, (n,), mask)
    pages = 3
    kc, vc = (torch.full((pages, 128, HKV, D) if paged else (1, pages * 128, HKV, D), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    table = int32([[2, 0, 1]])
    w = torch.full((1, HKV, pages * 128), float("nan"), device="cuda")
    at = 0
    for m in (130, 1, 120, *[1] * 49):
        part, lens = qkv[at:at + m], int32([at + m])
        at += m
        qo, cu = torch.empty(m, HQ, D, dtype=BF, device="cuda"), int32([0, m])
        common = (*split(part), layer.qw, layer.kw, layer.f, cu, lens)
        if paged:
            swaa.swaa_cache_append_paged(*common, table, qo, kc, vc, eps=EPS)
        else:
            swaa.swaa_cache_append(*common, qo, kc, vc, eps=EPS)
        assert torch.equal(qo, q[at - m:at])  # the same bits as the packed form
        out, lse = torch.empty_like(qo), torch.empty(HQ, m, device="cuda")
        if m == 1:
            size = swaa.decode_weighted_workspace_size(1, HQ, HKV, D, pages * 128, *mask)
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
            if paged:
                swaa.swaa_decode_weighted_paged(qo, kc, vc, out, w, w, table, lens, *mask, ws)
            else:
                swaa.swaa_decode_weighted(qo, kc, vc, out, w, w, lens, *mask, ws)
        else:
            ws = torch.empty(swaa.key_weights_workspace_size(1, m, pages * 128, HQ, HKV, *mask), dtype=torch.uint8, device="cuda")
            if paged:
                swaa.swaa_prefill_paged(qo, kc, vc, out, cu, lens, table, m, *mask, lse=lse)
                swaa.swaa_key_weights_paged(qo, kc, lse, w, w, cu, lens, table, m, *mask, ws)
            else:
                kk, vv = kc[0, :at].contiguous(), vc[0, :at].contiguous()
                swaa.swaa_prefill_chunked(qo, kk, vv, out, cu, int32([0, at]), m, at, *mask, lse=lse)
                swaa.swaa_key_weights(qo, kk, lse, w, w, cu, int32([0, at]), m, at, *mask, ws)
        assert swaa.last_device_status() == 0
        a, b = f64(out), f64(want[at - m:at])
        # both sides: P and the result rounded to bf16
        assert np.abs(a - b).max() <= 4 * ref.HALF_BF16 * np.abs(f64(v)).max()
    # a row's sum in the prefill kernels may be off by 1.0e-4 (exponentials of a share of the columns), as may the weights that go by it
    np.testing.assert_allclose(f64(w[:, :, :n]), f64(w_want), rtol=3e-4, atol=1e-7)


def test_ring_cache_of_a_window_layer():
    """Appending to the ring of a pure-SWA layer and decoding it whole is decoding the untrimmed cache under the window."""
    layer, W, S, B = Layer(3), 32, 4, 3
    start = (1, 30, 36)
    ring = [torch.zeros(B, W + S, HKV, D, dtype=BF, device="cuda") for _ in range(2)]
    full = [torch.zeros(B, 128, HKV, D, dtype=BF, device="cuda") for _ in range(2)]
    lens = [0] * B
    for step in range(80):
        new = list(start) if step == 0 else [1] * B
        lens = [n + m for n, m in zip(lens, new)]
        qkv, cu = layer.project(sum(new)), int32(np.concatenate([[0], np.cumsum(new)]).tolist())
        q = [torch.empty(sum(new), HQ, D, dtype=BF, device="cuda") for _ in range(2)]
        swaa.swaa_cache_append(*split(qkv), layer.qw, layer.kw, layer.f, cu, int32(lens), q[0], *ring, window=W, n_sink=S)
        swaa.swaa_cache_append(*split(qkv), layer.qw, layer.kw, layer.f, cu, int32(lens), q[1], *full)
        assert torch.equal(*q) and swaa.last_device_status() == 0
        last = q[0][(cu[1:] - 1).long()].contiguous()
        out = [torch.empty_like(last) for _ in range(2)]
        trimmed = [swaa.trimmed_cache_len(n, W, S) for n in lens]
        for o, (kc, vc), n, mask in ((out[0], ring, trimmed, (1, 0, True)), (out[1], full, lens, (W, S, False))):
            ws = torch.empty(swaa.decode_workspace_size(B, HQ, HKV, D, kc.shape[1], *mask), dtype=torch.uint8, device="cuda")
            swaa.swaa_decode(last, kc, vc, o, int32(n), *mask, ws)
        assert swaa.last_device_status() == 0
        # the same keys in another order: fp32 sums apart, P and results rounded to bf16 on both sides
        assert np.abs(f64(out[0]) - f64(out[1])).max() <= 4 * ref.HALF_BF16 * f64(full[1]).__abs__().max()


def test_training_step_through_norm_and_rotation():
    """Gradients of norm + rotation + attention against float64 differences of the whole chain."""
    layer, n, W, S = Layer(4), 40, 16, 2
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

    x0, w0, f = f64(qkv), (f64(layer.qw), f64(layer.kw)), f64(layer.f)

    def loss(x, wq, wk):
        a = ref.rotate(ref.norm(x[:, :HQ], wq, EPS)[0], np.arange(n), f, False)
        b = ref.rotate(ref.norm(x[:, HQ:HQ + HKV], wk, EPS)[0], np.arange(n), f, False)
        total = 0.0
        seen = ref.visible(np.arange(n)[:, None], np.arange(n)[None], W, S, False)
        for h in range(HQ):
            s = np.where(seen, a[:, h] @ b[:, h // (HQ // HKV)].T * D ** -0.5, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            total += (p / p.sum(-1, keepdims=True) @ x[:, HQ + HKV + h // (HQ // HKV)] * f64(dout)[:, h]).sum()
        return total

    rng, h = np.random.default_rng(5), 1e-4
    for what, got, scale in (("x", f64(dqkv), 1.0), ("qw", f64(dqw), 1.0), ("kw", f64(dkw), 1.0)):
        errs, size = [], []
        for _ in range(6):  # along random directions: the error of one entry is bf16's, over many it averages
            d = rng.standard_normal(got.shape)
            args = lambda s: (x0 + s * d, *w0) if what == "x" else (x0, w0[0] + s * d, w0[1]) if what == "qw" else (x0, w0[0], w0[1] + s * d)
            errs.append((loss(*args(h)) - loss(*args(-h))) / (2 * h) - (got * d).sum())
            size.append(np.linalg.norm(got))
        # q, k, v, P, dS, dq, dk and the result are rounded to bf16 on the way, half a step each of what they are: at most 8 of them
        # in the 2-norm, and along a random direction of unit variance an error vector of norm e shows with standard deviation e
        assert np.max(np.abs(errs)) <= 4 * 8 * ref.HALF_BF16 * np.mean(size), (what, errs, size)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements: append, decode with weights, eviction, pages and token strides at its far end."""
    Hkv, D, pages = 8, 128, 17200
    L = pages * 128
    assert L * Hkv * D > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(6)
    kc, vc = (torch.zeros(1, L, Hkv, D, dtype=BF, device="cuda") for _ in range(2))
    f = (1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    # append: the last entry, nothing else
    qkv = torch.randn(1, 3 * Hkv, D, generator=g, device="cuda").to(BF)
    q1, k1, v1 = qkv.split((Hkv, Hkv, Hkv), 1)
    q = torch.empty(1, Hkv, D, dtype=BF, device="cuda")
    swaa.swaa_cache_append(q1, k1, v1, None, None, f, int32([0, 1]), int32([L]), q, kc, vc)
    want, bound = ref.qk_rope(f64(k1), None, EPS, np.array([L - 1]), f64(f), False)
    assert (np.abs(f64(kc[:, L - 1]) - want) <= bound).all() and torch.equal(vc[:, L - 1], v1)
    assert not kc[0, :L - 1].any() and not vc[0, :L - 1].any()
    # decode with weights: every other key scores 0
    w = torch.full((1, Hkv, L), float("nan"), device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(swaa.decode_weighted_workspace_size(1, Hkv, Hkv, D, L, 1, 0, True), dtype=torch.uint8, device="cuda")
    swaa.swaa_decode_weighted(q, kc, vc, out, None, w, int32([L]), 1, 0, True, ws)
    assert swaa.last_device_status() == 0
    x = np.einsum("hd,hd->h", f64(q[0]), f64(kc[0, L - 1])) * D ** -0.5
    rest = 1 / (L - 1 + np.exp(x))
    # fp32 row sums of 2.2 million terms, in runs of a block's keys: 1e-4 is above the half steps of the longest run (15000 keys)
    np.testing.assert_allclose(f64(w[0, :, L - 1]), np.exp(x) * rest, rtol=2e-3)
    np.testing.assert_allclose(f64(w[0, :, [0, 1, L // 2, L - 2]]), np.repeat(rest[:, None], 4, 1), rtol=2e-3)
    np.testing.assert_allclose(f64(w[0].double().sum(-1)), 1.0, rtol=2e-3)
    # eviction: entries far apart
    w.zero_()
    at = [5, 1_000_000, L - 70_000, L - 3]
    for i, j in enumerate(at):
        w[0, :, j] = 1.0 + i
        kc[0, j], vc[0, j] = torch.randn(Hkv, D, generator=g, device="cuda").to(BF), torch.randn(Hkv, D, generator=g, device="cuda").to(BF)
    N = 8  # two sinks, two recent entries, those four
    ko, vo, wo = torch.empty(1, N, Hkv, D, dtype=BF, device="cuda"), torch.empty(1, N, Hkv, D, dtype=BF, device="cuda"), torch.empty(1, Hkv, N, device="cuda")
    kept, n_out = torch.empty(1, Hkv, N, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    swaa.swaa_cache_evict(kc, vc, w, int32([L]), N, 2, 2, ko, vo, wo, kept, n_out)
    assert swaa.last_device_status() == 0
    keep = sorted([0, 1, L - 2, L - 1] + at)
    assert kept.tolist() == [[keep] * Hkv] and torch.equal(ko[0], kc[0, keep]) and torch.equal(vo[0], vc[0, keep])
    # pages at both ends of the pool, against the same keys packed
    kp, table = kc.view(pages, 128, Hkv, D), int32([[pages - 1, pages - 2, 0]])
    kp[[pages - 1, pages - 2, 0]] = torch.randn(3, 128, Hkv, D, generator=g, device="cuda").to(BF)
    keys = torch.cat([kp[pages - 1], kp[pages - 2], kp[0]])[:300].contiguous()
    qq, lse = torch.randn(300, 2 * Hkv, D, generator=g, device="cuda").to(BF), 3 + torch.randn(2 * Hkv, 300, generator=g, device="cuda")
    got = [torch.zeros(1, Hkv, 384, device="cuda") for _ in range(2)]
    ws = torch.empty(swaa.key_weights_workspace_size(1, 300, 384, 2 * Hkv, Hkv, 1, 0, True), dtype=torch.uint8, device="cuda")
    swaa.swaa_key_weights_paged(qq, kp, lse, None, got[0], int32([0, 300]), int32([300]), table, 300, 1, 0, True, ws)
    swaa.swaa_key_weights(qq, keys, lse, None, got[1], int32([0, 300]), int32([0, 300]), 300, 300, 1, 0, True, ws)
    assert swaa.last_device_status() == 0 and torch.equal(*got) and got[0].any()
    # tokens more than 2^30 elements apart
    far = kc.view(-1).as_strided((3, Hkv, D), (1_100_000_000, D, 1))
    far.copy_(torch.randn(3, Hkv, D, generator=g, device="cuda"))
    res = [torch.empty(3, Hkv, D, dtype=BF, device="cuda") for _ in range(4)]
    pos = int32([1, 2, 3])
    swaa.swaa_qk_norm_rope(far, far, None, None, None, f, pos, res[0], res[1], None)
    near = far.contiguous()
    swaa.swaa_qk_norm_rope(near, near, None, None, None, f, pos, res[2], res[3], None)
    assert torch.equal(res[0], res[2]) and torch.equal(res[1], res[3])
    swaa.swaa_qk_norm_rope_backward(None, None, near, near, None, None, None, f, pos, far, res[1], None, None, None, None)
    swaa.swaa_qk_norm_rope_backward(None, None, near, near, None, None, None, f, pos, res[2], res[3], None, None, None, None)
    assert torch.equal(far, res[2]) and torch.equal(res[1], res[3]) and swaa.last_device_status() == 0


def test_calls_at_once_on_three_streams():
    """Prefill, key weights, decode with weights, eviction and norm + rotation, overlapping on three streams, give what they give one
    after another."""
    layer, n = Layer(7), 4000
    qkv = layer.project(n)
    q, k, v, _, _ = prefill(layer, qkv, (n,), (500, 4, False))
    cu, lse = int32([0, n]), torch.empty(HQ, n, device="cuda")
    swaa.swaa_prefill(q, k, v, torch.empty_like(q), cu, n, 500, 4, False, lse=lse)
    kc, vc, lens = k[None].contiguous(), v[None].contiguous(), int32([n])
    w_in = torch.rand(1, HKV, n, generator=layer.g, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")

    def work(i):
        """The calls of stream i with buffers of their own: (run, outputs)."""
        out = [torch.zeros_like(q) for _ in range(2)] + [torch.zeros(1, HKV, n, device="cuda") for _ in range(2)]
        ev = [torch.zeros(1, 300, HKV, D, dtype=BF, device="cuda") for _ in range(2)] + [torch.zeros(1, HKV, 300, device="cuda"), torch.zeros(1, HKV, 300, dtype=torch.int32, device="cuda"),
                                                                                         torch.zeros(1, dtype=torch.int32, device="cuda")]
        ro = [torch.zeros_like(x) for x in (q, k, v)]
        ws = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in (swaa.key_weights_workspace_size(1, n, n, HQ, HKV, 500, 4, False),
                                                                         swaa.decode_weighted_workspace_size(1, HQ, HKV, D, n, 1, 0, True))]
        dec = torch.zeros(1, HQ, D, dtype=BF, device="cuda")

        def run(stream):
            for step in range(3):
                for op in range(5):
                    what = (op + i) % 5  # every stream in another order
                    if what == 0:
                        swaa.swaa_prefill(q, k, v, out[0], cu, n, 500, 4, False, stream=stream)
                    elif what == 1:
                        swaa.swaa_key_weights(q, k, lse, None, out[2], cu, cu, n, n, 500, 4, False, ws[0], stream=stream)
                    elif what == 2:
                        swaa.swaa_decode_weighted(q[-1:], kc, vc, dec, w_in, out[3], lens, 1, 0, True, ws[1], stream=stream)
                    elif what == 3:
                        swaa.swaa_cache_evict(kc, vc, w_in, lens, 300, 4, 50, *ev, stream=stream)
                    else:
                        swaa.swaa_qk_norm_rope(*split(qkv), layer.qw, layer.kw, layer.f, pos, *ro, stream=stream)

        return run, [*out, *ev, *ro, dec]

    run, want = work(0)
    run(None)
    assert swaa.last_device_status() == 0
    jobs = [(torch.cuda.Stream(), *work(i)) for i in range(3)]
    torch.cuda.synchronize()
    for stream, run, _ in jobs:
        run(stream)
    torch.cuda.synchronize()
    assert swaa.last_device_status() == 0
    for _, _, got in jobs:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
