"""Plain float64 definitions of the operators around the key/value cache, for the tests: no tiling, no online sums, no code shared
with the library."""
import numpy as np

HALF_BF16 = 2.0 ** -8  # half a step of bf16, relative to the value
U32 = 2.0 ** -24       # half a step of fp32


def bf16(x):
    """The nearest bf16 values of an array, as float64 (ties to even)."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def pair_channels(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(y, positions, inv_freq, interleaved, back=False):
    """y [T, H, D] with its first 2 * len(inv_freq) channels rotated by position * inv_freq (back: by the negative)."""
    t = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(inv_freq, dtype=np.float64)
    c, s = np.cos(t), np.sin(t) * (-1 if back else 1)
    a, b = pair_channels(2 * len(inv_freq), interleaved)
    out = y.copy()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def partner(x, rot, interleaved):
    """|x| of the other channel of the pair, 0 for channels that are not rotated."""
    a, b = pair_channels(rot, interleaved)
    out = np.zeros_like(x)
    out[..., a], out[..., b] = np.abs(x[..., b]), np.abs(x[..., a])
    return out


def norm(x, weight, eps):
    """(weight * x / rms, 1 / rms) over the last axis; without a weight x itself."""
    if weight is None:
        return x, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return weight * x * r, r


def qk_rope(x, weight, eps, positions, inv_freq, interleaved):
    """(result, bound of the library's error): x [T, H, D].

    The bound: half a step of bf16 for the store; in fp32 the mean of D squares (in any order at most D roundings, halved by the root),
    the root's 2 ulp, two products, then the rotation's two products and a sum, and an angle and its sine and cosine off by at most
    8 half steps of 1: below (D / 2 + 32) half steps of fp32 of the two channels that enter."""
    y, _ = norm(x, weight, eps)
    z = rotate(y, positions, inv_freq, interleaved)
    rot = 2 * len(inv_freq)
    return z, HALF_BF16 * np.abs(z) + (1 + HALF_BF16) * (x.shape[-1] / 2 + 32) * U32 * (np.abs(y) + partner(y, rot, interleaved))


def qk_rope_backward(x, weight, eps, positions, inv_freq, interleaved, dz):
    """(dx, its bound, dweight, its bound).  The sums over D channels and over tokens and heads may be taken in any order."""
    g = rotate(dz, positions, inv_freq, interleaved, back=True)
    rot, D = 2 * len(inv_freq), dz.shape[-1]
    ga = np.abs(g) + np.abs(dz) + partner(dz, rot, interleaved)  # what enters g
    if weight is None:
        return g, HALF_BF16 * np.abs(g) + 40 * U32 * ga, None, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x * r
    dw = (g * u).sum((0, 1))
    n = x.shape[0] * x.shape[1]
    dw_bound = (n + D / 2 + 48) * U32 * (ga * np.abs(u)).sum((0, 1))
    wg = weight * g
    mean = (wg * u).mean(-1, keepdims=True)
    dx = r * (wg - u * mean)
    scale = r * (np.abs(weight) * ga + np.abs(u) * (np.abs(weight) * ga * np.abs(u)).mean(-1, keepdims=True))
    return dx, HALF_BF16 * np.abs(dx) + (1 + HALF_BF16) * (2 * D + 64) * U32 * scale, dw, dw_bound


def append(q, k, v, qw, kw, eps, inv_freq, interleaved, cu, seqlens, kc, vc, positions=None, table=None, window=0, n_sink=0):
    """Token by token: (q rotated, its bound, written cache rows {(outer, row): token}, k rotated, its bound); kc, vc are only looked at
    for their shapes."""
    pos = np.zeros(q.shape[0], dtype=np.int64)
    rows = {}
    for b in range(len(seqlens)):
        n, m = int(seqlens[b]), int(cu[b + 1] - cu[b])
        for i in range(m):
            e = n - m + i
            pos[cu[b] + i] = e if positions is None else positions[cu[b] + i]
            slot = e if window == 0 or e < n_sink else n_sink + (e - n_sink) % window
            at = (b, slot) if table is None else (int(table[b][slot // kc.shape[1]]), slot % kc.shape[1])
            rows[at] = cu[b] + i  # a later token of the call takes the row
    return (*qk_rope(q, qw, eps, pos, inv_freq, interleaved), rows, *qk_rope(k, kw, eps, pos, inv_freq, interleaved))


def evict(weights, n, budget, n_sink, recent):
    """Indices, ascending, of the entries that stay of one row of n weights: the heaviest first, the lower index first among equals; NaN
    is above every number."""
    if n <= budget:
        return list(range(n))
    j = np.arange(n)
    held = (j < n_sink) | (j >= n - recent)
    rest = j[~held]
    nan = np.isnan(weights[rest])
    order = np.lexsort((rest, -np.where(nan, 0.0, weights[rest]), ~nan))  # by the last key first
    return sorted(j[held].tolist() + rest[order[:budget - int(held.sum())]].tolist())


def visible(i, j, window, n_sink, full):
    return (j <= i) & (full | (j > i - window) | (j < n_sink))


def scores(q, k, scale):
    """(scaled scores [rows, keys], bound of their error): D products of bf16 values, exact in fp32, summed in any order and with any
    rounding of an fp32 sum, then one product with the scale."""
    D = q.shape[-1]
    x = q @ k.T * scale
    return x, (D + 2) * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T) * scale


def softmax_weights(q, k, seen, scale):
    """(p [rows, keys], bound): softmax over the visible keys of every row.  An exponent is off by the score's and the row's
    sum's error and by two fp32 roundings of numbers up to their own size in powers of two; the exponential and the logarithm by 4 half
    steps; the sum of n terms, in any order, by n half steps relative to itself."""
    x, err = scores(q, k, scale)
    x = np.where(seen, x, -np.inf)
    m = x.max(-1, keepdims=True)
    e = np.exp(x - m)
    total = e.sum(-1, keepdims=True)
    p = e / total
    worst = np.where(seen, err, 0).max(-1, keepdims=True)
    size = 4 * 1.45 * (np.abs(np.where(seen, x, 0)).max(-1, keepdims=True) + np.log(total) + 4) * U32
    # below the smallest normal fp32 number, 2^-126, an exponential is 0: the relative error is 1 there, the absolute one below 2^-126
    return p, p * np.expm1(2 * worst + size + (seen.sum(-1, keepdims=True) + 16) * U32) + 2.0 ** -126


def decode_weights(q, k, length, window, n_sink, full, scale):
    """Weights of the entries of one sequence, [Hkv, length], and their bound: q [Hq, D], k [length, Hkv, D]."""
    Hq, Hkv = q.shape[0], k.shape[1]
    G = Hq // Hkv
    seen = np.broadcast_to(visible(length - 1, np.arange(length), window, n_sink, full), (G, length))
    got = [softmax_weights(q[g * G:(g + 1) * G], k[:length, g], seen, scale) for g in range(Hkv)]
    return np.stack([p.sum(0) for p, _ in got]), np.stack([e.sum(0) + (G + 1) * U32 * p.sum(0) for p, e in got])


def key_weights(q, k, lse, i, window, n_sink, full, scale):
    """Weights that the queries at positions i give to the keys 0 .. len(k) - 1 of their sequence, [Hkv, keys], and their bound:
    q [rows, Hq, D], k [keys, Hkv, D], lse [Hq, rows] (natural logarithm, taken as given)."""
    Hq, Hkv = q.shape[1], k.shape[1]
    G, n = Hq // Hkv, k.shape[0]
    seen = visible(np.asarray(i)[:, None], np.arange(n)[None], window, n_sink, full)
    out, bound = np.zeros((Hkv, n)), np.zeros((Hkv, n))
    for h in range(Hq):
        x, err = scores(q[:, h], k[:, h // G], scale)
        x = np.where(seen, x, -np.inf) - lse[h][:, None]
        p = np.exp(x)
        size = 4 * 1.45 * (np.abs(np.where(seen, x, 0)) + 2 * np.abs(lse[h][:, None]) + 4) * U32
        out[h // G] += p.sum(0)
        bound[h // G] += (p * np.expm1(err + size) + 2.0 ** -126).sum(0)  # exponentials below 2^-126 are 0
    return out, bound + (len(i) * G + 16) * U32 * out
