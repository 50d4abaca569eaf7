"""The operators around a key/value cache whose attention the library computes, as cases that can be timed and compared.

What happens to a key on its way: queries and keys are normalised head by head and rotated by their position as they leave
the projection (`rope`, in training with the gradients: `rope_train`), at serving time in the same pass that writes keys and
values into the cache (`append`); while the cache is read, every key gathers the attention weight that it receives, over a
prompt (`weights`) and with every generated token (`decode`); when the cache outgrows its budget, the entries that gathered least
leave it (`evict`).  Sizes are those of the benchmark's workloads and of the tests, or generic.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
# (query heads, key/value heads)
HEADS = ((4, 2), (16, 4), (32, 8), (28, 4), (64, 8))
RAGGED = "22655,26778,2743,26868,16451,17879,21409,10827"
MAX_FLOPS = {"weights": 5.4e11, "decode": 2.0e10}  # of a drawn case of that kind
MAX_BYTES = 4.4e9


def listed():
    """
    rope_small       the prompt of a small model: launch latency
    rope_long        a 32k prompt, queries, keys and values as slices of one projection's output
    train_packed     forward and backward of short samples packed to one batch, head size 64, half of the channels rotated, in pairs
    train_long       forward and backward of a long fine-tuning sample
    append_tokens    one generated token of each of 16 users into a dense cache
    append_chunks    one step of a serving engine: prompt chunks next to generated tokens, paged cache
    weights_prompt   what every key of a 32k prompt receives under the sliding window, before FA decode over the whole cache
    weights_last     what the last 64 tokens of ragged prompts look at, the usual basis for a first eviction
    decode_one       one user, a token of a small model over the whole cache
    decode_batch     FA decode of a batch at 64k context
    evict_one        one user's paged cache cut to 2048 entries
    evict_batch      a batch of 32k caches cut to 4096 entries each
    """
    packed = "4096,700,1333,2048,3001,511,2500,2195"
    return [
        {"name": "rope_small", "kind": "rope", "lens": "1024", "Hq": 4, "Hkv": 2, "D": 64, "rot": 64, "pairs": False, "norm": True},
        {"name": "rope_long", "kind": "rope", "lens": "32768", "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "pairs": False, "norm": True},
        {"name": "train_packed", "kind": "train", "lens": packed, "Hq": 16, "Hkv": 4, "D": 64, "rot": 32, "pairs": True, "norm": True},
        {"name": "train_long", "kind": "train", "lens": "16384", "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "pairs": False, "norm": True},
        {"name": "append_tokens", "kind": "append", "new": ",".join(["1"] * 16), "ctx": ",".join(str(4000 + 17 * i) for i in range(16)), "page": 0,
         "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "pairs": False, "norm": True},
        {"name": "append_chunks", "kind": "append", "new": "2048,2048,1500,500" + ",1" * 24, "ctx": "2048,16384,31000,500" + "".join(",%d" % (1024 + 331 * i) for i in range(24)),
         "page": 128, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "pairs": False, "norm": True},
        {"name": "weights_prompt", "kind": "weights", "lens": "32768", "last": 0, "Hq": 32, "Hkv": 8, "D": 128, "window": 2048, "n_sink": 4, "full": False, "page": 0},
        {"name": "weights_last", "kind": "weights", "lens": RAGGED, "last": 64, "Hq": 32, "Hkv": 8, "D": 128, "window": 4096, "n_sink": 4, "full": True, "page": 0},
        {"name": "decode_one", "kind": "decode", "lens": "20011", "Lmax": 32768, "page": 0, "Hq": 16, "Hkv": 4, "D": 64, "window": 2048, "n_sink": 4, "full": True},
        {"name": "decode_batch", "kind": "decode", "lens": ",".join(["65536"] * 16), "Lmax": 65536, "page": 0, "Hq": 32, "Hkv": 8, "D": 128, "window": 4096, "n_sink": 4, "full": True},
        {"name": "evict_one", "kind": "evict", "lens": "20011", "Lmax": 20032, "page": 64, "budget": 2048, "n_sink": 4, "recent": 512, "Hkv": 4, "D": 64},
        {"name": "evict_batch", "kind": "evict", "lens": ",".join(["32768"] * 16), "Lmax": 32768, "page": 0, "budget": 4096, "n_sink": 4, "recent": 1024, "Hkv": 8, "D": 128},
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cut(rng: random.Random, total: int, n: int) -> list:
    cuts = sorted(rng.randrange(1, total) for _ in range(n - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total]) if b > a]


def _text(values) -> str:
    return ",".join(map(str, values))


def _one(rng: random.Random) -> dict:
    kind = rng.choice(("rope", "train", "append", "append", "weights", "weights", "decode", "decode", "evict", "evict"))
    Hq, Hkv = rng.choice(HEADS)
    c = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": rng.choice((64, 128, 128))}
    if kind in ("rope", "train", "append"):
        c.update(rot=rng.choice((c["D"], c["D"], c["D"] // 2, c["D"] // 4)), pairs=rng.random() < 0.3, norm=rng.random() < 0.75)
    if kind in ("rope", "train"):
        c["lens"] = _text(_cut(rng, _log_int(rng, 64, 32768 if kind == "rope" else 16384), rng.choice((1, 1, 2, 5, 8))))
    elif kind == "append":
        new = [1] * _log_int(rng, 1, 128) if rng.random() < 0.5 else [_log_int(rng, 1, 2048) for _ in range(rng.randint(1, 6))] + [1] * rng.randint(0, 32)
        c.update(new=_text(new), ctx=_text(n + rng.choice((0, _log_int(rng, 16, 8192))) for n in new), page=rng.choice((0, 64, 128, 256)))
    elif kind == "weights":
        c.update(lens=_text(_cut(rng, _log_int(rng, 256, 32768), rng.choice((1, 1, 2, 5)))), last=rng.choice((0, 0, 16, 64, 100)), page=rng.choice((0, 0, 128, 256)),
                 window=_log_int(rng, 128, 8192), n_sink=rng.choice((0, 4, 4, 64)), full=rng.random() < 0.5)
    else:
        n = _log_int(rng, 1, 32)
        hi = _log_int(rng, 512, 65536)
        lens = [hi if n == 1 or rng.random() < 0.5 else _log_int(rng, max(1, hi // 16), hi) for _ in range(n)]
        page = rng.choice((0, 0, 64, 128))
        c.update(lens=_text(lens), page=page, Lmax=max(lens) + rng.choice((0, 1, 200)) if page == 0 else -(-max(lens) // page) * page)
        if kind == "decode":
            c.update(window=_log_int(rng, 128, 8192), n_sink=rng.choice((0, 4, 4, 64)), full=rng.random() < 0.7)
        else:
            del c["Hq"]
            budget = _log_int(rng, 64, max(128, hi))
            sink = rng.choice((0, 4, 16))
            c.update(budget=budget, n_sink=sink, recent=rng.randint(0, budget - sink))
    return c


def draw(rng: random.Random) -> dict:
    """One more case of the same ranges; one that would cost more than the largest listed one of its kind is drawn again."""
    while True:
        c = _one(rng)
        w = work(c)
        if w["flops"] <= MAX_FLOPS.get(c["kind"], math.inf) and w["bytes"] <= MAX_BYTES and _cache_bytes(c) <= MAX_BYTES:
            return c


# ------------------------------------------------------------------------------------------ lengths
def _ints(text: str) -> list:
    return [int(x) for x in text.split(",")]


def _cache_bytes(c: dict) -> int:
    per = c["Hkv"] * c["D"] * 4
    if c["kind"] == "append":
        ctx = _ints(c["ctx"])
        return per * (len(ctx) * max(ctx) if c["page"] == 0 else sum(ctx))
    if c["kind"] in ("decode", "evict"):
        return per * len(_ints(c["lens"])) * c["Lmax"]
    return 0


def _seen(c: dict, nq: int, nk: int) -> tuple:
    """(visible query/key pairs, keys that some query sees) of the last nq of nk tokens."""
    i = np.arange(nk - nq, nk, dtype=np.int64)
    if c["full"]:
        return int((i + 1).sum()), nk
    before = np.maximum(i + 1 - c["window"], 0)
    first = max(0, nk - nq + 1 - c["window"])
    return int((i + 1 - before + np.minimum(before, c["n_sink"])).sum()), nk - first + min(c["n_sink"], first)


def work(c: dict) -> dict:
    kind, D, Hkv, Hq = c["kind"], c["D"], c["Hkv"], c.get("Hq", 0)
    if kind in ("rope", "train", "append"):
        T = sum(_ints(c["new"] if kind == "append" else c["lens"]))
        qk, v = T * (Hq + Hkv) * D, T * Hkv * D
        if kind != "train":  # in and out; per channel: square, two products and a sum of the rotation, two of the norm
            return {"bytes": 2 * 2 * (qk + v) + 4 * T, "flops": 8 * qk}
        read = 2 * qk if c["norm"] else qk  # the gradient reads the input again where it is normalised
        return {"bytes": 2 * 2 * (qk + v) + 2 * (read + qk + 2 * v) + 8 * T, "flops": 8 * qk + 16 * qk}
    lens = _ints(c["lens"])
    if kind == "weights":
        got = [(min(c["last"] or n, n), *_seen(c, min(c["last"] or n, n), n)) for n in lens]
        rows, pairs, keys = (sum(x) for x in zip(*got))
        return {"bytes": rows * Hq * (2 * D + 4) + keys * Hkv * D * 2 + sum(lens) * Hkv * 4, "flops": (2 * D + 4) * Hq * pairs}
    if kind == "decode":
        pairs, keys = (sum(x) for x in zip(*(_seen(c, 1, n) for n in lens)))
        return {"bytes": keys * Hkv * D * 4 + 2 * sum(lens) * Hkv * 4 + len(lens) * Hq * D * 4, "flops": (4 * D + 8) * Hq * pairs}
    kept = sum(min(n, c["budget"]) for n in lens)
    return {"bytes": sum(lens) * Hkv * 4 + kept * Hkv * (2 * D * 4 + 8), "flops": sum(lens) * Hkv}


# ------------------------------------------------------------------------------------------- inputs
def _randn(gen: torch.Generator, *shape) -> torch.Tensor:
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _int32(values) -> torch.Tensor:
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _packed(lengths) -> torch.Tensor:
    return _int32([0] + np.cumsum(lengths).tolist())


def _empty(*shape) -> torch.Tensor:
    return torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")


def _table(gen: torch.Generator, lengths, page: int) -> tuple:
    """Pages of all sequences in a common pool, in random order: (block table, pages of the pool)."""
    used = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(used), generator=gen, device="cuda").to(torch.int32)
    at = np.concatenate([[0], np.cumsum(used)])
    slot = np.minimum(at[:-1, None] + np.arange(max(used))[None], sum(used) - 1)
    inside = torch.tensor(np.arange(max(used))[None] < np.array(used)[:, None], device="cuda")
    return torch.where(inside, order[torch.tensor(slot, device="cuda")], torch.zeros((), dtype=torch.int32, device="cuda")), sum(used)


def _prepare_rope(c, gen):
    """Slices of one projection's output, as a model has them; weights around 1, a rotation base of 10^6."""
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    lens = _ints(c["new"] if c["kind"] == "append" else c["lens"])
    T = sum(lens)
    s = {"qkv": _randn(gen, T, Hq + 2 * Hkv, D) * 1.5}
    s["q"], s["k"], s["v"] = s["qkv"].split((Hq, Hkv, Hkv), dim=1)
    for name in ("qw", "kw"):
        s[name] = 1 + 0.2 * torch.randn(D, generator=gen, device="cuda") if c["norm"] else None
    s["inv_freq"] = (1e6 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])).float()
    s.update(q_out=_empty(T, Hq, D))
    if c["kind"] != "append":
        s.update(k_out=_empty(T, Hkv, D), v_out=_empty(T, Hkv, D), pos=torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lens]))
    if c["kind"] == "train":
        s.update(dq_out=_randn(gen, T, Hq, D), dk_out=_randn(gen, T, Hkv, D), dv_out=_randn(gen, T, Hkv, D), dqkv=_empty(T, Hq + 2 * Hkv, D))
        s["dq"], s["dk"], s["dv"] = s["dqkv"].split((Hq, Hkv, Hkv), dim=1)
        s.update(dqw=torch.zeros(D, device="cuda") if c["norm"] else None, dkw=torch.zeros(D, device="cuda") if c["norm"] else None)
    return s


def _prepare_append(c, gen):
    s = _prepare_rope(c, gen)
    new, ctx, Hkv, D = _ints(c["new"]), _ints(c["ctx"]), c["Hkv"], c["D"]
    s.update(cu=_packed(new), lens=_int32(ctx))
    if c["page"]:
        s["table"], pages = _table(gen, ctx, c["page"])
        shape = (pages, c["page"], Hkv, D)
    else:
        shape = (len(ctx), max(ctx), Hkv, D)
    s.update(kc=_randn(gen, *shape), vc=_randn(gen, *shape))
    return s


def _visible(qpos, kpos, W: int, S: int, full: bool):
    seen = kpos <= qpos
    return seen if full else seen & ((kpos > qpos - W) | (kpos < S))


def _row_blocks(c, n: int, rows: int):
    """Query rows [a, b) of a sequence of n tokens, and the keys that some of them see: [lo, b) and the sinks before lo."""
    W, S, full = c["window"], c["n_sink"], c["full"]
    for a in range(n - rows, n, 512):
        b = min(a + 512, n)
        lo = 0 if full else max(0, a - W + 1)
        lo = 0 if lo <= S else lo
        keys = torch.arange(lo, b, device="cuda")
        yield a, b, torch.cat([torch.arange(S, device="cuda"), keys]) if lo else keys


def _scores(c, q, k, qpos, kpos):
    """[Hkv, G * rows, keys] scaled scores in 32 bits, and which of them are visible, [rows, keys]."""
    G, n = c["Hq"] // c["Hkv"], q.shape[0]
    qh = q.float().view(n, c["Hkv"], G, c["D"]).permute(1, 2, 0, 3).reshape(c["Hkv"], G * n, c["D"])
    return torch.matmul(qh, k.float().permute(1, 2, 0)) / math.sqrt(c["D"]), _visible(qpos[:, None], kpos[None], c["window"], c["n_sink"], c["full"])


def _prepare_weights(c, gen):
    """Queries, keys, and the log-sum-exp rows that the attention of the prompt has left."""
    lens, Hq, Hkv, D = _ints(c["lens"]), c["Hq"], c["Hkv"], c["D"]
    T, B = sum(lens), len(lens)
    s = {"q": _randn(gen, T, Hq, D), "cu": _packed(lens), "max_len": max(lens)}
    k = _randn(gen, T, Hkv, D)
    at = [0] + np.cumsum(lens).tolist()
    k[at[:-1]] += (torch.randn(Hkv, D, generator=gen, device="cuda") * (3 / math.sqrt(D))).bfloat16()  # first tokens draw attention
    lse = torch.zeros(Hq, T, device="cuda")
    for n, first in zip(lens, at):
        for a, b, keys in _row_blocks(c, n, min(c["last"] or n, n)):
            x, seen = _scores(c, s["q"][first + a:first + b], k[first + keys], torch.arange(a, b, device="cuda"), keys)
            x = x.view(Hq, b - a, -1).masked_fill_(~seen, -math.inf)
            lse[:, first + a:first + b] = torch.logsumexp(x, -1)
    s.update(lse=lse, weights=torch.zeros(B, Hkv, max(lens), device="cuda"))
    if c["page"]:
        s["table"], pages = _table(gen, lens, c["page"])
        s.update(k=_empty(pages, c["page"], Hkv, D), lens=_int32(lens))
        rows = torch.cat([s["table"][b].long().repeat_interleave(c["page"])[:n] * c["page"] + torch.arange(n, device="cuda") % c["page"] for b, n in enumerate(lens)])
        s["k"].view(-1, Hkv, D)[rows] = k
    else:
        s["k"] = k
    return s


def _gathered(gen: torch.Generator, lens: torch.Tensor, Hkv: int, length: int) -> torch.Tensor:
    """Weights as they gather: few large, many small, some keys never looked at."""
    shape = (lens.numel(), Hkv, length)
    w = torch.exp(2 * torch.randn(shape, generator=gen, device="cuda"))
    return w * (torch.rand(shape, generator=gen, device="cuda") > 0.1)


def _prepare_cache(c, gen):
    lens, Hkv, D = _ints(c["lens"]), c["Hkv"], c["D"]
    B = len(lens)
    s = {"lens": _int32(lens)}
    if c["page"]:
        s["table"], pages = _table(gen, lens, c["page"])
        shape = (pages, c["page"], Hkv, D)
    else:
        shape = (B, c["Lmax"], Hkv, D)
    s.update(kc=_randn(gen, *shape), vc=_randn(gen, *shape), w=_gathered(gen, s["lens"], Hkv, c["Lmax"]))
    if c["kind"] == "decode":
        return {**s, "q": _randn(gen, B, c["Hq"], D), "out": _empty(B, c["Hq"], D), "w_out": torch.zeros_like(s["w"])}
    N = c["budget"]
    if c["page"]:
        s["table_out"], pages = _table(gen, [N] * B, c["page"])
        shape = (pages, c["page"], Hkv, D)
    else:
        shape = (B, N, Hkv, D)
    s.update(kc_out=_empty(*shape), vc_out=_empty(*shape), w_out=torch.zeros(B, Hkv, N, device="cuda"))
    s.update(kept=torch.zeros(B, Hkv, N, dtype=torch.int32, device="cuda"), lens_out=torch.zeros(B, dtype=torch.int32, device="cuda"))
    return s


PREPARE = {"rope": _prepare_rope, "train": _prepare_rope, "append": _prepare_append, "weights": _prepare_weights, "decode": _prepare_cache, "evict": _prepare_cache}


def _workspace(c, s):
    """Scratch that a user's program holds for its calls."""
    import paper_2512_10411_b200 as swaa

    nbytes = 0
    if c["kind"] == "train":
        nbytes = swaa.qk_norm_rope_backward_workspace_size(s["q"].shape[0], c["Hq"], c["Hkv"], c["D"])
    elif c["kind"] == "weights":
        nbytes = swaa.key_weights_workspace_size(len(_ints(c["lens"])), s["max_len"], s["max_len"], c["Hq"], c["Hkv"], c["window"], c["n_sink"], c["full"], c["last"])
    elif c["kind"] == "decode":
        nbytes = swaa.decode_weighted_workspace_size(s["q"].shape[0], c["Hq"], c["Hkv"], c["D"], c["Lmax"], c["window"], c["n_sink"], c["full"])
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": dict(case), **PREPARE[case["kind"]](case, gen)}
    if own:
        s["ws"] = _workspace(case, s)
    return s


# ------------------------------------------------------------------------------------- plain forms
def _angles(c, s, pos):
    """cos and sin of position x frequency, 1 and 0 for the channels that are not rotated: [T, 1, D / 2]."""
    a = pos.double()[:, None] * s["inv_freq"].double()
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _rotated(c, x, cos, sin):
    R = c["rot"]
    if c["pairs"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., R:]], -1)
    a, b = x[..., :R // 2], x[..., R // 2:R]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., R:]], -1)


def _unit(x):
    """(x / rms(x), 1 / rms(x)) of every head."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _rope_of(c, x, w, cos, sin):
    return _rotated(c, x.float() if w is None else _unit(x)[0] * w, cos, sin).bfloat16()


def _rope_grads(c, x, w, dy, cos, sin):
    g = _rotated(c, dy.float(), cos, -sin)
    if w is None:
        return g.bfloat16(), None
    u, r = _unit(x)
    dw = (g * u).sum((0, 1), dtype=torch.float64).float()
    g = g * w
    return (r * (g - u * (g * u).mean(-1, keepdim=True))).bfloat16(), dw


def _run_rope(c, s):
    cos, sin = _angles(c, s, s["pos"])
    out = {"q": _rope_of(c, s["q"], s["qw"], cos, sin), "k": _rope_of(c, s["k"], s["kw"], cos, sin), "v": s["v"].contiguous()}
    if c["kind"] == "train":
        dq, dqw = _rope_grads(c, s["q"], s["qw"], s["dq_out"], cos, sin)
        dk, dkw = _rope_grads(c, s["k"], s["kw"], s["dk_out"], cos, sin)
        out["dqkv"] = torch.cat([dq, dk, s["dv_out"]], 1)
        if c["norm"]:
            out.update(dqw=dqw, dkw=dkw)
    return out


def _rows_of(s, seq, at, page: int, length: int):
    """Row of a cache, seen as a list of rows, that holds entry `at` of sequence `seq`."""
    return s["table"][seq, at // page].long() * page + at % page if page else seq * length + at


def _run_append(c, s):
    B = s["lens"].numel()
    t = torch.arange(s["q"].shape[0], device="cuda")
    seq = (t[:, None] >= s["cu"][None, 1:B]).sum(1)
    pos = (t - s["cu"][1:][seq] + s["lens"][seq]).long()
    cos, sin = _angles(c, s, pos)
    rows = _rows_of(s, seq, pos, c["page"], s["kc"].shape[1])
    s["kc"].view(-1, *s["kc"].shape[2:])[rows] = _rope_of(c, s["k"], s["kw"], cos, sin)
    s["vc"].view(-1, *s["vc"].shape[2:])[rows] = s["v"]
    return {"q": _rope_of(c, s["q"], s["qw"], cos, sin), "kc": s["kc"], "vc": s["vc"]}


def _run_weights(c, s):
    """Blocks of 512 query rows, so that the scores fit the card, over the keys that they see; sums of blocks in 64 bits."""
    lens, G = _ints(c["lens"]), c["Hq"] // c["Hkv"]
    out = torch.zeros_like(s["weights"])
    first = 0
    for i, n in enumerate(lens):
        if c["page"]:
            k = s["k"].view(-1, *s["k"].shape[2:])[_rows_of(s, i, torch.arange(n, device="cuda"), c["page"], 0)]
        else:
            k = s["k"][first:first + n]
        total = torch.zeros(c["Hkv"], n, dtype=torch.float64, device="cuda")
        for a, b, keys in _row_blocks(c, n, min(c["last"] or n, n)):
            x, seen = _scores(c, s["q"][first + a:first + b], k[keys], torch.arange(a, b, device="cuda"), keys)
            x = torch.exp(x.view(c["Hkv"], G, b - a, -1) - s["lse"][:, first + a:first + b].view(c["Hkv"], G, b - a, 1)) * seen
            total.index_add_(1, keys, x.sum((1, 2)).double())
        out[i, :, :n] = total.float()
        first += n
    return out


def _run_decode(c, s):
    B, Hkv, D, L = s["lens"].numel(), c["Hkv"], c["D"], c["Lmax"]
    j = torch.arange(L, device="cuda")
    valid = j < s["lens"][:, None]
    if c["page"]:
        rows = torch.where(valid, _rows_of(s, torch.arange(B, device="cuda")[:, None], j[None], c["page"], L), 0)
        k, v = (s[x].view(-1, Hkv, D)[rows] for x in ("kc", "vc"))
    else:
        k, v = s["kc"], s["vc"]
    seen = _visible((s["lens"] - 1)[:, None], j[None], c["window"], c["n_sink"], c["full"])
    q = s["q"].float().view(B, Hkv, -1, D)
    x = torch.matmul(q, k.float().permute(0, 2, 3, 1)) / math.sqrt(D)
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    p = x / x.sum(-1, keepdim=True, dtype=torch.float64).float()
    out = torch.matmul(p, v.float().permute(0, 2, 1, 3)).view(B, -1, D).bfloat16()
    old = torch.where(j < (s["lens"] - 1)[:, None], 1.0, 0.0)[:, None] * s["w"]  # the entry of the token itself starts from 0
    return {"out": out, "weights": torch.where(valid[:, None], old + p.sum(2), 0)}


def _run_evict(c, s):
    B, Hkv, D, L, N = s["lens"].numel(), c["Hkv"], c["D"], c["Lmax"], c["budget"]
    j = torch.arange(L, device="cuda")
    n = s["lens"][:, None]
    held = (j < c["n_sink"]) | (j >= n - c["recent"])
    rank = torch.where((j < n)[:, None], torch.where(held[:, None], math.inf, s["w"]), -math.inf)
    lens = torch.minimum(s["lens"], torch.tensor(N, device="cuda"))
    left = torch.arange(N, device="cuda") < lens[:, None]  # [B, N]
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :N]
    if L < N:
        first = torch.nn.functional.pad(first, (0, N - L))
    kept = torch.where(left[:, None], first, L).sort(-1).values
    kept = torch.where(left[:, None], kept, 0)
    seq = torch.arange(B, device="cuda")
    rows = _rows_of(s, seq[:, None, None], kept, c["page"], L)
    heads = torch.arange(Hkv, device="cuda")[None, :, None]
    out = {"kept": kept.int(), "lens": lens.int(), "weights": torch.where(left[:, None], s["w"].gather(-1, kept), 0)}
    to = torch.arange(N, device="cuda")[None].expand(B, N)
    if c["page"]:
        to = s["table_out"].long().gather(1, to // c["page"]) * c["page"] + to % c["page"]
    else:
        to = seq[:, None] * N + to
    for name in ("kc", "vc"):
        got = s[name].view(-1, Hkv, D)[rows, heads].permute(0, 2, 1, 3)  # [B, N, Hkv, D]
        out[name] = torch.zeros_like(s[name + "_out"])
        out[name].view(-1, Hkv, D)[to.reshape(-1)] = torch.where(left[..., None, None], got, 0).reshape(-1, Hkv, D)
    return out


PLAIN = {"rope": _run_rope, "train": _run_rope, "append": _run_append, "weights": _run_weights, "decode": _run_decode, "evict": _run_evict}


# ------------------------------------------------------------------------------- the framework's calls
def _call(c, s):
    import paper_2512_10411_b200 as swaa

    kind, pairs = c["kind"], c.get("pairs", False)
    if kind in ("rope", "train"):
        swaa.swaa_qk_norm_rope(s["q"], s["k"], s["v"], s["qw"], s["kw"], s["inv_freq"], s["pos"], s["q_out"], s["k_out"], s["v_out"], eps=EPS, interleaved=pairs)
        out = {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
        if kind == "train":
            swaa.swaa_qk_norm_rope_backward(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dv_out"], s["qw"], s["kw"], s["inv_freq"], s["pos"],
                                            s["dq"], s["dk"], s["dv"], s["dqw"], s["dkw"], s["ws"], eps=EPS, interleaved=pairs)
            out["dqkv"] = s["dqkv"]
            if c["norm"]:
                out.update(dqw=s["dqw"], dkw=s["dkw"])
        return out
    if kind == "append":
        if c["page"]:
            swaa.swaa_cache_append_paged(s["q"], s["k"], s["v"], s["qw"], s["kw"], s["inv_freq"], s["cu"], s["lens"], s["table"], s["q_out"], s["kc"], s["vc"], eps=EPS, interleaved=pairs)
        else:
            swaa.swaa_cache_append(s["q"], s["k"], s["v"], s["qw"], s["kw"], s["inv_freq"], s["cu"], s["lens"], s["q_out"], s["kc"], s["vc"], eps=EPS, interleaved=pairs)
        return {"q": s["q_out"], "kc": s["kc"], "vc": s["vc"]}
    if kind == "evict":
        keep = (c["budget"], c["n_sink"], c["recent"])
        if c["page"]:
            swaa.swaa_cache_evict_paged(s["kc"], s["vc"], s["w"], s["lens"], s["table"], *keep, s["kc_out"], s["vc_out"], s["table_out"], s["w_out"], s["kept"], s["lens_out"])
        else:
            swaa.swaa_cache_evict(s["kc"], s["vc"], s["w"], s["lens"], *keep, s["kc_out"], s["vc_out"], s["w_out"], s["kept"], s["lens_out"])
        return {"kept": s["kept"], "lens": s["lens_out"], "weights": s["w_out"], "kc": s["kc_out"], "vc": s["vc_out"]}
    mask = (c["window"], c["n_sink"], c["full"])
    if kind == "weights":
        if c["page"]:
            swaa.swaa_key_weights_paged(s["q"], s["k"], s["lse"], None, s["weights"], s["cu"], s["lens"], s["table"], s["max_len"], *mask, s["ws"], last=c["last"])
        else:
            swaa.swaa_key_weights(s["q"], s["k"], s["lse"], None, s["weights"], s["cu"], s["cu"], s["max_len"], s["max_len"], *mask, s["ws"], last=c["last"])
        return s["weights"]
    if c["page"]:
        swaa.swaa_decode_weighted_paged(s["q"], s["kc"], s["vc"], s["out"], s["w"], s["w_out"], s["table"], s["lens"], *mask, s["ws"])
    else:
        swaa.swaa_decode_weighted(s["q"], s["kc"], s["vc"], s["out"], s["w"], s["w_out"], s["lens"], *mask, s["ws"])
    return {"out": s["out"], "weights": s["w_out"]}


def run(state: dict):
    if own:
        return _call(state["case"], state)
    return PLAIN[state["case"]["kind"]](state["case"], state)


# --------------------------------------------------------------- the operators' definitions in 64 bits
def _exact_turn(c, s, pos) -> torch.Tensor:
    """e^(i angle) of every token and frequency, [T, 1, rot / 2], complex."""
    a = torch.outer(pos.double(), s["inv_freq"].double())
    return torch.polar(torch.ones_like(a), a)[:, None]


def _exact_apply(c, y, turn):
    """Channels that form a pair, as a complex number, times `turn`."""
    y, R = y.clone(), c["rot"]
    at = (slice(0, R, 2), slice(1, R, 2)) if c["pairs"] else (slice(0, R // 2), slice(R // 2, R))
    z = torch.complex(y[..., at[0]], y[..., at[1]]) * turn
    y[..., at[0]], y[..., at[1]] = z.real, z.imag
    return y


def _exact_rope(c, x, w, turn):
    x = x.double()
    return _exact_apply(c, x if w is None else w.double() * x / (x.square().mean(-1, keepdim=True) + EPS).sqrt(), turn)


def _exact_rope_grads(c, x, w, dy, turn):
    g = _exact_apply(c, dy.double(), turn.conj())
    if w is None:
        return g, None
    x = x.double()
    m = x.square().mean(-1, keepdim=True) + EPS
    dw = (g * x / m.sqrt()).sum((0, 1))
    g = g * w.double()
    return g / m.sqrt() - x * (g * x).sum(-1, keepdim=True) / (c["D"] * m * m.sqrt()), dw


def _exact_train(c, s):
    turn = _exact_turn(c, s, s["pos"])
    out = {"q": _exact_rope(c, s["q"], s["qw"], turn), "k": _exact_rope(c, s["k"], s["kw"], turn), "v": s["v"].double()}
    if c["kind"] == "train":
        (dq, dqw), (dk, dkw) = (_exact_rope_grads(c, s[x], s[x + "w"], s["d" + x + "_out"], turn) for x in ("q", "k"))
        out["dqkv"] = torch.cat([dq, dk, s["dv_out"].double()], 1)
        if c["norm"]:
            out.update(dqw=dqw, dkw=dkw)
    return out


def _exact_append(c, s):
    new, ctx = _ints(c["new"]), _ints(c["ctx"])
    turn = _exact_turn(c, s, torch.cat([torch.arange(n - m, n, device="cuda") for m, n in zip(new, ctx)]))
    k, kc, vc = _exact_rope(c, s["k"], s["kw"], turn), s["kc"].double(), s["vc"].double()
    first = 0
    for b, (m, n) in enumerate(zip(new, ctx)):
        for j in range(0, n, c["page"] or n):  # page by page
            page, row, size = (int(s["table"][b, j // c["page"]]), j, c["page"]) if c["page"] else (b, 0, n)
            lo, hi = max(j, n - m), min(j + size, n)
            if lo < hi:
                kc[page, lo - row:hi - row] = k[first + lo - (n - m):first + hi - (n - m)]
                vc[page, lo - row:hi - row] = s["v"][first + lo - (n - m):first + hi - (n - m)].double()
        first += m
    return {"q": _exact_rope(c, s["q"], s["qw"], turn), "kc": kc, "vc": vc}


def _exact_keys(c, s, name: str, b: int, n: int) -> torch.Tensor:
    """The first n entries of sequence b of a dense or paged cache, [n, Hkv, D], in 64 bits."""
    x = s[name]
    if c["page"]:
        return torch.cat([x[p] for p in s["table"][b, :-(-n // c["page"])].tolist()])[:n].double()
    return x[b, :n].double()


def _exact_weights(c, s):
    lens, G, W, S = _ints(c["lens"]), c["Hq"] // c["Hkv"], c["window"], c["n_sink"]
    out = torch.zeros(len(lens), c["Hkv"], max(lens), dtype=torch.float64, device="cuda")
    first = 0
    for b, n in enumerate(lens):
        k = _exact_keys(c, s, "k", b, n) if c["page"] else s["k"][first:first + n].double()
        j = torch.arange(n, device="cuda")
        for h in range(c["Hq"]):
            for a in range(n - min(c["last"] or n, n), n, 4096):
                i = torch.arange(a, min(a + 4096, n), device="cuda")[:, None]
                p = torch.exp(s["q"][first + a:first + a + len(i), h].double() @ k[:, h // G].T * c["D"] ** -0.5 - s["lse"][h, first + a:first + a + len(i), None].double())
                hidden = (j > i) if c["full"] else (j > i) | ((j <= i - W) & (j >= S))
                out[b, h // G, :n] += p.masked_fill(hidden, 0).sum(0)
        first += n
    return out


def _exact_decode(c, s):
    G, D = c["Hq"] // c["Hkv"], c["D"]
    out, weights = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_ints(c["lens"])):
        k, v = _exact_keys(c, s, "kc", b, n), _exact_keys(c, s, "vc", b, n)
        j = torch.arange(n, device="cuda")
        hidden = torch.zeros_like(j, dtype=torch.bool) if c["full"] else (j <= n - 1 - c["window"]) & (j >= c["n_sink"])
        x = torch.einsum("hgd,nhd->hgn", s["q"][b].double().view(-1, G, D), k) * D ** -0.5
        p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
        out[b] = torch.einsum("hgn,nhd->hgd", p, v).reshape(-1, D)
        weights[b, :, :n] = p.sum(1)
        weights[b, :, :n - 1] += s["w"][b, :, :n - 1].double()
    return {"out": out, "weights": weights}


def _exact_evict(c, s):
    N, Hkv = c["budget"], c["Hkv"]
    lens, w = _ints(c["lens"]), s["w"].cpu().numpy()
    kept = np.zeros((len(lens), Hkv, N), dtype=np.int32)
    out = {"kept": None, "lens": _int32([min(n, N) for n in lens]), "weights": torch.zeros(s["w_out"].shape, dtype=torch.float64, device="cuda")}
    for name in ("kc", "vc"):
        out[name] = torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        for h in range(Hkv):
            always = [j for j in range(n) if j < c["n_sink"] or j >= n - c["recent"]] if n > N else range(n)
            rest = np.setdiff1d(np.arange(n), always)
            best = rest[np.lexsort((rest, -w[b, h, rest]))][:N - len(always)] if len(rest) else rest
            kept[b, h, :min(n, N)] = np.sort(np.concatenate([np.array(always, dtype=np.int64), best]))
        at = torch.tensor(kept[b, :, :min(n, N)], device="cuda").long()
        out["weights"][b, :, :at.shape[1]] = s["w"][b].gather(1, at).double()
        for name in ("kc", "vc"):
            rows = _exact_keys(c, s, name, b, n).gather(0, at.T[..., None].expand(-1, -1, c["D"]))
            if c["page"]:
                for p, part in zip(s["table_out"][b].tolist(), rows.split(c["page"])):
                    out[name][p, :len(part)] = part
            else:
                out[name][b, :len(rows)] = rows
    out["kept"] = torch.tensor(kept, device="cuda")
    return out


EXACT = {"rope": _exact_train, "train": _exact_train, "append": _exact_append, "weights": _exact_weights, "decode": _exact_decode, "evict": _exact_evict}


def exact(case: dict, seed: int):
    return EXACT[case["kind"]](case, prepare(case, seed))
