"""Refusals of the operators around the cache: arguments are looked at on the host, before any device is needed (CPU)."""
import ctypes

import pytest
import torch

import paper_2512_10411_b200 as swaa
from paper_2512_10411_b200.build import build_library

OK, INVALID, UNSUPPORTED, CUDA, WORKSPACE = 0, -1, -2, -3, -4
P = 1 << 20  # an aligned address; nothing here gets as far as to use it


@pytest.fixture(scope="module")
def lib():
    build_library()
    return swaa.load_library()


def needs_device(rc):
    """What a call with sound arguments gives: it went on to the device, and there is none (or it is a B200 and no case here is run there)."""
    return rc in (CUDA, UNSUPPORTED)


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")

ROPE = dict(q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P, rotary_dim=64, interleaved=0,
            positions=P, T=3, Hq=4, Hkv=2, D=64, q_out=P, k_out=P, v_out=P, stream=None)
GRAD = dict(q=P, k=P, q_stride=256, k_stride=128, dq_out=P, dk_out=P, dv_out=P, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P, rotary_dim=64,
            interleaved=0, positions=P, T=3, Hq=4, Hkv=2, D=64, dq=P, dk=P, dv=P, dq_stride=256, dk_stride=128, dv_stride=128, dq_weight=P,
            dk_weight=P, workspace=P, workspace_bytes=1 << 30, stream=None)
APPEND = dict(q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P, rotary_dim=64, interleaved=0,
              positions=None, cu=P, seqlens=P, B=2, Tq=3, Lmax=10, Hq=4, Hkv=2, D=64, window=0, n_sink=0, q_out=P, kcache=P, vcache=P, stream=None)
PAGED = dict(q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P, rotary_dim=64, interleaved=0,
             positions=None, cu=P, seqlens=P, table=P, B=2, Tq=3, max_blocks=4, num_pages=8, page_size=64, Hq=4, Hkv=2, D=64, q_out=P, kpages=P,
             vpages=P, stream=None)

EVICT = dict(k=P, v=P, weights=4 * P, seqlens=5 * P, B=1, Lmax=64, weights_rows=64, Hkv=2, D=64, budget=16, n_sink=4, recent=8, k_out=2 * P, v_out=3 * P,
             Lmax_out=16, weights_out=6 * P, weights_out_rows=16, kept=7 * P, seqlens_out=8 * P, stream=None)
EVICT_PAGED = dict(k=P, v=P, weights=4 * P, seqlens=5 * P, table=9 * P, B=1, max_blocks=1, num_pages=3, page_size=64, weights_rows=64, Hkv=2, D=64, budget=16,
                   n_sink=4, recent=8, k_out=P, v_out=P, table_out=10 * P, max_blocks_out=1, num_pages_out=3, page_size_out=64, weights_out=6 * P,
                   weights_out_rows=16, kept=7 * P, seqlens_out=8 * P, stream=None)
EVICT_COMMON = [(dict(B=-1), INVALID), (dict(budget=0, n_sink=0, recent=0), INVALID), (dict(n_sink=9), INVALID), (dict(recent=-1), INVALID),
                (dict(n_sink=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(weights_out_rows=15), INVALID), (dict(D=80), UNSUPPORTED), (dict(B=65536), UNSUPPORTED),
                (dict(Hkv=0), INVALID), (dict(weights=None), INVALID), (dict(kept=None), INVALID), (dict(kept=7 * P + 1), INVALID), (dict(v=P + 4), INVALID),
                (dict(weights_out=4 * P + 400), INVALID), (dict(seqlens_out=5 * P), INVALID), (dict(weights_rows=0), INVALID), (dict(B=0), OK)]

DECODE = dict(q=P, k=P, v=P, out=P, weights_in=2 * P, weights_out=3 * P, seqlens=P, B=2, Lmax=64, weights_rows=64, Hq=4, Hkv=2, D=64, window=8, n_sink=4,
              is_full=1, scale=0.0, workspace=P, workspace_bytes=1 << 30, stream=None)
DECODE_PAGED = dict(q=P, k=P, v=P, out=P, weights_in=2 * P, weights_out=3 * P, table=P, seqlens=P, B=2, max_blocks=1, num_pages=2, page_size=64, weights_rows=64,
                    Hq=4, Hkv=2, D=64, window=8, n_sink=4, is_full=1, scale=0.0, workspace=P, workspace_bytes=1 << 30, stream=None)
DECODE_COMMON = [(dict(weights_out=None), INVALID), (dict(weights_out=2 * P + 64), INVALID), (dict(weights_in=2 * P + 2), INVALID), (dict(weights_rows=0), INVALID),
                 (dict(B=65536), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(Hq=5), UNSUPPORTED), (dict(window=0, is_full=0), INVALID), (dict(q=None), INVALID),
                 (dict(k=P + 8), INVALID), (dict(n_sink=-1), INVALID), (dict(Hq=8194), UNSUPPORTED), (dict(B=0), OK)]

WEIGHTS = dict(q=P, k=P, lse=P, weights_in=2 * P, weights_out=3 * P, cu_q=P, cu_k=P, B=2, Tq=10, Tk=20, max_q=5, max_k=10, weights_rows=64, Hq=4, Hkv=2, D=64,
               window=8, n_sink=4, is_full=0, scale=0.0, last=0, workspace=P, workspace_bytes=1 << 30, stream=None)
WEIGHTS_PAGED = dict(q=P, k=P, lse=P, weights_in=2 * P, weights_out=3 * P, cu_q=P, seqlens_k=P, table=P, B=2, Tq=10, max_q=5, max_blocks=2, num_pages=3,
                     page_size=128, weights_rows=64, Hq=4, Hkv=2, D=64, window=8, n_sink=4, is_full=0, scale=0.0, last=0, workspace=P, workspace_bytes=1 << 30,
                     stream=None)
WEIGHTS_COMMON = [(dict(weights_out=None), INVALID), (dict(weights_out=2 * P + 64), INVALID), (dict(weights_in=2 * P + 2), INVALID), (dict(weights_rows=0), INVALID),
                  (dict(last=-1), INVALID), (dict(window=0), INVALID), (dict(n_sink=-1), INVALID), (dict(max_q=-1), INVALID), (dict(D=96), UNSUPPORTED), (dict(Hq=5), UNSUPPORTED),
                  (dict(lse=None), INVALID), (dict(lse=P + 2), INVALID), (dict(q=P + 8), INVALID), (dict(k=None), INVALID), (dict(cu_q=None), INVALID),
                  (dict(workspace=None), WORKSPACE), (dict(workspace=P + 128), WORKSPACE), (dict(workspace_bytes=8), WORKSPACE), (dict(B=-1), INVALID),
                  (dict(B=2 ** 30), UNSUPPORTED)]

ROPE_COMMON = [(dict(D=96), UNSUPPORTED), (dict(Hq=5), UNSUPPORTED), (dict(rotary_dim=80), UNSUPPORTED), (dict(rotary_dim=24), UNSUPPORTED),
               (dict(rotary_dim=-16), INVALID), (dict(Hq=0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
               (dict(inv_freq=None), INVALID), (dict(inv_freq=P + 2), INVALID), (dict(q_weight=P + 1), INVALID), (dict(positions=P + 2), INVALID)]


def cases(name, base, extra):
    return [(name, base, change, want) for change, want in extra]


CASES = (
    cases("swaa_qk_norm_rope", ROPE, ROPE_COMMON + [
        (dict(T=-1), INVALID), (dict(q=None), INVALID), (dict(k_out=None), INVALID), (dict(positions=None), INVALID), (dict(v_out=None), INVALID),
        (dict(v=None), INVALID), (dict(q=P + 8), INVALID), (dict(v_out=P + 2), INVALID), (dict(q_stride=252), INVALID), (dict(k_stride=120), INVALID),
        (dict(v_stride=64), INVALID), (dict(T=0), OK)])
    + cases("swaa_qk_norm_rope_backward", GRAD, ROPE_COMMON + [
        (dict(q=None), INVALID), (dict(dq_weight=None), INVALID), (dict(q_weight=None), INVALID), (dict(dv=None), INVALID), (dict(dk=None), INVALID),
        (dict(dq_stride=250), INVALID), (dict(dv_stride=8), INVALID), (dict(workspace=None), WORKSPACE), (dict(workspace=P + 16), WORKSPACE),
        (dict(workspace_bytes=8), WORKSPACE), (dict(dk_weight=P + 2), INVALID), (dict(dq=P + 4), INVALID)])
    + cases("swaa_cache_append", APPEND, ROPE_COMMON + [
        (dict(B=-1), INVALID), (dict(Lmax=0), INVALID), (dict(window=-1), INVALID), (dict(n_sink=-1), INVALID), (dict(window=9, n_sink=2), INVALID),
        (dict(window=2 ** 31 - 1, n_sink=2 ** 31 - 1), INVALID), (dict(v=None), INVALID), (dict(cu=None), INVALID), (dict(seqlens=P + 1), INVALID),
        (dict(kcache=P + 8), INVALID), (dict(v_stride=100), INVALID), (dict(B=0), OK), (dict(Tq=0), OK)])
    + cases("swaa_cache_append_paged", PAGED, ROPE_COMMON + [
        (dict(table=None), INVALID), (dict(page_size=32), UNSUPPORTED), (dict(page_size=0), INVALID), (dict(num_pages=0), INVALID), (dict(max_blocks=0), INVALID),
        (dict(max_blocks=2 ** 26), UNSUPPORTED), (dict(vpages=None), INVALID)])
    + cases("swaa_key_weights", WEIGHTS, WEIGHTS_COMMON + [(dict(cu_k=None), INVALID), (dict(max_k=-1), INVALID), (dict(Tk=-1), INVALID), (dict(B=0), OK),
                                                           (dict(max_k=0), OK), (dict(max_k=2 ** 31 - 1), UNSUPPORTED)])
    + cases("swaa_key_weights_paged", WEIGHTS_PAGED, WEIGHTS_COMMON + [(dict(table=None), INVALID), (dict(page_size=64), UNSUPPORTED), (dict(seqlens_k=None), INVALID)])
    + cases("swaa_decode_weighted", DECODE, DECODE_COMMON + [(dict(Lmax=2 ** 31 - 1), UNSUPPORTED), (dict(Lmax=0), INVALID)])
    + cases("swaa_decode_weighted_paged", DECODE_PAGED, DECODE_COMMON + [(dict(table=None), INVALID), (dict(page_size=32), UNSUPPORTED)])
    + cases("swaa_cache_evict", EVICT, EVICT_COMMON + [(dict(Lmax_out=15), INVALID), (dict(k_out=P + 4096), INVALID), (dict(v_out=P), INVALID), (dict(Lmax=0), INVALID)])
    + cases("swaa_cache_evict_paged", EVICT_PAGED, EVICT_COMMON + [(dict(table_out=None), INVALID), (dict(page_size_out=16), UNSUPPORTED), (dict(num_pages_out=0), INVALID)])
)


@pytest.mark.parametrize("name,base,change,want", CASES, ids=[f"{n}-{c}" for n, _, c, _ in CASES])
def test_refusals(lib, name, base, change, want):
    if "workspace_bytes" in change and not torch.cuda.is_available():
        want = CUDA  # how much it needs goes by the device, which is asked first
    got = getattr(lib, name)(*{**base, **change}.values())
    assert got == want, (swaa.status_str(got), swaa.status_str(want))


@no_gpu
@pytest.mark.parametrize("name,base", [("swaa_qk_norm_rope", ROPE), ("swaa_qk_norm_rope_backward", GRAD), ("swaa_cache_append", APPEND), ("swaa_cache_append_paged", PAGED),
                                       ("swaa_cache_evict", EVICT), ("swaa_cache_evict_paged", EVICT_PAGED), ("swaa_key_weights", WEIGHTS), ("swaa_key_weights_paged", WEIGHTS_PAGED), ("swaa_decode_weighted", DECODE),
                                       ("swaa_decode_weighted_paged", DECODE_PAGED)])
def test_sound_arguments_get_to_the_device(lib, name, base):
    assert needs_device(getattr(lib, name)(*base.values()))


def test_workspace_sizes_of_refused_shapes(lib):
    assert swaa.qk_norm_rope_backward_workspace_size(0, 4, 2, 64) == 256
    assert swaa.qk_norm_rope_backward_workspace_size(10, 4, 2, 80) == 256
    small, large = (swaa.qk_norm_rope_backward_workspace_size(T, 32, 8, 128) for T in (1, 1 << 20))
    assert 0 < small <= large < 1 << 22


def test_binding_refuses_shapes_and_kinds(lib):
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    w, pos, f = torch.ones(64), torch.zeros(3, dtype=torch.int32), torch.ones(32)
    with pytest.raises(TypeError, match="CUDA"):
        swaa.swaa_qk_norm_rope(x, x, x, w, w, f, pos, x, x, x)
    with pytest.raises(TypeError, match="CUDA"):
        swaa.swaa_qk_norm_rope(x, x, x, None, None, None, pos, x, x, x)
    with pytest.raises(ValueError, match="q_weight must be"):
        swaa.swaa_qk_norm_rope(x, x, None, w[:32], w, f, pos, x, x, None)
    with pytest.raises(ValueError, match="inv_freq must be"):
        swaa.swaa_qk_norm_rope(x, x, None, None, None, f[None], pos, x, x, None)
    with pytest.raises(ValueError, match="q must be"):
        swaa.swaa_qk_norm_rope_backward(x[:2], x, x, x, None, None, None, None, pos, x, x, None, None, None, None)
    cu = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="v is needed"):
        swaa.swaa_cache_append(x, x, None, None, None, None, cu, cu[:2], x, x, x)
    with pytest.raises(ValueError, match="seqlens_k"):
        swaa.swaa_cache_append(x, x, x, None, None, None, cu, cu, x, x, x)


def test_key_weights_workspace_grows_with_what_is_cut(lib):
    """Chunks of 16 query tiles of 128; below, a bound for what small calls cut finer (4 x 128 sums per SM), whatever the call.  A workspace
    for longer sequences, more of them or more queries does for less."""
    size = swaa.key_weights_workspace_size
    least = size(3, 9000, 9000, 8, 2, 1000, 4, False, last=64)
    assert least % (4 * 128 * 4) == 0 and least == size(1, 1, 1, 1, 1, 1, 0, True)
    assert size(3, 2049, 90000, 8, 2, 1, 0, True) == 2 * 3 * 2 * 704 * 128 * 4
    assert size(3, 9000, 9000, 8, 2, 1000, 0, False) == least
    assert size(300, 9000, 9000, 8, 2, 1000, 4, False) == 5 * 300 * 2 * 128 * 4
    assert size(0, 9000, 9000, 8, 2, 1000, 4, False) == 256
    for full, window, n_sink in ((True, 1, 0), (False, 300, 4), (False, 2048, 700)):
        for B in (1, 2, 5, 40):
            last = 0
            for n in (1, 70, 128, 500, 1024, 2048, 2100, 4096, 9000, 20000, 70000):
                now = size(B, n, n, 28, 4, window, n_sink, full)
                assert now >= last and size(B, min(n, 64), n, 28, 4, window, n_sink, full) <= now and size(max(B // 2, 1), n, n, 28, 4, window, n_sink, full) <= now
                last = now
