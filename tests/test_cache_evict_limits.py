"""Limits of the eviction that the host checks (CPU): addresses are not real, every call is refused before a launch."""
import pytest

from test_cache_ops_refusals import CUDA, EVICT, EVICT_PAGED, INVALID, UNSUPPORTED, lib, no_gpu  # noqa: F401 (lib: fixture)

MOST = 2 ** 31 - 2 ** 16  # entries of a row that the selection's int steps get through
FAR = 1 << 50             # outputs out of the way of rows that long
LONG = dict(weights_out=FAR, k_out=2 * FAR, v_out=3 * FAR)
LONG_PAGED = dict(weights_out=FAR)


@pytest.mark.parametrize("name,args", [("swaa_cache_evict", {**EVICT, **LONG, "Lmax": n, "weights_rows": n}) for n in (MOST + 1, 2 ** 31 - 1)]
                         + [("swaa_cache_evict_paged", {**EVICT_PAGED, **LONG_PAGED, "max_blocks": 2 ** 25 - 1, "weights_rows": 2 ** 31 - 1})])
def test_rows_too_long_for_the_selection(lib, name, args):  # noqa: F811
    assert getattr(lib, name)(*args.values()) == UNSUPPORTED


@no_gpu
@pytest.mark.parametrize("name,args", [("swaa_cache_evict", {**EVICT, **LONG, "Lmax": MOST, "weights_rows": 2 ** 31 - 1}), ("swaa_cache_evict", {**EVICT, "weights_rows": 2 ** 10, "Lmax": 2 ** 31 - 1, **LONG}),
                                       ("swaa_cache_evict_paged", {**EVICT_PAGED, **LONG_PAGED, "max_blocks": 2 ** 25 - 2 ** 10, "weights_rows": 2 ** 31 - 1})])
def test_longest_rows_get_to_the_device(lib, name, args):  # noqa: F811
    assert getattr(lib, name)(*args.values()) == CUDA  # there is none


@pytest.mark.parametrize("v_out", [EVICT["k_out"], EVICT["k_out"] + 16, EVICT["k_out"] + 16 * 2 * 64 * 2 - 16, EVICT["k_out"] - 16])
def test_new_keys_and_values_share_no_row(lib, v_out):  # noqa: F811
    """16 entries of 2 heads of 64 each: two writers of one row would leave either's bytes."""
    assert lib.swaa_cache_evict(*{**EVICT, "v_out": v_out}.values()) == INVALID


@no_gpu
@pytest.mark.parametrize("by", [1, -1])
def test_new_keys_and_values_may_be_neighbours(lib, by):  # noqa: F811
    assert lib.swaa_cache_evict(*{**EVICT, "v_out": EVICT["k_out"] + by * 16 * 2 * 64 * 2}.values()) == CUDA
