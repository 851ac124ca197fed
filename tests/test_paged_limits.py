"""Sizes at the ends of 32 bits that the paged cache's calls take or refuse,
without a GPU: every one ends at the host's checks."""
import ctypes

import pytest

from test_paged_abi import _paged, _paged_call, _rr

TOP = 2 ** 31 - 1


@pytest.mark.parametrize("n_q,heads,kv", [(TOP, 1, 1), (TOP - 126, 1, 1), (TOP - 127, 1, 1), (TOP // 2 - 60, 2, 2),
                                          (TOP // 7, 7, 1), (TOP // 8 - 1, 8, 2)])
@pytest.mark.parametrize("dtype,cache,d", [(1, 1, 64), (1, 1, 128), (1, 1, 256), (1, 2, 128), (0, 0, 64)])
def test_query_rows_near_2_31(n_q, heads, kv, dtype, cache, d):
    """Up to 2^31 - 1 query rows: the workspace is that of a full launch (512
    workgroups' two parts of 128 rows of d + 4 numbers, and the items' heads of
    a second launch, which a call of that many rows does not take)."""
    rr = _rr()
    scale = 0x1000 if cache == 2 else None
    c = _paged(rr, n_q=n_q, n_heads=heads, n_kv_heads=kv, n_seqs=1, d=d, dtype=dtype, cache_dtype=cache, k_scale=scale,
               v_scale=scale)
    n = rr.lib.rr_paged_workspace_bytes(ctypes.byref(c))
    # (0: refused, where tiles of rows times units of keys pass 2^31)
    assert n == 0 or 2048 < n <= 2048 + 1024 * 128 * (d + 4) * 4
    assert n > 0 or rr.lib.rr_last_error()


def test_units_of_a_launch_stay_below_32_bits():
    """Units of 128 keys (and one for an item's rows) times 1386 key heads:
    2^31 - 2 of them, of which the last runs would end past 32 bits, are
    refused; a page less of each head is taken."""
    rr = _rr()
    for units, ok in ((1549410, False), (1549409, True)):
        c = _paged(rr, n_heads=1386, n_kv_heads=1386, n_seqs=1, page=128, max_pages=units)
        assert (rr.lib.rr_paged_workspace_bytes(ctypes.byref(c)) > 0) is ok
        if not ok:
            assert b"too large" in rr.lib.rr_last_error()
            assert _paged_call(rr, c) == -5
