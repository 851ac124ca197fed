"""Sizes at the ends of 32 bits that the paged cache's calls take or refuse,
without a GPU: every one ends at the host's checks."""
import ctypes

import pytest

from test_paged_abi import _append, _append_call, _paged, _paged_call, _rr

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


def test_elements_of_a_token_stay_below_32_bits():
    """A token's rows of keys and queries are 2^30 elements together at most."""
    rr = _rr()
    for heads, kv, q, ok in ((2 ** 20 - 2, 2, True, True), (2 ** 20 - 1, 2, True, False), (2 ** 20 + 7, 2, False, True),
                             (2, 2 ** 20, False, True), (2, 2 ** 20 + 1, False, False), (TOP, TOP, True, False)):
        c = _append(rr, n_heads=heads, n_kv_heads=kv, d=1024, rot=0, n_tokens=0)
        more = {} if q else dict(Q=None, Q_out=None)
        assert _append_call(rr, c, **more) == (0 if ok else -5), (heads, kv, q)
    # (nothing is launched for no tokens; with some a call of that size is refused too)
    assert _append_call(rr, _append(rr, n_heads=2 ** 21, d=1024, rot=0)) == -5
