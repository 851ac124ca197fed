"""rr_profile_stop for programs built against an earlier header, whose arrays
hold the kinds that it named."""
import ctypes


def _rr():
    from paper_2609_07306_amd import routerelay
    return routerelay


def test_profile_stop_fills_the_kinds_of_an_earlier_header():
    """Eight kinds before those of the paged cache: their entries are filled,
    and nothing past them is written.  Any other length short of
    RR_KERNEL_KINDS is refused."""
    rr = _rr()
    n = len(rr.KERNEL_KINDS)
    assert rr.KERNEL_KINDS.index("append") == 8
    for size, status in ((7, -1), (8, 0), (9, -1), (n - 1, -1), (n, 0)):
        ms, cnt = (ctypes.c_double * n)(*([-7.0] * n)), (ctypes.c_int64 * n)(*([-7] * n))
        assert rr.lib.rr_profile_start() == 0
        assert rr.lib.rr_profile_stop(ms, cnt, size) == status, size
        filled = size if status == 0 else 0
        assert list(ms) == [0.0] * filled + [-7.0] * (n - filled)
        assert list(cnt) == [0] * filled + [-7] * (n - filled)
    assert rr.lib.rr_profile_stop(None, None, 0) == 0
