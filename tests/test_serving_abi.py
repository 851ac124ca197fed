"""The calls around the paged cache without a GPU: struct layouts, and refusals
of bad sizes, types, strides and pointers before anything is launched, through
the C ABI and through the binding."""
import ctypes

import pytest
import torch

from test_paged_abi import FAKE, ODD, _append

OTHER = ctypes.c_void_p(0x2000)
BF, I32 = torch.bfloat16, torch.int32


def _rr():
    from paper_2609_07306_amd import routerelay
    return routerelay


def test_struct_layouts():
    rr = _rr()
    assert ctypes.sizeof(rr._Axes) == 24 and rr._Axes.real.offset == 20
    assert ctypes.sizeof(rr._RotateConfig) == 64 and rr._RotateConfig.x_token.offset == 32
    assert ctypes.sizeof(rr._PagesConfig) == 40
    assert ctypes.sizeof(rr._VerifyConfig) == 48 and rr._VerifyConfig.p_seq.offset == 16


# ------------------------------------------------------------------ rotate

def _axes(rr, **kw):
    return rr._Axes(*dict(dict(positions=0x1000, axis=0x1000, n_axes=3, real=0), **kw).values())


def _rotate(rr, X=FAKE, freqs=FAKE, axes="some", Y=OTHER, cfg="some", **kw):
    base = dict(n_heads=4, n_tokens=6, d=128, rot=128, interleaved=0, inverse=0, dtype=rr.RR_BF16, reserved=0, x_token=512,
                x_head=128, y_token=512, y_head=128)
    c = rr._RotateConfig(*dict(base, **kw).values()) if cfg else None
    a = _axes(rr) if axes == "some" else axes
    return rr.lib.rr_rotate(c, X, freqs, a, Y, None)


@pytest.mark.parametrize("kw,status", [
    ({"n_heads": 0}, -1), ({"n_tokens": -1}, -1), ({"n_tokens": 1 << 24}, -5), ({"d": 0}, -1), ({"d": 12}, -1),
    ({"d": 1032}, -1), ({"rot": -2}, -1), ({"rot": 130}, -1), ({"rot": 5}, -1), ({"interleaved": 2}, -1), ({"inverse": 2}, -1),
    ({"dtype": 2}, -1), ({"reserved": 1}, -1), ({"x_token": -1}, -1), ({"x_head": -1}, -1), ({"y_token": 127}, -1),
    ({"y_head": 0}, -1), ({"X": None}, -1), ({"Y": None}, -1), ({"freqs": None}, -1), ({"axes": None}, -1), ({"cfg": None}, -1),
    ({"Y": FAKE, "x_token": 640}, -1), ({"Y": FAKE, "x_head": 0}, -1),
    ({"n_tokens": 0, "X": None, "Y": None}, 0),  # nothing to do: nothing is launched
])
def test_rotate_refuses(kw, status):
    rr = _rr()
    assert _rotate(rr, **kw) == status
    assert status == 0 or rr.lib.rr_last_error()


def test_rotate_of_too_many_heads():
    """(shares of them are rounded up in 32 bits)"""
    rr = _rr()
    for heads in (1 << 24, 2 ** 31 - 1):
        assert _rotate(rr, n_heads=heads, x_head=0) == -5
        assert b"n_heads" in rr.lib.rr_last_error()


@pytest.mark.parametrize("kw", [{"n_axes": 0}, {"n_axes": -3}, {"real": 2}, {"positions": None}])
def test_bad_axes(kw):
    rr = _rr()
    assert _rotate(rr, axes=_axes(rr, **kw)) == -1
    c = _append(rr)
    assert rr.lib.rr_cache_append_axes(c, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, _axes(rr, **kw), FAKE, FAKE, OTHER, None) == -1
    assert rr.lib.rr_last_error()


def test_append_by_axes_refuses_what_the_append_does():
    rr = _rr()
    for kw, status in (({"d": 12}, -1), ({"rot": 130}, -1), ({"n_tokens": 1 << 24}, -5), ({"ldk": -1}, -1)):
        c = _append(rr, **kw)
        assert rr.lib.rr_cache_append_axes(c, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, _axes(rr), FAKE, FAKE, OTHER, None) == status


# ------------------------------------------------------------------- pages

def test_fork_refuses():
    rr = _rr()
    base = dict(n_seqs=4, max_pages=8, n_pages=100, parent=FAKE, table=FAKE, lengths=FAKE, refs=FAKE, stream=None)

    def call(**kw):
        return rr.lib.rr_cache_fork(*dict(base, **kw).values())

    for kw in ({"n_seqs": 0}, {"max_pages": 0}, {"n_pages": 0}, {"parent": None}, {"table": None}, {"lengths": None},
               {"refs": None}):
        assert call(**kw) == -1, kw
        assert rr.lib.rr_last_error()
    assert call(n_seqs=4097) == -5 and call(max_pages=1 << 24) == -5


PAGES = dict(n_kv_heads=2, d=128, page=16, n_pages=100, cache_dtype=1, n_pools=3, max_pages=8, n_seqs=4, n_new=1, reserved=0)


def _pages_call(rr, compact, cfg="some", pools=(0x1000, 0x2000, 0x3000), lengths=FAKE, table=FAKE, refs=FAKE, ids=FAKE,
                used=FAKE, ws=FAKE, size=1 << 40, **kw):
    c = rr._PagesConfig(*dict(PAGES, **kw).values()) if cfg else None
    p = None if pools is None else (ctypes.c_void_p * len(pools))(*pools)
    if compact:
        return rr.lib.rr_cache_compact(c, p, table, refs, ids, used, ws, size, None)
    return rr.lib.rr_cache_resize(c, p, None, lengths, table, refs, None, ws, size, None)


@pytest.mark.parametrize("compact", [False, True])
@pytest.mark.parametrize("kw,status", [
    ({"cfg": None}, -1), ({"n_kv_heads": 0}, -1), ({"d": 4}, -1), ({"d": 2048}, -1), ({"page": 0}, -1), ({"n_pages": 0}, -1),
    ({"n_pages": (1 << 28) + 1}, -1), ({"cache_dtype": 3}, -1), ({"n_pools": 0}, -1), ({"n_pools": 4097}, -1),
    ({"max_pages": 0}, -1), ({"max_pages": 1 << 27}, -1), ({"n_seqs": 0}, -1), ({"n_new": -1}, -1), ({"reserved": 1}, -1),
    ({"n_kv_heads": 1 << 18, "page": 1 << 9}, -5), ({"n_kv_heads": 2 ** 31 - 1}, -5),
    ({"n_seqs": 1 << 17, "max_pages": 1 << 14}, -5), ({"pools": None}, -1), ({"pools": (0x1000, 0, 0x3000)}, -1),
    ({"pools": (0x1000, 0x2008, 0x3000)}, -1), ({"table": None}, -1), ({"refs": None}, -1), ({"ws": None}, -1), ({"ws": ODD}, -1),
    ({"size": 0}, -1),
])
def test_resize_and_compact_refuse(compact, kw, status):
    rr = _rr()
    assert _pages_call(rr, compact, **kw) == status
    assert rr.lib.rr_last_error()


@pytest.mark.parametrize("compact", [False, True])
def test_tables_past_the_count_of_rounds(compact):
    """Entries are counted on in rounds of 1024, in 32 bits: the largest tables
    that 31 bits hold leave that count no room."""
    rr = _rr()
    for n_seqs, max_pages in ((1 << 16, 1 << 14), (2 ** 31 - 1, 1), (127, 2 ** 24)):
        assert _pages_call(rr, compact, n_seqs=n_seqs, max_pages=max_pages, page=1) == -5
        assert b"2^30" in rr.lib.rr_last_error()


def test_pages_workspace():
    rr = _rr()
    assert _pages_call(rr, False, lengths=None) == -1
    assert _pages_call(rr, True, ids=None) == -1 and _pages_call(rr, True, used=None) == -1
    for n in (0, -1, (1 << 28) + 1):
        assert rr.lib.rr_pages_workspace_bytes(n) == 0 and rr.lib.rr_last_error()
    need = rr.lib.rr_pages_workspace_bytes(100)
    assert 1200 <= need < 2048
    for compact in (False, True):
        assert _pages_call(rr, compact, size=need - 1) == -1
        assert b"workspace" in rr.lib.rr_last_error()
    assert rr.lib.rr_pages_workspace_bytes(1 << 28) > 12 << 28


# ------------------------------------------------------------------ drafts

def _verify(rr, cfg="some", P=FAKE, Q=FAKE, drafts=FAKE, u=FAKE, accepted=FAKE, tokens=FAKE, ws=FAKE, size=1 << 40, **kw):
    base = dict(n_seqs=4, n_drafts=3, vocab=1000, dtype=0, p_seq=4000, p_row=1000, q_seq=3000, q_row=1000)
    c = rr._VerifyConfig(*dict(base, **kw).values()) if cfg else None
    return c, rr.lib.rr_verify_drafts(c, P, Q, drafts, None, u, None, accepted, tokens, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    ({"cfg": None}, -1), ({"n_seqs": 0}, -1), ({"n_drafts": -1}, -1), ({"n_drafts": (1 << 20) + 1}, -1), ({"vocab": 0}, -1),
    ({"vocab": 1 << 24}, -5), ({"dtype": 2}, -1), ({"p_seq": -1}, -1), ({"p_row": -1}, -1), ({"q_seq": -1}, -1),
    ({"q_row": -1}, -1), ({"P": None}, -1), ({"drafts": None}, -1), ({"u": None}, -1), ({"accepted": None}, -1),
    ({"tokens": None}, -1), ({"ws": None}, -1), ({"ws": ODD}, -1), ({"size": 0}, -1),
])
def test_verify_refuses(kw, status):
    rr = _rr()
    c, got = _verify(rr, **kw)
    assert got == status and rr.lib.rr_last_error()
    if c is not None and any(k in kw for k in ("n_seqs", "n_drafts", "vocab", "dtype", "p_seq", "p_row", "q_seq", "q_row")):
        assert rr.lib.rr_verify_workspace_bytes(c) == 0


def test_verify_workspace():
    rr = _rr()
    assert rr.lib.rr_verify_workspace_bytes(None) == 0
    c, _ = _verify(rr, size=0)
    need = rr.lib.rr_verify_workspace_bytes(c)
    assert need > 65536
    assert _verify(rr, size=need - 1)[1] == -1 and b"workspace" in rr.lib.rr_last_error()
    # bounded however many sequences a call has: they take turns
    many, _ = _verify(rr, n_seqs=2 ** 31 - 1, size=0)
    assert rr.lib.rr_verify_workspace_bytes(many) < 1 << 20


# ----------------------------------------------------------------- binding

def test_binding_checks_tensors():
    """Shapes, types and places that the binding refuses before any call."""
    rr = _rr()
    X, f = torch.zeros((6, 2, 64), dtype=BF), torch.zeros(32, dtype=torch.float64)
    pos = torch.zeros((3, 6), dtype=I32)
    with pytest.raises(ValueError, match="GPU"):
        rr.rotate(X, pos, f)
    with pytest.raises(TypeError):
        rr.rotate(X.half(), pos, f)
    with pytest.raises(ValueError, match="tokens"):
        rr.rotate(X, pos, f, tokens=2)
    pool = torch.zeros((10, 2, 16, 64), dtype=BF)
    table, lens, refs = torch.zeros((2, 4), dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(10, dtype=I32)
    with pytest.raises(ValueError, match="GPU"):
        rr.cache_append(X[:, :2], X[:, :2], pool, pool, table, lens, freqs=f, positions=pos)
    with pytest.raises(ValueError, match="GPU"):
        rr.Pools(pool, pool)
    with pytest.raises(ValueError, match="GPU"):
        rr.Pools([pool, pool], [pool, pool])
    with pytest.raises(ValueError, match="as many"):
        rr.Pools([pool, pool], [pool])
    with pytest.raises(ValueError, match="as many"):
        rr.Pools([], [])
    with pytest.raises(ValueError, match="one shape"):
        rr.Pools(pool, pool[:9])
    with pytest.raises(ValueError, match="one type"):
        rr.Pools(pool, pool.float())
    with pytest.raises(TypeError):
        rr.Pools(pool.half(), pool.half())
    with pytest.raises(TypeError):
        rr.Pools(pool[0], pool[0])
    with pytest.raises(ValueError, match="contiguous"):
        rr.Pools(pool.transpose(0, 1), pool.transpose(0, 1))
    with pytest.raises(ValueError, match="GPU"):
        rr.cache_fork(table, lens, refs, lens)
    P, drafts, u = torch.zeros((2, 4, 50)), torch.zeros((2, 3), dtype=I32), torch.zeros((2, 4))
    with pytest.raises(ValueError, match="GPU"):
        rr.verify_drafts(P, drafts, u)


@pytest.mark.parametrize("kw", [dict(P=(2, 3, 50)), dict(P=(2, 4)), dict(drafts=(2, 3, 1)), dict(uniforms=(2, 3)),
                                dict(uniforms=(3, 4)), dict(draft_probs=(2, 4, 50)), dict(draft_probs=(2, 3, 49)),
                                dict(n_drafts=(3,)), dict(lengths=(1,)), dict(accepted=(2, 1)), dict(tokens=(2, 3)),
                                dict(kind=torch.float16), dict(draft_kind=BF), dict(u_kind=torch.float64)])
def test_verify_binding_checks_shapes(kw, monkeypatch):
    """(With a device made up, as every tensor here is the host's.)"""
    rr = _rr()
    monkeypatch.setattr(rr, "_device_of", lambda tensors: 0)
    shapes = dict(dict(P=(2, 4, 50), drafts=(2, 3), uniforms=(2, 4), draft_probs=(2, 3, 50), n_drafts=(2,), lengths=(2,),
                       accepted=(2,), tokens=(2, 4)), **kw)
    types = dict(P=kw.get("kind", torch.float32), uniforms=kw.get("u_kind", torch.float32),
                 draft_probs=kw.get("draft_kind", torch.float32))
    t = {k: torch.zeros(s, dtype=types.get(k, I32)) for k, s in shapes.items() if not k.endswith("kind")}
    monkeypatch.setattr(rr, "_launch", lambda *a: pytest.fail("launched"))
    with pytest.raises((ValueError, TypeError)):
        rr.verify_drafts(t["P"], t["drafts"], t["uniforms"], **{k: t[k] for k in ("draft_probs", "n_drafts", "lengths",
                                                                                  "accepted", "tokens")},
                         workspace=torch.zeros(1 << 17, dtype=torch.uint8))


@pytest.mark.parametrize("kw", [dict(positions=(3, 5)), dict(positions=(2, 3, 6)), dict(positions=(0, 6)),
                                dict(axis=(31,)), dict(kind=torch.int64), dict(axis_kind=torch.int64), dict(out=(6, 2, 32)),
                                dict(freqs_kind=torch.float32), dict(out_kind=torch.float32)])
def test_rotate_binding_checks_shapes(kw, monkeypatch):
    rr = _rr()
    monkeypatch.setattr(rr, "_device_of", lambda tensors: 0)
    monkeypatch.setattr(rr, "_launch", lambda *a: pytest.fail("launched"))
    t = dict(positions=torch.zeros(kw.get("positions", (3, 6)), dtype=kw.get("kind", I32)),
             axis=torch.zeros(kw.get("axis", (32,)), dtype=kw.get("axis_kind", I32)),
             freqs=torch.zeros(32, dtype=kw.get("freqs_kind", torch.float64)),
             out=torch.zeros(kw.get("out", (6, 2, 64)), dtype=kw.get("out_kind", BF)))
    with pytest.raises((ValueError, TypeError)):
        rr.rotate(torch.zeros((6, 2, 64), dtype=BF), **t)


def test_profile_stop_fills_the_kinds_of_the_header_before():
    """Eleven kinds before those of rows, drafts and pages: their entries alone."""
    rr = _rr()
    n = len(rr.KERNEL_KINDS)
    assert rr.KERNEL_KINDS.index("rotate") == 11
    ms, cnt = (ctypes.c_double * n)(*([-7.0] * n)), (ctypes.c_int64 * n)(*([-7] * n))
    assert rr.lib.rr_profile_start() == 0
    for size in (10, 12, n - 1):
        assert rr.lib.rr_profile_stop(ms, cnt, size) == -1
    assert rr.lib.rr_profile_stop(ms, cnt, 11) == 0
    assert list(ms) == [0.0] * 11 + [-7.0] * (n - 11) and list(cnt) == [0] * 11 + [-7] * (n - 11)


@pytest.mark.parametrize("shape,n,fits", [((), 0, False), ((), 1, False), ((0,), 0, True), ((0,), 4, False), ((3, 0), 0, True),
                                          ((0, 4), 4, False), ((4,), 4, True), ((3, 4), 4, True), ((4, 3), 4, False),
                                          ((1, 3, 4), 4, False)])
def test_shapes_of_positions(shape, n, fits):
    """One axis without a dimension of its own, or some; no tokens are none to place."""
    rr = _rr()
    positions = torch.zeros(shape, dtype=torch.int32)
    if fits:
        axes = rr._axes_of(positions, None, 4, n)
        assert axes.n_axes == (shape[0] if len(shape) == 2 else 1)
    else:
        with pytest.raises(ValueError, match="positions must be"):
            rr._axes_of(positions, None, 4, n)


def test_a_verification_s_workspace_serves_smaller_ones():
    """Fewer sequences, a smaller vocabulary (whose rows may have more parts) and
    the shorter type need no more bytes."""
    rr = _rr()

    def need(n_seqs, vocab, dtype):
        return rr.lib.rr_verify_workspace_bytes(rr._VerifyConfig(n_seqs, 3, vocab, dtype, 0, 0, 0, 0))

    edges = [e + x for k in range(24) for e in (1 << k, 3 << k) for x in (-1, 0, 1)]
    sizes = sorted({v for v in edges + [1000, 32000, 50257, 128256, 151936, 262144, 300001] if 1 <= v < 1 << 24})
    for n_seqs in (1, 7, 1024, 5000):
        for dtype in (rr.RR_F32, rr.RR_BF16):
            got = [need(n_seqs, v, dtype) for v in sizes]
            assert got == sorted(got) and got[0] > 65536
    for v in sizes:
        assert need(7, v, rr.RR_BF16) <= need(7, v, rr.RR_F32) <= need(8, v, rr.RR_F32)


def test_rotate_refuses_rows_that_overlap():
    """Each element of Y is of one row at most: against the rows laid out (where they
    are not, no tokens or a NULL pointer ends the call before anything is launched)."""
    rr = _rr()
    d = 8
    for tokens in (1, 2, 3, 5):
        for heads in (1, 2, 4):
            for y_token in range(d, 5 * d + 2):
                for y_head in range(d, 5 * d + 2, 1 if tokens * heads < 9 else 3):
                    at = [i * y_token + h * y_head + e for i in range(tokens) for h in range(heads) for e in range(d)]
                    status = _rotate(rr, X=None, n_tokens=tokens, n_heads=heads, d=d, rot=d, y_token=y_token, y_head=y_head)
                    assert status == -1
                    overlap = b"overlap" in rr.lib.rr_last_error()
                    assert overlap == (len(set(at)) < len(at)), (tokens, heads, y_token, y_head)
    # the largest calls: one after the other, and shifted by less than a row
    many = (1 << 24) - 1
    for y_token, y_head, overlap in ((128, 128 * many, False), (128 * many, 128, False), (128, 128 * many - 1, True),
                                     (1 << 62, 1 << 62, True), ((1 << 62) - 64, 1 << 62, True), (129, 129 * 2, True)):
        assert _rotate(rr, X=None, n_tokens=many, n_heads=many, y_token=y_token, y_head=y_head) == -1
        assert (b"overlap" in rr.lib.rr_last_error()) == overlap, (y_token, y_head)
