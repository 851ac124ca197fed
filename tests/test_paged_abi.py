"""The paged cache's C ABI without a GPU: where tokens lie (the kernels' index
arithmetic compiled for the host, bad pages among its cases), struct layouts,
and refusals of bad sizes, types and pointers before anything is launched."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FAKE = ctypes.c_void_p(0x1000)  # never dereferenced
ODD = ctypes.c_void_p(0x1008)


def _rr():
    from paper_2609_07306_amd import routerelay
    return routerelay


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_index_arithmetic_is_exact(tmp_path):
    exe = str(tmp_path / "paged")
    r = subprocess.run([HIPCC, "-O2", "-std=c++17", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
                        "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2609_07306_amd", "csrc"),
                        "-o", exe, os.path.join(ROOT, "tests", "sanitize", "paged_driver.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and "paged driver ok" in out.stdout, out.stdout[-300:] + out.stderr[-300:]
    n = {}
    for line in out.stdout.splitlines():
        f = line.split()
        n[f[0]] = n.get(f[0], 0) + 1
        if f[0] == "div":
            assert int(f[3]) == int(f[1]) // int(f[2]), line
        elif f[0] == "page":
            assert int(f[3]) == (int(f[1]) if 0 <= int(f[1]) < int(f[2]) else -1), line
        elif f[0] == "row":
            phys, kv, g, page, place, d = (int(x) for x in f[1:7])
            assert int(f[7]) == ((phys * kv + g) * page + place) * d, line
        elif f[0] == "held":
            assert int(f[3]) == min(max(int(f[1]), 0), int(f[2])), line
        elif f[0] == "seq":
            i, got, start = int(f[1]), int(f[2]), [int(x) for x in f[4:]]
            own = [b for b in range(len(start) - 1) if start[b] <= i < start[b + 1]]
            assert [got] == (own or [-1]), line
    assert n["div"] > 8000 and n["seq"] > 1000 and n["row"] == 200


def test_struct_layouts():
    rr = _rr()
    assert ctypes.sizeof(rr._AppendConfig) == 88 and rr._AppendConfig.ldq.offset == 48
    assert rr._AppendConfig.k_scale.offset == 72
    assert ctypes.sizeof(rr._PagedConfig) == 80 and rr._PagedConfig.scale.offset == 56
    assert rr._PagedConfig.reserved.offset == 60 and rr._PagedConfig.k_scale.offset == 64


def _append(rr, **kw):
    base = dict(n_heads=4, n_kv_heads=2, d=128, page=64, n_pages=10, max_pages=4, n_seqs=2, n_tokens=6, rot=128,
                interleaved=0, dtype=rr.RR_BF16, cache_dtype=rr.RR_BF16, ldq=512, ldk=256, ldv=256, k_scale=None,
                v_scale=None)
    base.update(kw)
    return rr._AppendConfig(*base.values())


def _paged(rr, **kw):
    base = dict(n_heads=4, n_kv_heads=2, d=128, page=64, n_pages=10, max_pages=4, n_seqs=2, n_q=1, k=0, n_sink=0,
                n_recent=0, n_prefix=0, dtype=rr.RR_BF16, cache_dtype=rr.RR_BF16, scale=0.0, reserved=0, k_scale=None,
                v_scale=None)
    base.update(kw)
    return rr._PagedConfig(*base.values())


def _append_call(rr, c, **kw):
    a = dict(K=FAKE, V=FAKE, Q=FAKE, seq_start=FAKE, lengths=FAKE, table=FAKE, freqs=FAKE, Kc=FAKE, Vc=FAKE,
             Q_out=ctypes.c_void_p(0x2000), stream=None)
    a.update(kw)
    return rr.lib.rr_cache_append(None if c is None else ctypes.byref(c), *a.values())


CACHE_FAULTS = [
    ({"n_kv_heads": 0}, -1), ({"page": 0}, -1), ({"n_pages": 0}, -1), ({"max_pages": 0}, -1), ({"n_seqs": 0}, -1),
    ({"page": 1 << 20, "max_pages": 1 << 11}, -1), ({"dtype": 2}, -1), ({"dtype": 7}, -1), ({"cache_dtype": 0}, -1),
    ({"dtype": 0, "cache_dtype": 2}, -1), ({"cache_dtype": 2}, -1), ({"k_scale": 0x1000, "v_scale": 0x1000}, -1),
    ({"cache_dtype": 2, "k_scale": 0x1000}, -1),
]


@pytest.mark.parametrize("kw,status", CACHE_FAULTS + [
    ({"d": 4}, -1), ({"d": 132}, -1), ({"d": 1032}, -1), ({"rot": -2}, -1), ({"rot": 130}, -1), ({"rot": 3}, -1),
    ({"interleaved": 2}, -1), ({"n_tokens": -1}, -1), ({"ldk": -1}, -1), ({"ldv": -1}, -1), ({"ldq": -1}, -1),
    ({"n_heads": 0}, -1),
])
def test_append_rejects_bad_configs(kw, status):
    rr = _rr()
    assert _append_call(rr, _append(rr, **kw)) == status
    assert rr.lib.rr_last_error()


def test_append_rejects_bad_pointers():
    rr = _rr()
    c = _append(rr)
    assert _append_call(rr, None) == -1
    for name in ("K", "V", "Q", "lengths", "table", "freqs", "Kc", "Vc", "Q_out"):
        assert _append_call(rr, c, **{name: None}) == -1, name
    # queries rotated in place only where their rows lie as the output's do
    assert _append_call(rr, _append(rr, ldq=768), Q_out=FAKE) == -1
    # without starts every sequence has as many new tokens
    assert _append_call(rr, _append(rr, n_tokens=7), seq_start=None) == -1
    # nothing to append: nothing is launched (the pointers are not real)
    assert _append_call(rr, _append(rr, n_tokens=0), K=None, V=None) == 0


def _paged_call(rr, c, prefix=False, **kw):
    a = dict(Q=FAKE, Kc=FAKE, Vc=FAKE, table=FAKE, lengths=FAKE, third=FAKE if prefix or (c and c.k) else None, O=FAKE,
             lse=None, ws=FAKE, n=1 << 40, stream=None)
    a.update(kw)
    f = rr.lib.rr_prefix_attention if prefix else rr.lib.rr_paged_attention
    return f(None if c is None else ctypes.byref(c), *a.values())


@pytest.mark.parametrize("kw,status", CACHE_FAULTS + [
    ({"n_heads": 3}, -1), ({"n_heads": 0}, -1), ({"n_q": 0}, -1), ({"k": -1}, -1), ({"n_sink": -1}, -1),
    ({"n_recent": -1}, -1), ({"k": 250, "n_sink": 4, "n_recent": 3}, -1), ({"n_prefix": -1}, -1),
    ({"n_prefix": 8, "k": 2}, -1), ({"n_prefix": 8, "n_recent": 1}, -1), ({"n_prefix": (1 << 30) + 1}, -1),
    ({"reserved": 1}, -1), ({"scale": -1.0}, -1), ({"scale": math.inf}, -1), ({"scale": math.nan}, -1),
    ({"d": 96}, -5), ({"d": 32}, -5), ({"dtype": 0, "cache_dtype": 0, "d": 256}, -5),
    ({"n_seqs": 1 << 20, "n_q": 1 << 12}, -5),
])
def test_paged_attention_rejects_bad_configs(kw, status):
    rr = _rr()
    c = _paged(rr, **kw)
    assert rr.lib.rr_paged_workspace_bytes(ctypes.byref(c)) == 0
    assert rr.lib.rr_last_error()
    assert _paged_call(rr, c, prefix=c.n_prefix != 0) == status


def test_paged_attention_rejects_bad_pointers():
    rr = _rr()
    c, p = _paged(rr), _paged(rr, n_prefix=8)
    assert rr.lib.rr_paged_workspace_bytes(None) == 0
    assert _paged_call(rr, None) == -1 and _paged_call(rr, None, prefix=True) == -1
    for name in ("Q", "Kc", "Vc", "table", "lengths", "O", "ws"):
        assert _paged_call(rr, c, **{name: None}) == -1, name
        assert _paged_call(rr, p, prefix=True, **{name: None}) == -1, name
    for name in ("Q", "Kc", "Vc", "O", "ws"):
        assert _paged_call(rr, c, **{name: ODD}) == -1, name
    # each call's own third input, and no other's
    assert _paged_call(rr, c, third=FAKE) == -1
    assert _paged_call(rr, _paged(rr, k=2), third=None) == -1
    assert _paged_call(rr, p) == -1
    assert _paged_call(rr, p, prefix=True, third=None) == -1
    assert _paged_call(rr, c, prefix=True) == -1
    for x, prefix in ((c, False), (p, True)):
        need = rr.lib.rr_paged_workspace_bytes(ctypes.byref(x))
        assert need > 0
        assert _paged_call(rr, x, prefix=prefix, n=need - 1) == -1
        assert b"workspace" in rr.lib.rr_last_error()


def test_limits_of_a_launch():
    """Tokens of an append and query rows behind a prefix take a workgroup each,
    and a launch has less than 2^24."""
    rr = _rr()
    assert _append_call(rr, _append(rr, n_tokens=1 << 24)) == -5
    assert rr.lib.rr_last_error()
    rows = dict(n_heads=8, n_kv_heads=2, n_seqs=1 << 10)
    for n_q, prefix, ok in ((1 << 11, 8, False), ((1 << 11) - 1, 8, True), (1 << 11, 0, True)):
        c = _paged(rr, n_q=n_q, n_prefix=prefix, **rows)
        assert (rr.lib.rr_paged_workspace_bytes(ctypes.byref(c)) > 0) is ok
        if not ok:
            assert _paged_call(rr, c, prefix=True) == -5


def test_workspace_is_bounded():
    """A workspace holds parts of a fixed number of workgroups, whatever the
    lengths that the page table allows."""
    rr = _rr()
    few = rr.lib.rr_paged_workspace_bytes(ctypes.byref(_paged(rr, n_heads=32, n_kv_heads=8, max_pages=1 << 12)))
    many = rr.lib.rr_paged_workspace_bytes(ctypes.byref(_paged(rr, n_heads=32, n_kv_heads=8, max_pages=1 << 20)))
    assert few == many < 64 << 20


def test_binding_checks_tensors():
    """Shapes, types and places that the binding refuses before any call."""
    rr = _rr()
    bf, i32 = torch.bfloat16, torch.int32
    K = torch.zeros((6, 2, 64), dtype=bf)
    pool = torch.zeros((10, 2, 16, 64), dtype=bf)
    table, lens = torch.zeros((2, 4), dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(ValueError, match="GPU"):
        rr.cache_append(K, K, pool, pool, table, lens)
    with pytest.raises(TypeError):
        rr.cache_append(K.half(), K.half(), pool, pool, table, lens)
    with pytest.raises(TypeError, match="queries' type"):
        rr.cache_append(K.float(), K.float(), pool, pool, table, lens)
    with pytest.raises(ValueError, match="scale"):
        rr.cache_append(K, K, pool, pool, table, lens, k_scale=torch.ones(2), v_scale=torch.ones(2))
    with pytest.raises(ValueError, match="scale"):
        rr.cache_append(K, K, pool.to(torch.float8_e4m3fn), pool.to(torch.float8_e4m3fn), table, lens)
    with pytest.raises(ValueError, match="one shape"):
        rr.cache_append(K, K, pool, pool[:9], table, lens)
    Q = torch.zeros((2, 1, 4, 64), dtype=bf)
    with pytest.raises(ValueError, match="GPU"):
        rr.paged_attention(Q, pool, pool, table, lens)
    with pytest.raises(TypeError):
        rr.paged_attention(Q[0], pool, pool, table, lens)
    with pytest.raises(ValueError, match="features"):
        rr.paged_attention(Q[..., :32], pool, pool, table, lens)
    with pytest.raises(ValueError, match="page_table"):
        rr.paged_attention(Q, pool, pool, table[:1], lens)
    with pytest.raises(ValueError, match="routes"):
        rr.paged_attention(Q, pool, pool, table, lens, routes=torch.zeros((7, 3), dtype=i32))
    with pytest.raises(TypeError, match="one type"):
        rr.paged_attention(Q, pool, pool.float(), table, lens)
