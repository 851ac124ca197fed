"""GPU parity of the paged cache through the C ABI against the binary64
oracle: appending rotated tokens, attention of the newest tokens over the
cache (all of it, along routes of pages, behind a shared prefix), and a run of
them together with pooling and routing.

Tolerances, from the arithmetic (u = half a step of the output's type).
Append: the angle is reduced in binary64 and rounded to binary32 in turns
(at most 2^-26 turns off: pi 2^-25 radians), sine and cosine and the two
products and their sum round to 2^-24 relative each or twice that: 8 * 2^-24 *
(|x| + |y|) for partners x, y, then u relative (e4m3: 2^-4, or half its
smallest step, 2^-10).
Attention: with S the largest scaled sum of |q_i k_i| of a row, a score is off
by at most (d + 8) 2^-24 S (products exact or rounded once, d additions, the
scaling, the shift by the maximum), so each weight by as much relatively, and
the normalised weights by twice that; sums of n weights add (n + 8) 2^-24;
with bf16 queries a weight enters the value product as two bf16 numbers, 2^-16
off, or as one, 2^-8 off, where more than 16 rows are multiplied together.
Together err = 2 (d + 8) 2^-24 S + (n + 8) 2^-24 (+ 2^-16 or 2^-8), the output
is off by err * sum_u w_u |v_u| + u |o|; the logarithm of the sum, which takes the
weights as they are, by err without its last part."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import paged as op
from paper_2609_07306_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)
    yield


def rrmod():
    from paper_2609_07306_amd import routerelay
    return routerelay


def note(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _np(t):
    return t.float().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _nan_pool(shape, dtype):
    """A pool that holds NaN wherever no token is written."""
    if dtype == E4M3:
        return torch.full(shape, 0x7F, dtype=torch.uint8, device=DEV).view(E4M3)
    return torch.full(shape, math.nan, dtype=dtype, device=DEV)


def _values(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TYPE[dtype]).to(DEV)


class Cache:
    """Sequences of given lengths in pages of any order; every place that holds
    no token holds NaN, table entries past a sequence's pages are bad."""

    def __init__(self, rng, lens, Hkv, d, page, dtype, spare=2, width=2):
        self.page, self.d, self.Hkv, self.dtype = page, d, Hkv, dtype
        n = [-(-x // page) for x in lens]
        n_pages = sum(n) + spare
        self.K, self.V = (_nan_pool((n_pages, Hkv, page, d), TYPE[dtype]) for _ in range(2))
        order = rng.permutation(n_pages)
        self.table = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31], size=(len(lens), max(n + [1]) + width)).astype(np.int64)
        at = 0
        self.scales = (None, None)
        if dtype == "e4m3":
            self.scales = tuple((0.01 + 0.02 * rng.random(Hkv)).astype(np.float32) for _ in range(2))
        for b, length in enumerate(lens):
            self.table[b, :n[b]] = order[at:at + n[b]]
            at += n[b]
            if length:
                self.put(b, 0, *((rng.standard_normal((length, Hkv, d))) for _ in range(2)))
        self.lens = list(lens)

    def put(self, b, first, k, v):
        """Token rows from position `first` on, as the cache's type holds them."""
        u = np.arange(first, first + len(k))
        phys = torch.from_numpy(self.table[b, u // self.page]).to(DEV)
        place = torch.from_numpy(u % self.page).to(DEV)
        for pool, x, s in ((self.K, k, self.scales[0]), (self.V, v, self.scales[1])):
            x = torch.from_numpy(np.asarray(x, np.float32)).to(DEV)
            if s is not None:
                x = (x / torch.from_numpy(s).to(DEV)[:, None])
                finite = x.isfinite()
                x = torch.where(finite, x.clamp(-448, 448), x).to(E4M3)
                pool.view(torch.uint8)[phys, :, place] = x.view(torch.uint8)
            else:
                pool[phys, :, place] = x.to(pool.dtype)

    def args(self):
        return self.K, self.V, _i32(self.table), _i32(self.lens)

    def kw(self):
        return {} if self.scales[0] is None else {n: torch.from_numpy(s).to(DEV)
                                                   for n, s in zip(("k_scale", "v_scale"), self.scales)}

    def oracle(self, Q, **kw):
        K, V = _np(self.K), _np(self.V)
        if self.scales[0] is not None:
            kw.update(k_scale=self.scales[0], v_scale=self.scales[1])
        return op.attention(_np(Q), K, V, self.table, self.lens, **kw)


def _check(O, lse, ref, d, n, qtype, rows=1):
    """rows: query rows that are multiplied with a key head's tokens together."""
    exact, elog, W, S = ref
    got = O.double().cpu().numpy()
    err = 2 * (d + 8) * 2.0 ** -24 * S + (n + 8) * 2.0 ** -24
    weight = 0 if qtype == "f32" else 2.0 ** -16 if rows <= 16 else 2.0 ** -8
    tol = 1.01 * ((err + weight)[..., None] * W + HALF[qtype] * np.abs(exact)) + 1e-30
    off = np.abs(got - exact)
    bad = np.argwhere(~(off <= tol))
    assert len(bad) == 0, f"{len(bad)} outputs beyond tolerance, first {bad[:4].tolist()}: " \
                          f"{got[tuple(bad[0])]} vs {exact[tuple(bad[0])]} (tol {tol[tuple(bad[0])]})"
    if lse is not None:
        glog = lse.double().cpu().numpy()
        none = np.isneginf(elog)
        assert np.array_equal(np.isneginf(glog), none)
        loff = np.abs(glog[~none] - elog[~none])
        # (its own rounding, and the logarithm's)
        assert np.all(loff <= 1.01 * err[~none] + 4 * 2.0 ** -24 * (1 + np.abs(elog[~none]))), loff.max()


# ------------------------------------------------------------------ append

APPEND = [
    # name, H, Hkv, d, dtype, cache, page, new tokens, tokens before, rot, interleaved, fused
    ("one_token", 8, 2, 128, "bf16", "bf16", 64, [1], [63], 128, False, False),
    ("decode_e4m3", 8, 2, 128, "bf16", "e4m3", 16, [1] * 9, [0, 1, 15, 16, 31, 32, 100, 7, 8], 128, False, True),
    ("ragged", 4, 4, 64, "bf16", "bf16", 16, [0, 5, 0, 33, 1], [3, 0, 7, 2, 130], 64, False, False),
    ("partial_rotation", 6, 2, 64, "f32", "f32", 48, [3, 50], [1, 40], 32, True, False),
    ("odd_rotation", 6, 2, 64, "f32", "f32", 7, [3, 11], [0, 4], 20, False, True),
    ("odd_rotation_interleaved", 5, 1, 72, "bf16", "e4m3", 7, [3, 11], [0, 4], 22, True, False),
    ("odd_rotation_bf16", 3, 3, 40, "bf16", "bf16", 1, [4, 2], [5, 0], 20, False, False),
    ("no_rotation", 2, 1, 256, "bf16", "e4m3", 32, [4], [30], 0, False, False),
    ("wide_rows", 2, 1, 1024, "f32", "f32", 5, [4], [3], 1024, False, False),
    ("interleaved_vectors", 8, 8, 256, "bf16", "bf16", 100, [70], [150], 256, True, True),
    ("far_positions", 4, 1, 128, "f32", "f32", 64, [3, 2], [900000, 64 * 16384 - 2], 128, False, False),
]


@pytest.mark.parametrize("case", APPEND, ids=[c[0] for c in APPEND])
@pytest.mark.parametrize("with_q", [True, False])
def test_append_parity(case, with_q):
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, new, before, rot, inter, fused = case
    note(f"append {case} with_q={with_q}")
    rng = np.random.default_rng(len(name) + d)
    n, B = sum(new), len(new)
    left = 3  # rows past the last sequence's
    lens = [a + b for a, b in zip(new, before)]
    # (far sequences hold their last pages only)
    first = [max(0, b // page - 1) for b in before]
    n_pages = sum(-(-x // page) - f for x, f in zip(lens, first)) + 2
    width = max(-(-x // page) for x in lens) + 1
    table = np.full((B, width), -1, np.int64)
    order, at = rng.permutation(n_pages), 0
    for b, x in enumerate(lens):
        c = -(-x // page) - first[b]
        table[b, first[b]:first[b] + c] = order[at:at + c]
        at += c
    start = np.concatenate([[0], np.cumsum(new)])
    if fused:
        qkv = _values(rng, (n + left, H + 2 * Hkv, d), dtype)
        Q, K, V = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        Q, K, V = (_values(rng, (n + left, h, d), dtype) for h in (H, Hkv, Hkv))
    scales = [(0.004 + 0.01 * rng.random(Hkv)).astype(np.float32) for _ in range(2)] if cache == "e4m3" else [None, None]
    freqs = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    Kc, Vc = (_values(rng, (n_pages, Hkv, page, d), cache) for _ in range(2))
    K0, V0 = _np(Kc), _np(Vc)
    Q_out = torch.full((n + left, H, d), 7.0, dtype=TYPE[dtype], device=DEV)
    got = rr.cache_append(K, V, Kc, Vc, _i32(table), _i32(lens), seq_start=_i32(start),
                          freqs=torch.from_numpy(freqs).to(DEV) if rot else None, interleaved=inter,
                          Q=Q if with_q else None, Q_out=Q_out if with_q else None,
                          **({} if cache != "e4m3" else dict(k_scale=torch.from_numpy(scales[0]).to(DEV),
                                                             v_scale=torch.from_numpy(scales[1]).to(DEV))))
    torch.cuda.synchronize()
    assert (got is Q_out) if with_q else got is None
    Kn, Vn, Qn = _np(K), _np(V), _np(Q)
    Kg, Vg, Qg = _np(Kc), _np(Vc), _np(Q_out)
    touched = np.zeros((n_pages, page), bool)
    half = rot // 2

    def held(x, s):  # what the cache's type is to round
        return x if s is None else np.clip(x / s.astype(np.float64)[:, None], -448, 448)

    def near(got, x, size, s, t):
        y, z = held(x, s), size if s is None else size / s.astype(np.float64)[:, None]
        small = 2.0 ** -10 if t == "e4m3" else 0.0
        tol = 8 * 2.0 ** -24 * z + np.maximum(HALF[t] * (np.abs(y) + 8 * 2.0 ** -24 * z), small)
        assert np.all(np.abs(got - y) <= tol * 1.001), np.max(np.abs(got - y) - tol)

    def partners(x):  # |x| + |y| of every rotated feature
        out = np.abs(x).astype(np.float64)
        if half:
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, half), slice(half, rot))
            out[:, a], out[:, b] = np.abs(x[:, a]) + np.abs(x[:, b]), np.abs(x[:, a]) + np.abs(x[:, b])
        return out

    for i, (pos, phys, place) in enumerate(op.places(start, lens, table, n_pages, page, n)):
        assert pos >= 0 and phys >= 0
        touched[phys, place] = True
        near(Kg[phys, :, place], op.rotate(Kn[i], pos, freqs, inter), partners(Kn[i]), scales[0], cache)
        near(Vg[phys, :, place], Vn[i].astype(np.float64), 0 * np.abs(Vn[i]), scales[1], cache)
        if with_q:
            near(Qg[i], op.rotate(Qn[i], pos, freqs, inter), partners(Qn[i]), None, dtype)
    assert np.array_equal(Kg.transpose(0, 2, 1, 3)[~touched], K0.transpose(0, 2, 1, 3)[~touched])
    assert np.array_equal(Vg.transpose(0, 2, 1, 3)[~touched], V0.transpose(0, 2, 1, 3)[~touched])
    assert np.all(Qg[n:] == 7.0) and (with_q or np.all(Qg == 7.0))


def test_append_leaves_out_what_has_no_place():
    """Bad page numbers, positions before a sequence's first token and past its
    table, a table of other sequences: nothing else is written."""
    rr = rrmod()
    note("append without a place")
    rng = np.random.default_rng(3)
    Hkv, d, page, n_pages = 2, 64, 4, 6
    table = np.array([[0, 6], [-1, 1], [2 ** 31 - 1, -2 ** 31], [2, 3], [4, 5]])
    new = [6, 6, 3, 3, 3]
    lens = [6, 6, 3, 2, 10]  # the fourth has a token before its first, the fifth's last two lie past its table
    start = np.concatenate([[0], np.cumsum(new)])
    n = sum(new)
    K, V, Q = (_values(rng, (n, Hkv, d), "f32") for _ in range(3))
    Kc, Vc = (torch.full((n_pages, Hkv, page, d), 7.0, device=DEV) for _ in range(2))
    Qo = torch.full((n, Hkv, d), 7.0, device=DEV)
    rr.cache_append(K, V, Kc, Vc, _i32(table), _i32(lens), seq_start=_i32(start), Q=Q, Q_out=Qo)
    torch.cuda.synchronize()
    want = torch.full_like(Kc, 7.0)
    wantq = torch.full_like(Qo, 7.0)
    placed = 0
    for i, (pos, phys, place) in enumerate(op.places(start, lens, table, n_pages, page, n)):
        if phys >= 0:
            want[phys, :, place] = K[i]
            placed += 1
        if pos >= 0:  # (the query of a token that has a position is rotated, whether or not its page is there)
            wantq[i] = Q[i]
    assert placed == 4 + 2 + 0 + 2 + 1
    assert torch.equal(Kc, want) and torch.equal(Qo, wantq)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 300])
def test_append_finds_a_tokens_sequence(B):
    """Sequences without new tokens among others, rows before the first one's
    and after the last one's, starts that begin past 0: values go where they
    should and nowhere else."""
    rr = rrmod()
    note(f"append to {B} sequences")
    rng = np.random.default_rng(B)
    Hkv, d, page = 1, 8, 4
    new = rng.integers(0, 4, size=B) * (rng.random(B) < 0.7)
    new[B // 2] = 5
    lens = new + rng.integers(0, 9, size=B)
    start = 2 + np.concatenate([[0], np.cumsum(new)])
    n = int(start[-1]) + 3
    width = -(-int(lens.max()) // page)
    n_pages = B * width
    table = rng.permutation(n_pages).reshape(B, width)
    K, V = (_values(rng, (n, Hkv, d), "f32") for _ in range(2))
    Kc, Vc = (torch.full((n_pages, Hkv, page, d), 7.0, device=DEV) for _ in range(2))
    want_k, want_v = Kc.clone(), Vc.clone()
    rr.cache_append(K, V, Kc, Vc, _i32(table), _i32(lens), seq_start=_i32(start))
    torch.cuda.synchronize()
    for b in range(B):
        for j in range(new[b]):
            u, i = int(lens[b] - new[b] + j), int(start[b] + j)
            want_k[table[b, u // page], :, u % page] = K[i]
            want_v[table[b, u // page], :, u % page] = V[i]
    assert torch.equal(Kc, want_k) and torch.equal(Vc, want_v)


def test_append_starts_past_the_tokens():
    """seq_start may count more tokens than the call brings: those alone count."""
    rr = rrmod()
    note("append with starts past n_tokens")
    K = torch.ones((3, 1, 8), device=DEV)
    Kc, Vc = (torch.zeros((4, 1, 2, 8), device=DEV) for _ in range(2))
    rr.cache_append(K, 2 * K, Kc, Vc, _i32([[0, 1], [2, 3]]), _i32([2, 4]), seq_start=_i32([0, 2, 6]))
    torch.cuda.synchronize()
    # sequence 1's tokens 2 .. 5 are its positions 0 .. 3: token 2 alone is there
    want = torch.zeros_like(Kc)
    want[0], want[2, :, 0] = 1.0, 1.0
    assert torch.equal(Kc, want) and torch.equal(Vc, 2 * want)


def test_append_in_place_and_broadcast():
    """Queries rotated in place; one token's values for all (a stride of 0)."""
    rr = rrmod()
    note("append in place, stride 0")
    rng = np.random.default_rng(8)
    K, Q = (_values(rng, (5, 2, 128), "bf16") for _ in range(2))
    V = _values(rng, (1, 2, 128), "bf16").expand(5, 2, 128)
    f = torch.from_numpy(10000.0 ** (-np.arange(0, 128, 2) / 128)).to(DEV)
    table, lens = _i32([[0, 1, 2]]), _i32([12])
    pools = [torch.zeros((3, 2, 4, 128), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    a = rr.cache_append(K, V, pools[0], pools[1], table, lens, freqs=f, Q=Q)
    b = rr.cache_append(K, V.contiguous(), pools[2], pools[3], table, lens, freqs=f, Q=Q, Q_out=Q)
    torch.cuda.synchronize()
    assert b is Q and torch.equal(a, Q)
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    assert torch.equal(pools[1][1, :, 3], V[0])


def test_append_e4m3_borders():
    """Past the largest finite value an 8-bit cache holds that one; NaN stays
    NaN; ties go to the even one."""
    rr = rrmod()
    note("append e4m3 borders")
    x = torch.tensor([448, 449, 464, 465, 1e30, -448, -1e30, math.inf, -math.inf, math.nan, 0.0, -0.0, 2.0 ** -9,
                      2.0 ** -10, 3 * 2.0 ** -10, 17, 19, 2.0 ** -11, 100, -100, 240, 248, 256, 1], device=DEV)
    V = x.to(torch.bfloat16).repeat(1, 1, 1)
    Kc, Vc = (torch.zeros((1, 1, 1, 24), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    one = torch.ones(1, device=DEV)
    rr.cache_append(V, V, Kc, Vc, _i32([[0]]), _i32([1]), k_scale=one, v_scale=one)
    torch.cuda.synchronize()
    b = x.to(torch.bfloat16).float()
    want = torch.where(b.isnan(), b, b.clamp(-448, 448)).to(E4M3).float()
    assert torch.equal(Vc.float().flatten().nan_to_num(nan=-1), want.nan_to_num(nan=-1))
    assert torch.equal(Kc.view(torch.uint8), Vc.view(torch.uint8))


# --------------------------------------------------------------- attention

PAGED = [
    # name, H, Hkv, d, dtype, cache, page, lengths, n_q
    ("bf16_d128", 8, 2, 128, "bf16", "bf16", 64, [1, 2, 63, 64, 65, 500, 129], 1),
    ("bf16_d64_empty", 4, 4, 64, "bf16", "bf16", 16, [0, 1, 0, 130, 17], 1),
    ("bf16_d256_page1", 4, 2, 256, "bf16", "bf16", 1, [1, 300, 1100], 1),
    ("bf16_page300", 2, 1, 128, "bf16", "bf16", 300, [299, 301, 1, 900], 2),
    ("bf16_drafts_two_blocks", 14, 2, 128, "bf16", "bf16", 7, [3, 200, 2, 61], 3),
    ("bf16_drafts_two_tiles", 16, 2, 64, "bf16", "bf16", 48, [9, 400, 30], 9),
    ("bf16_d128_four_blocks", 8, 1, 128, "bf16", "bf16", 16, [7, 300, 260], 7),
    ("bf16_d256_blocks", 8, 1, 256, "bf16", "bf16", 32, [5, 200], 6),
    ("e4m3_d64", 4, 2, 64, "bf16", "e4m3", 16, [1, 40, 333], 1),
    ("e4m3_d128", 8, 2, 128, "bf16", "e4m3", 16, [1, 128, 1000, 0], 2),
    ("e4m3_d128_blocks", 12, 1, 128, "bf16", "e4m3", 5, [30, 500], 4),
    ("e4m3_d256", 4, 1, 256, "bf16", "e4m3", 64, [65, 700], 5),
    ("f32_d64", 6, 2, 64, "f32", "f32", 48, [5, 1, 700, 97, 0], 5),
    ("f32_d128", 4, 4, 128, "f32", "f32", 16, [1, 15, 16, 17, 1025], 1),
    ("f32_d128_blocks", 12, 2, 128, "f32", "f32", 33, [3, 321], 4),
]


@pytest.mark.parametrize("case", PAGED, ids=[c[0] for c in PAGED])
def test_paged_attention_parity(case):
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, lens, nq = case
    note(f"paged attention {case}")
    rng = np.random.default_rng(sum(lens) + d)
    c = Cache(rng, lens, Hkv, d, page, cache)
    Q = _values(rng, (len(lens), nq, H, d), dtype, 2.0)
    lse = torch.full((len(lens), nq, H), 7.0, device=DEV)
    O = rr.paged_attention(Q, *c.args(), lse=lse, **c.kw())
    torch.cuda.synchronize()
    _check(O, lse, c.oracle(Q), d, max(lens), dtype, nq * H // Hkv)
    # the same inputs give the same bits
    again = rr.paged_attention(Q, *c.args(), **c.kw())
    assert torch.equal(O, again)


@pytest.mark.parametrize("dtype,cache,d", [("bf16", "bf16", 128), ("bf16", "e4m3", 64), ("f32", "f32", 128)])
def test_paged_attention_long_and_short(dtype, cache, d):
    """One long sequence among short ones: its keys are cut over many
    workgroups, whose parts are joined; sampled rows against the oracle."""
    rr = rrmod()
    note(f"long and short {dtype} {cache} {d}")
    rng = np.random.default_rng(5)
    lens = [40000, 3, 0, 700, 1, 129]
    c = Cache(rng, lens, 2, d, 64, cache)
    Q = _values(rng, (len(lens), 1, 8, d), dtype, 2.0)
    lse = torch.empty((len(lens), 1, 8), device=DEV)
    O = rr.paged_attention(Q, *c.args(), lse=lse, **c.kw())
    torch.cuda.synchronize()
    _check(O, lse, c.oracle(Q), d, max(lens), dtype)


def test_paged_attention_bad_pages_and_lengths():
    """Pages that are none hide their tokens; lengths are taken between 0 and
    what the table holds."""
    rr = rrmod()
    note("bad pages, lengths out of range")
    rng = np.random.default_rng(6)
    c = Cache(rng, [100, 90, 64, 50], 2, 64, 16, "bf16", width=0)
    c.table[0, 2], c.table[1, 0], c.table[1, 5] = -1, 2 ** 31 - 1, -5
    c.table[2, :] = 99
    Q = _values(rng, (4, 2, 4, 64), "bf16", 2.0)
    for lens in ([100, 90, 64, 50], [112, 90, 64, -3], [2 ** 31 - 1, 90, 0, -2 ** 31]):
        c.lens = lens
        if max(lens) > 100:  # (what the cache holds past the tokens)
            c.put(0, 100, *(rng.standard_normal((12, 2, 64)) for _ in range(2)))
        O = rr.paged_attention(Q, *c.args())
        torch.cuda.synchronize()
        _check(O, None, c.oracle(Q), 64, 112, "bf16")
        assert not O[2].any()


@pytest.mark.parametrize("heads", [8, 24])  # (16 rows, and more)
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
def test_values_of_later_tokens_do_not_reach_earlier_queries(dtype, cache, heads):
    """Draft tokens whose rows hold NaN (and infinities): queries before them
    are as if they held zeros, theirs are not finite."""
    rr = rrmod()
    note(f"later tokens not finite {dtype} {cache} {heads}")
    rng = np.random.default_rng(9)
    lens, nq, d = [150, 33, 4], 4, 128
    c = Cache(rng, lens, 2, d, 16, cache)
    Q = _values(rng, (3, nq, heads, d), dtype)
    want = c.oracle(Q)
    for b, n in enumerate(lens):
        bad = np.full((1, 2, d), math.nan)
        if cache != "e4m3" and b == 1:
            bad[:] = math.inf
        c.put(b, n - 1, bad, bad)  # the newest token
    O = rr.paged_attention(Q, *c.args(), **c.kw())
    torch.cuda.synchronize()
    first = tuple(x[:, :nq - 1] for x in want)
    _check(O[:, :nq - 1], None, first, d, 150, dtype, nq * heads // 2)
    assert not O[:, nq - 1].isfinite().any()


def test_scores_far_apart():
    """Scores over a range whose exponentials overflow, and queries that are
    not finite themselves."""
    rr = rrmod()
    note("scores far apart")
    rng = np.random.default_rng(10)
    c = Cache(rng, [300, 257], 1, 64, 32, "f32")
    Q = _values(rng, (2, 1, 2, 64), "f32", 60.0)
    O = rr.paged_attention(Q, *c.args())
    torch.cuda.synchronize()
    _check(O, None, c.oracle(Q), 64, 300, "f32")
    Q[0, 0, 1] = math.nan
    P = rr.paged_attention(Q, *c.args())
    torch.cuda.synchronize()
    assert P[0, 0, 1].isnan().all() and torch.equal(P[1], O[1]) and torch.equal(P[0, 0, 0], O[0, 0, 0])


ROUTED = [
    # name, H, Hkv, d, dtype, cache, page, lengths, n_q, k, sinks, recent
    ("bf16_d128", 8, 2, 128, "bf16", "bf16", 64, [1, 700, 64, 65, 1300], 1, 6, 1, 2),
    ("bf16_drafts", 4, 2, 64, "bf16", "bf16", 16, [5, 300, 2], 3, 9, 0, 1),
    ("page1", 4, 4, 64, "bf16", "bf16", 1, [300, 40, 0], 1, 200, 8, 48),
    ("routes_alone", 4, 1, 128, "bf16", "e4m3", 33, [400, 1], 2, 5, 0, 0),
    ("recent_alone", 4, 1, 128, "bf16", "bf16", 33, [400, 1, 90], 2, 0, 0, 3),
    ("sinks_alone", 4, 1, 256, "bf16", "bf16", 20, [400, 1, 90], 1, 0, 2, 0),
    ("f32", 6, 2, 64, "f32", "f32", 48, [900, 10, 96], 2, 7, 1, 1),
    ("f32_d128", 2, 2, 128, "f32", "f32", 16, [500], 1, 20, 2, 2),
    ("one_head", 1, 1, 128, "bf16", "bf16", 64, [4000], 1, 60, 1, 1),
    ("two_heads_d256", 2, 1, 256, "bf16", "bf16", 128, [8000], 1, 70, 1, 1),
    ("two_tokens_d256", 1, 1, 256, "bf16", "e4m3", 128, [8000], 2, 70, 1, 1),
]


@pytest.mark.parametrize("case", ROUTED, ids=[c[0] for c in ROUTED])
def test_routed_parity(case):
    """Routes that name pages twice, pages after the query, none and bad ones;
    rows that see nothing."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, lens, nq, k, sinks, recent = case
    note(f"routed {case}")
    rng = np.random.default_rng(len(name) * 7 + d)
    c = Cache(rng, lens, Hkv, d, page, cache)
    B = len(lens)
    R = np.full((B * H * nq, k), -1, np.int64)
    for r in range(len(R)):
        pages = max(1, -(-lens[r // (H * nq)] // page))
        R[r] = rng.integers(-1, pages + 2, size=k)  # some twice, some after the query, some none
        if k > 3 and r % 3 == 0:
            R[r, 2], R[r, 3] = R[r, 0], 2 ** 31 - 1
        if r % 5 == 4:
            R[r] = -1
    Q = _values(rng, (B, nq, H, d), dtype, 2.0)
    lse = torch.empty((B, nq, H), device=DEV)
    routes = _i32(R) if k else None
    O = rr.paged_attention(Q, *c.args(), routes=routes, n_sink=sinks, n_recent=recent, lse=lse, **c.kw())
    torch.cuda.synchronize()
    _check(O, lse, c.oracle(Q, routes=R if k else None, n_sink=sinks, n_recent=recent), d, max(lens), dtype)
    if sinks == recent == 0:  # rows without any page
        assert not O.view(B, nq, H, d)[0, 0].any(-1).all()


def test_routed_over_every_page_is_attention_over_all():
    rr = rrmod()
    note("every page routed")
    rng = np.random.default_rng(4)
    lens = [1000, 513]
    c = Cache(rng, lens, 2, 128, 64, "bf16")
    Q = _values(rng, (2, 1, 8, 128), "bf16", 2.0)
    R = np.tile(rng.permutation(16), (16, 1))
    O = rr.paged_attention(Q, *c.args(), routes=_i32(R))
    torch.cuda.synchronize()
    _check(O, None, c.oracle(Q), 128, 1000, "bf16")


PREFIX = [
    # name, H, Hkv, d, dtype, cache, page, prefix, lengths behind it, n_q
    ("few_d64", 8, 2, 64, "bf16", "bf16", 32, 200, [1, 40, 7], 1),
    ("one_block_d128", 4, 1, 128, "bf16", "bf16", 64, 128, [1, 130, 64, 65], 1),
    ("two_blocks", 8, 2, 128, "bf16", "bf16", 16, 777, [3, 100, 20, 16, 17, 1], 1),
    ("four_blocks_tiles", 8, 2, 128, "bf16", "bf16", 64, 1000, [5 + 7 * i for i in range(40)], 2),
    ("d64_tiles", 8, 1, 64, "bf16", "bf16", 7, 300, [1 + i for i in range(20)], 1),
    ("d256_tiles", 4, 1, 256, "bf16", "bf16", 48, 500, [1 + 9 * i for i in range(13)], 1),
    ("e4m3_d128", 8, 2, 128, "bf16", "e4m3", 16, 1500, [2 + 30 * i for i in range(17)], 2),
    ("e4m3_d64", 4, 4, 64, "bf16", "e4m3", 64, 64, [1, 2], 1),
    ("f32_d64", 6, 2, 64, "f32", "f32", 48, 600, [4 + i for i in range(15)], 4),
    ("f32_d128", 4, 2, 128, "f32", "f32", 16, 100, [1, 2, 50], 1),
    ("one_token_prefix", 4, 2, 128, "bf16", "bf16", 64, 1, [1, 70], 1),
    ("whole_sequence_shared", 4, 2, 128, "bf16", "bf16", 16, 90, [0, 0, 3], 1),
    ("drafts_shared", 4, 2, 64, "bf16", "bf16", 16, 90, [0, 1, 3], 4),
]


def _prefix_cache(rng, Hkv, d, page, cache, prefix, lens):
    """Sequences that share their first `prefix` tokens, whose table entries
    before the page that the prefix ends in are bad."""
    c = Cache(rng, [prefix + x for x in lens] + [prefix], Hkv, d, page, cache)
    pages = c.table[-1, :-(-prefix // page)].copy()
    c.table, c.lens = c.table[:-1].copy(), c.lens[:-1]
    c.table[:, :prefix // page] = -1
    # what a sequence's own page holds before the prefix's end is not read
    return c, pages


@pytest.mark.parametrize("case", PREFIX, ids=[c[0] for c in PREFIX])
def test_prefix_parity(case):
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, prefix, lens, nq = case
    note(f"prefix {case}")
    rng = np.random.default_rng(len(name) * 11 + d)
    c, pages = _prefix_cache(rng, Hkv, d, page, cache, prefix, lens)
    B = len(lens)
    Q = _values(rng, (B, nq, H, d), dtype, 2.0)
    lse = torch.empty((B, nq, H), device=DEV)
    O = rr.prefix_attention(Q, *c.args(), _i32(pages), prefix, lse=lse, **c.kw())
    torch.cuda.synchronize()
    ref = c.oracle(Q, prefix_pages=pages, n_prefix=prefix)
    _check(O, lse, ref, d, max(c.lens), dtype, B * nq * H // Hkv)
    again = rr.prefix_attention(Q, *c.args(), _i32(pages), prefix, **c.kw())
    assert torch.equal(O, again)


def test_prefix_with_sequences_that_are_done():
    """Padded rows (length 0) and sequences shorter than the prefix see what
    they hold of it; NaN past that does not reach them."""
    rr = rrmod()
    note("prefix, short sequences")
    rng = np.random.default_rng(21)
    for dtype, cache in (("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3")):
        prefix, lens = 300, [0, 20, -300, -270, 2, -299, -100]
        c, pages = _prefix_cache(rng, 2, 64, 16, cache, prefix, [max(x, 0) for x in lens])
        c.lens = [prefix + x for x in lens]
        Q = _values(rng, (7, 2, 4, 64), dtype, 2.0)
        want = c.oracle(Q, prefix_pages=pages, n_prefix=prefix)
        O = rr.prefix_attention(Q, *c.args(), _i32(pages), prefix, **c.kw())
        torch.cuda.synchronize()
        _check(O, None, want, 64, 320, dtype, 28)
        assert not O[2].any()
        # the prefix's token 250 is past the sequences of 0, 30, 1 and 200 tokens
        phys, place = pages[250 // 16], 250 % 16
        if cache == "e4m3":
            c.V.view(torch.uint8)[phys, :, place] = 0x7F
        else:
            c.V[phys, :, place] = math.nan
        P = rr.prefix_attention(Q, *c.args(), _i32(pages), prefix, **c.kw())
        torch.cuda.synchronize()
        for b in (2, 3, 5, 6):
            _check(P[b:b + 1], None, tuple(x[b:b + 1] for x in want), 64, 320, dtype, 28)
        for b in (0, 1, 4):
            assert not P[b].isfinite().any()


# ------------------------------------------------------------- as it is used

def test_offsets_past_32_bits():
    """Pools of more than 2^32 bytes and 2^31 elements: tokens in their last
    pages."""
    rr = rrmod()
    note("large pools")
    Hkv, d, page = 8, 128, 64
    n_pages = (1 << 31) // (Hkv * page * d) + 300  # elements past 2^31
    rng = np.random.default_rng(2)
    Kc, Vc = (torch.zeros((n_pages, Hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens = [200, 70]
    table = np.array([[n_pages - 1, 5, n_pages - 3, n_pages - 2], [n_pages - 200, n_pages - 201, 0, 0]])
    K, V = (_values(rng, (270, Hkv, d), "bf16") for _ in range(2))
    rr.cache_append(K, V, Kc, Vc, _i32(table), _i32(lens), seq_start=_i32([0, 200, 270]))
    Q = _values(rng, (2, 1, 16, d), "bf16", 2.0)
    O = rr.paged_attention(Q, Kc, Vc, _i32(table), _i32(lens))
    torch.cuda.synchronize()
    used = sorted(set(table.flatten().tolist()))
    small = np.searchsorted(used, table)
    at = torch.tensor(used, device=DEV)
    ref = op.attention(_np(Q), _np(Kc[at]), _np(Vc[at]), small, lens)
    _check(O, None, ref, d, 200, "bf16")
    for b, first in ((0, 0), (1, 200)):
        for i in range(lens[b]):
            assert torch.equal(Kc[table[b, i // page], :, i % page], K[first + i])


def test_decode_steps_together():
    """Prompts appended, pages pooled, routes from the router, decode steps
    along them and over everything, through the binding: the cache grows by the
    new tokens alone, and every step's outputs match the oracle on it."""
    rr = rrmod()
    note("decode steps")
    rng = np.random.default_rng(12)
    H, Hkv, d, page, B, k = 8, 2, 128, 32, 3, 4
    lens = np.array([300, 170, 33])
    c = Cache(rng, [0] * B, Hkv, d, page, "bf16", spare=40, width=12)
    order = rng.permutation(40)
    for b in range(B):
        c.table[b] = order[13 * b:13 * b + 13]
    K, V, Q = (_values(rng, (int(lens.sum()), h, d), "bf16") for h in (Hkv, Hkv, H))
    f = torch.from_numpy(10000.0 ** (-np.arange(0, d, 2) / d)).to(DEV)
    start = np.concatenate([[0], np.cumsum(lens)])
    c.lens = lens.tolist()
    Kc, Vc, table, lengths = c.args()
    rr.cache_append(K, V, Kc, Vc, table, lengths, seq_start=_i32(start), freqs=f, Q=Q)
    for step in range(3):
        c.lens = [x + 1 for x in c.lens]
        lengths += 1
        k1, v1, q1 = (_values(rng, (B, h, d), "bf16") for h in (Hkv, Hkv, H))
        q = rr.cache_append(k1, v1, Kc, Vc, table, lengths, freqs=f, Q=q1).view(B, 1, H, d)
        # whole pages' representations, in the sequences' order; a page that is
        # not full yet is among the last ones, which are always seen
        n_pages = Kc.shape[0]
        reps = rr.pool_chunks(Kc.view(n_pages * Hkv, page, d), page).view(n_pages, Hkv, d)
        most = 1 + max(c.lens) // page
        full = torch.tensor([n // page for n in c.lens], device=DEV)
        Kr = reps[table[:, :most].long()]
        Kr = torch.where((torch.arange(most, device=DEV) < full[:, None])[..., None, None], Kr, torch.zeros_like(Kr))
        cfg = rr.Config(B * H, B * Hkv, 1, most, d, k, dtype="bf16")
        routes = torch.empty((B * H, k), dtype=torch.int32, device=DEV)
        rr.full_route(cfg, q.view(B * H, 1, d), Kr.transpose(1, 2).reshape(B * Hkv, most, d).contiguous(), routes)
        sparse = rr.paged_attention(q, Kc, Vc, table, lengths, routes=routes, n_sink=1, n_recent=2)
        dense = rr.paged_attention(q, Kc, Vc, table, lengths)
        torch.cuda.synchronize()
        _check(sparse, None, c.oracle(q, routes=routes.cpu().numpy(), n_sink=1, n_recent=2), d, max(c.lens), "bf16")
        _check(dense, None, c.oracle(q), d, max(c.lens), "bf16")
        for b, n in enumerate(c.lens):  # the new token alone lies where it should; what follows is still empty
            phys, place = int(c.table[b, (n - 1) // page]), (n - 1) % page
            assert torch.equal(Vc[phys, :, place], v1[b])
            assert place + 1 == page or Vc[phys, :, place + 1:].isnan().all()


def test_captured_step():
    """A decode step captured once and replayed with the lengths and inputs of
    later steps, eager work between the replays; two graphs with a workspace
    each; a call on a stream of the caller's."""
    rr = rrmod()
    note("captured step")
    rng = np.random.default_rng(13)
    H, Hkv, d, page, B = 8, 2, 64, 16, 4
    lens = [100, 1, 500, 64]
    c = Cache(rng, lens, Hkv, d, page, "bf16", spare=20, width=3)
    free = sorted(set(range(c.K.shape[0])) - set(int(x) for row, n in zip(c.table, lens) for x in row[:-(-n // page)]))
    for b, n in enumerate(lens):
        for j in range(-(-n // page), c.table.shape[1]):
            c.table[b, j] = free.pop() if free and j < -(-n // page) + 2 else -1
    Kc, Vc, table, lengths = c.args()
    f = torch.from_numpy(10000.0 ** (-np.arange(0, d, 2) / d)).to(DEV)
    k1, v1, q1 = (torch.zeros((B, h, d), dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, H))
    q = torch.empty((B, H, d), dtype=torch.bfloat16, device=DEV)
    O, O2 = (torch.empty((B, 1, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    prefix = _i32(c.table[2, :2])
    ws = rr.paged_workspace(q.view(B, 1, H, d), Kc, table)
    ws2 = rr.paged_workspace(q.view(B, 1, H, d), Kc, table, n_prefix=0)

    def step(out, w):
        lengths.add_(1)
        rr.cache_append(k1, v1, Kc, Vc, table, lengths, freqs=f, Q=q1, Q_out=q)
        rr.paged_attention(q.view(B, 1, H, d), Kc, Vc, table, lengths, out=out, workspace=w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rr.paged_attention(q.view(B, 1, H, d), Kc, Vc, table, lengths, out=O, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for out, w in ((O, ws), (O2, ws2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(out, w)
        graphs.append((g, out))
    torch.cuda.synchronize()
    lengths.copy_(_i32(lens))
    for i in range(6):
        for t in (k1, v1, q1):
            t.copy_(_values(rng, tuple(t.shape), "bf16"))
        g, out = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        c.lens = [n + i + 1 for n in lens]
        assert lengths.tolist() == c.lens
        _check(out, None, c.oracle(q.view(B, 1, H, d)), d, max(c.lens), "bf16")
        eager = rr.paged_attention(q.view(B, 1, H, d), Kc, Vc, table, lengths)
        side.wait_stream(torch.cuda.current_stream())
        other = rr.paged_attention(q.view(B, 1, H, d), Kc, Vc, table, lengths, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(eager, out) and torch.equal(other, out)
    assert prefix.numel() == 2


def test_one_workspace_for_calls_of_many_shapes():
    """A workspace of the largest call serves smaller and larger ones in any
    order, and its first bytes are zero after each."""
    rr = rrmod()
    note("one workspace")
    rng = np.random.default_rng(15)
    calls = []
    for H, Hkv, d, lens, nq, k, prefix in ((8, 2, 128, [3000, 5, 900], 1, 0, 0), (4, 4, 64, [700], 3, 0, 0),
                                           (32, 2, 128, [2500, 40], 2, 0, 0), (8, 2, 64, [400] * 5, 1, 3, 0),
                                           (8, 2, 128, [1200 + 9 * i for i in range(9)], 1, 0, 1100)):
        c = Cache(rng, lens, Hkv, d, 64, "bf16")
        Q = _values(rng, (len(lens), nq, H, d), "bf16", 2.0)
        R = _i32(rng.integers(0, 6, size=(len(lens) * H * nq, k))) if k else None
        if prefix:
            pages = _i32(c.table[0, :-(-prefix // 64)])
            call = lambda ws, c=c, Q=Q, pages=pages, n=prefix: rr.prefix_attention(Q, *c.args(), pages, n, workspace=ws)  # noqa: E731
        else:
            call = lambda ws, c=c, Q=Q, R=R: rr.paged_attention(Q, *c.args(), routes=R, workspace=ws)  # noqa: E731
        ws = rr.paged_workspace(Q, c.K, _i32(c.table), routes=R, n_prefix=prefix)
        calls.append((call, ws, call(None)))
    largest = max((w for _, w, _ in calls), key=lambda w: w.numel())
    for i in (0, 4, 1, 2, 0, 3, 4, 2, 1, 0):
        call, _, want = calls[i]
        assert torch.equal(call(largest), want), i
        assert not largest[:2048].any()


def test_profiled_kinds():
    rr = rrmod()
    note("kernel kinds")
    rng = np.random.default_rng(14)
    c = Cache(rng, [40, 50], 1, 64, 16, "f32")
    Q = _values(rng, (2, 1, 2, 64), "f32")
    rr.profile_start()
    rr.cache_append(Q[:, 0, :1], Q[:, 0, :1], *c.args())
    rr.paged_attention(Q, *c.args())
    got = rr.profile_stop()
    assert got["append"][1] == 1 and got["paged"][1] == 1 and got["join"][1] <= 1
    assert got["append"][0] > 0 and got["paged"][0] > 0


# ------------------------------------------------------- batches and long runs

MANY = [
    # name, H, Hkv, d, dtype, cache, page, sequences, n_q, longest, prefix
    ("seventy", 8, 2, 128, "bf16", "bf16", 16, 70, 1, 300, 0),
    ("many_items", 8, 2, 64, "bf16", "bf16", 32, 300, 1, 400, 0),
    ("many_items_e4m3", 8, 2, 128, "bf16", "e4m3", 16, 300, 2, 200, 0),
    ("many_items_f32", 8, 4, 64, "f32", "f32", 16, 260, 1, 200, 0),
    ("many_rows", 16, 2, 128, "bf16", "bf16", 16, 300, 4, 200, 0),
    ("many_rows_e4m3", 16, 2, 64, "bf16", "e4m3", 16, 70, 4, 300, 0),
    ("prefix_seventy", 8, 2, 64, "bf16", "bf16", 16, 70, 1, 150, 200),
    ("prefix_many_items", 8, 2, 128, "bf16", "bf16", 16, 300, 1, 150, 333),
    ("prefix_many_rows", 16, 2, 128, "bf16", "bf16", 16, 70, 5, 150, 333),
    ("prefix_many_rows_items", 16, 2, 64, "bf16", "e4m3", 16, 300, 5, 100, 130),
    ("prefix_d256_rows", 8, 1, 256, "bf16", "bf16", 16, 70, 3, 100, 200),
    ("prefix_f32", 8, 2, 64, "f32", "f32", 16, 70, 2, 150, 200),
    ("prefix_many_rows_f32", 8, 2, 64, "f32", "f32", 16, 70, 4, 60, 100),
    ("prefix_many_rows_d256", 16, 2, 256, "bf16", "bf16", 16, 70, 2, 60, 300),
    ("prefix_rounds", 32, 8, 64, "bf16", "bf16", 16, 130, 16, 60, 200),
    ("prefix_rounds_narrow", 32, 8, 64, "bf16", "bf16", 16, 520, 4, 40, 150),
]


@pytest.mark.parametrize("case", MANY, ids=[c[0] for c in MANY])
def test_many_sequences(case):
    """More sequences than a wave has lanes or a workgroup threads, more items
    than workgroups, more splits of a prefix than workgroups: outputs of some
    sequences against the oracle, of all of them against a call for each."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, B, nq, longest, prefix = case
    note(f"many sequences {case}")
    rng = np.random.default_rng(B + d + nq)
    lens = rng.integers(0, longest, size=B)
    lens[rng.random(B) < 0.2] = 0
    lens[-1], lens[B // 2] = longest, 1
    kw = {}
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, page, cache, prefix, lens.tolist())
        kw = dict(prefix_pages=pages, n_prefix=prefix)
    else:
        c = Cache(rng, lens.tolist(), Hkv, d, page, cache)
    Q = _values(rng, (B, nq, H, d), dtype, 2.0)
    lse = torch.empty((B, nq, H), device=DEV)
    Kc, Vc, table, lengths = c.args()

    def call(sel, lse=None):
        if prefix:
            return rr.prefix_attention(Q[sel], Kc, Vc, table[sel], lengths[sel], _i32(pages), prefix, lse=lse, **c.kw())
        return rr.paged_attention(Q[sel], Kc, Vc, table[sel], lengths[sel], lse=lse, **c.kw())

    O = call(slice(0, B), lse=lse)
    torch.cuda.synchronize()
    some = sorted({0, 1, B // 2, B - 1, *rng.integers(0, B, size=4).tolist()})
    whole = c.table, c.lens
    c.table, c.lens = c.table[some], [c.lens[b] for b in some]
    ref = c.oracle(Q[some], **kw)
    c.table, c.lens = whole
    rows = nq * H // Hkv * (B if prefix else 1)
    _check(O[some], lse[some], ref, d, max(c.lens), dtype, rows)
    # one call for each part of the batch: other runs and splits.  Both are off
    # by (err + 2^-8) * W + 2^-8 |o| at most for bf16, W and |o| <= max |v| < 6;
    # err (scores of at most 100, 350 tokens) stays below 2^-9
    parts = torch.cat([call(slice(b, min(b + 61, B))) for b in range(0, B, 61)])
    torch.cuda.synchronize()
    loose = 2 * (2.0 ** -9 + (2.0 ** -7 if dtype == "bf16" else 0.0))
    assert float((O.double() - parts.double()).abs().max()) <= loose * 6


LONG = [
    # name, H, Hkv, d, dtype, cache, lengths, n_q, prefix (pages of one token)
    ("narrow", 4, 4, 64, "bf16", "bf16", [22000, 21000, 22001], 1, 0),
    ("wide", 16, 4, 64, "bf16", "bf16", [22000, 21000, 22001], 5, 0),
    ("wide_e4m3", 16, 4, 64, "bf16", "e4m3", [22000, 300, 42001], 5, 0),
    ("prefix", 8, 4, 64, "bf16", "bf16", [7 * i for i in range(40)], 4, 40000),
    ("prefix_f32", 4, 2, 64, "f32", "f32", [7, 0, 30], 2, 70000),
]


@pytest.mark.parametrize("case", LONG, ids=[c[0] for c in LONG])
def test_more_pages_than_are_held_at_a_time(case):
    """Pages of one token, and runs of more of them than a workgroup holds the
    numbers of."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, lens, nq, prefix = case
    note(f"many pages {case}")
    rng = np.random.default_rng(len(name))
    B = len(lens)
    Q = _values(rng, (B, nq, H, d), dtype, 2.0)
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, 1, cache, prefix, lens)
        O = rr.prefix_attention(Q, *c.args(), _i32(pages), prefix, **c.kw())
    else:
        c, pages = Cache(rng, lens, Hkv, d, 1, cache), None
        O = rr.paged_attention(Q, *c.args(), **c.kw())
    torch.cuda.synchronize()
    some = [0, B - 1]
    c.table, c.lens = c.table[some], [c.lens[b] for b in some]
    ref = c.oracle(Q[some], prefix_pages=pages, n_prefix=prefix)
    _check(O[some], None, ref, d, max(c.lens), dtype, nq * H // Hkv * (B if prefix else 1))


@pytest.mark.parametrize("cache,nq", [("bf16", 6), ("e4m3", 1), ("e4m3", 6)])
def test_offsets_past_32_bits_of_other_bodies(cache, nq):
    """The last pages of pools of more than 2^31 elements, for more query rows
    and for 8-bit caches."""
    rr = rrmod()
    note(f"large pools {cache} {nq}")
    Hkv, d, page = 2, 128, 64
    n_pages = (1 << 31) // (Hkv * page * d) + 30
    rng = np.random.default_rng(2)
    kw = {}
    if cache == "e4m3":
        Kc, Vc = (torch.zeros((n_pages, Hkv, page, d), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
        scales = [np.array([0.01, 0.02], np.float32), np.array([0.03, 0.01], np.float32)]
        kw = dict(k_scale=torch.from_numpy(scales[0]).to(DEV), v_scale=torch.from_numpy(scales[1]).to(DEV))
    else:
        Kc, Vc = (torch.zeros((n_pages, Hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens = [200, 70]
    table = np.array([[n_pages - 1, 5, n_pages - 3, n_pages - 2], [n_pages - 20, n_pages - 21, 0, 0]])
    K, V = (_values(rng, (270, Hkv, d), "bf16") for _ in range(2))
    rr.cache_append(K, V, Kc, Vc, _i32(table), _i32(lens), seq_start=_i32([0, 200, 270]), **kw)
    Q = _values(rng, (2, nq, 8, d), "bf16", 2.0)
    O = rr.paged_attention(Q, Kc, Vc, _i32(table), _i32(lens), **kw)
    torch.cuda.synchronize()
    used = sorted(set(table.flatten().tolist()))
    small = np.searchsorted(used, table)
    at = torch.tensor(used, device=DEV)
    pick = (lambda x: _np(x.view(torch.uint8)[at].view(E4M3))) if cache == "e4m3" else (lambda x: _np(x[at]))
    okw = dict(k_scale=scales[0], v_scale=scales[1]) if kw else {}
    ref = op.attention(_np(Q), pick(Kc), pick(Vc), small, lens, **okw)
    _check(O, None, ref, d, 200, "bf16", nq * 4)


CUT = [
    # name, H, Hkv, d, dtype, cache, page, lengths, n_q
    ("rows_16", 16, 1, 128, "bf16", "bf16", 16, [3000], 1),
    ("rows_17", 17, 1, 128, "bf16", "bf16", 16, [2000, 0, 40], 1),
    ("rows_32", 32, 1, 64, "bf16", "bf16", 64, [5000, 1], 1),
    ("rows_32_e4m3", 16, 2, 128, "bf16", "e4m3", 16, [2500, 700, 3], 4),
    ("rows_24_e4m3_d64", 12, 1, 64, "bf16", "e4m3", 16, [2500], 2),
    ("rows_33", 33, 1, 128, "bf16", "bf16", 16, [1800, 100], 1),
    ("rows_90", 6, 2, 128, "bf16", "bf16", 48, [1500, 20, 300], 30),
    ("rows_128_e4m3", 8, 1, 128, "bf16", "e4m3", 64, [2000], 16),
    ("rows_200", 8, 2, 64, "bf16", "bf16", 64, [1000, 700], 50),
    ("rows_40_d256", 8, 1, 256, "bf16", "bf16", 32, [1600, 900], 5),
    ("rows_12_d256", 12, 1, 256, "bf16", "e4m3", 32, [3000], 1),
    ("rows_15_f32", 6, 2, 64, "f32", "f32", 48, [3000, 900, 2], 5),
    ("rows_32_f32", 16, 2, 128, "f32", "f32", 16, [1500, 700], 4),
    ("rows_70_f32", 14, 1, 64, "f32", "f32", 16, [900, 80], 5),
    ("rows_in_all_2560", 32, 4, 64, "bf16", "bf16", 16, [700, 3, 400, 520, 0], 16),
    ("rows_in_all_2064_d256", 16, 2, 256, "bf16", "e4m3", 16, [500, 30, 260], 43),
    ("rows_in_all_2048_f32", 16, 2, 128, "f32", "f32", 48, [400, 333, 18, 1], 32),
]


@pytest.mark.parametrize("case", CUT, ids=[c[0] for c in CUT])
def test_few_items_cut_into_many_parts(case):
    """Parts joined by the last workgroup or by a second launch, some items
    whole; newest tokens that are not finite reach their own rows alone."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, lens, nq = case
    note(f"cut {case}")
    rng = np.random.default_rng(sum(lens) + H)
    c = Cache(rng, lens, Hkv, d, page, cache)
    Q = _values(rng, (len(lens), nq, H, d), dtype, 2.0)
    lse = torch.empty((len(lens), nq, H), device=DEV)
    args = c.args()
    ws = rr.paged_workspace(Q, args[0], args[2])
    O = rr.paged_attention(Q, *args, lse=lse, workspace=ws, **c.kw())
    torch.cuda.synchronize()
    want = c.oracle(Q)
    _check(O, lse, want, d, max(lens), dtype, nq * H // Hkv)
    assert not ws[:2048].any()
    assert torch.equal(rr.paged_attention(Q, *args, workspace=ws, **c.kw()), O)
    if nq > 1:
        c.put(0, lens[0] - 1, *(np.full((1, Hkv, d), math.nan) for _ in range(2)))
        P = rr.paged_attention(Q, *args, workspace=ws, **c.kw())
        torch.cuda.synchronize()
        _check(P[:, :nq - 1], None, tuple(x[:, :nq - 1] for x in want), d, max(lens), dtype, nq * H // Hkv)
        assert not P[0, nq - 1].isfinite().any()


def test_captured_prefix_and_routes():
    """Calls with a prefix and along routes, captured and replayed with later
    lengths, eager calls in the same workspace between the replays."""
    rr = rrmod()
    note("captured prefix and routes")
    rng = np.random.default_rng(31)
    H, Hkv, d, page, prefix, B, nq = 8, 2, 128, 16, 150, 9, 2
    c, pages = _prefix_cache(rng, Hkv, d, page, "bf16", prefix, [60 + 13 * i for i in range(B)])
    full = list(c.lens)
    table = c.table.copy()
    table[:, :prefix // page] = pages[:prefix // page]
    c.table = table
    Kc, Vc, tab, lengths = c.args()
    Q = _values(rng, (B, nq, H, d), "bf16", 2.0)
    pg = _i32(pages)
    R = rng.integers(0, 12, size=(B * H * nq, 5))
    routes = _i32(R)
    ws = rr.paged_workspace(Q, Kc, tab, n_prefix=prefix)
    if rr.paged_workspace(Q, Kc, tab, routes=routes, n_recent=1).numel() > ws.numel():
        ws = rr.paged_workspace(Q, Kc, tab, routes=routes, n_recent=1)
    O1, O2 = (torch.empty_like(Q) for _ in range(2))
    rr.prefix_attention(Q, Kc, Vc, tab, lengths, pg, prefix, out=O1, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rr.prefix_attention(Q, Kc, Vc, tab, lengths, pg, prefix, out=O1, workspace=ws)
        rr.paged_attention(Q, Kc, Vc, tab, lengths, routes=routes, n_recent=1, out=O2, workspace=ws)
    for i in range(4):
        c.lens = [n - 7 * i for n in full]
        lengths.copy_(_i32(c.lens))
        Q.copy_(_values(rng, tuple(Q.shape), "bf16", 2.0))
        g.replay()
        torch.cuda.synchronize()
        _check(O1, None, c.oracle(Q, prefix_pages=pages, n_prefix=prefix), d, max(full), "bf16", B * nq * 4)
        _check(O2, None, c.oracle(Q, routes=R, n_recent=1), d, max(full), "bf16")
        assert torch.equal(rr.prefix_attention(Q, Kc, Vc, tab, lengths, pg, prefix, workspace=ws), O1)
        assert torch.equal(rr.paged_attention(Q, Kc, Vc, tab, lengths, routes=routes, n_recent=1, workspace=ws), O2)
