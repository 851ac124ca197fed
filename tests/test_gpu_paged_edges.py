"""The paged cache at its edges, against binary64: values that are not finite
behind scores so low that their weights are 0, queries before their sequence's
first token beside others that see such values, routes without slots, the
precision of the weights, and every row of large batches.  Tolerances as in
test_gpu_paged."""
import functools
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import DEV, MANY, TYPE, Cache, _check, _i32, _prefix_cache, _values, note, rrmod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)
    yield


LOW = [
    # name, H, Hkv, d, dtype, cache, page, lengths, n_q, prefix, which tokens of the first have low scores
    ("wave_bf16", 8, 2, 128, "bf16", "bf16", 16, [128, 3], 1, 0, lambda u: u // 32 == 1),
    ("wave_e4m3", 8, 2, 64, "bf16", "e4m3", 16, [128, 3], 1, 0, lambda u: u // 32 == 1),
    ("wave_f32", 4, 2, 64, "f32", "f32", 16, [64, 3], 1, 0, lambda u: u // 32 == 1),
    ("blocks_bf16", 32, 1, 128, "bf16", "bf16", 16, [128, 3], 1, 0, lambda u: u // 32 % 2 == 1),
    ("blocks_e4m3", 32, 1, 64, "bf16", "e4m3", 16, [128, 3], 1, 0, lambda u: u // 32 % 2 == 1),
    ("run_bf16", 8, 2, 128, "bf16", "bf16", 64, [8000, 3], 1, 0, lambda u: u < 3000),
    ("run_one_launch", 32, 8, 128, "bf16", "bf16", 64, [8000, 3], 1, 0, lambda u: u < 3000),
    ("run_e4m3", 32, 8, 128, "bf16", "e4m3", 64, [8000, 3], 1, 0, lambda u: u >= 5000),
    ("run_f32", 4, 4, 128, "f32", "f32", 48, [6000, 3], 1, 0, lambda u: u < 3000),
    ("run_rows_one_launch", 18, 1, 64, "bf16", "bf16", 64, [300] * 100, 1, 0, lambda u: u < 128),
    ("run_rows_two_launches", 64, 1, 128, "bf16", "bf16", 64, [6000, 3], 2, 0, lambda u: u < 3000),
    ("run_rows_e4m3", 64, 1, 64, "bf16", "e4m3", 64, [6000, 3], 2, 0, lambda u: u < 3000),
    ("run_rows_f32", 32, 1, 64, "f32", "f32", 64, [6000, 3], 2, 0, lambda u: u < 3000),
    ("run_rows_d256", 24, 1, 256, "bf16", "bf16", 64, [3000, 3], 1, 0, lambda u: u < 1500),
    ("prefix_bf16", 4, 2, 128, "bf16", "bf16", 16, [268, 3], 1, 208, lambda u: u < 208),
    ("prefix_rows", 32, 1, 128, "bf16", "bf16", 16, [1200, 3], 2, 1008, lambda u: u < 1008),
    ("prefix_rows_e4m3", 32, 1, 64, "bf16", "e4m3", 16, [1200, 3], 1, 1008, lambda u: u < 1008),
    ("behind_prefix_f32", 8, 2, 64, "f32", "f32", 16, [268, 3], 1, 208, lambda u: 208 <= u < 267),
    ("behind_prefix_rows", 32, 1, 64, "bf16", "bf16", 16, [1200, 3], 1, 1008, lambda u: u >= 1008),
]


@pytest.mark.parametrize("case,infinite_keys", [
    pytest.param(c, x, id=c[0] + ("_infinite_keys" if x else "")) for c in LOW for x in (False, True)
    if not (x and c[5] == "e4m3")])
def test_values_that_are_not_finite_behind_low_scores(case, infinite_keys):
    """Where a query sees a value that is not finite that feature of its output
    is not either, also if the score is more than 350 below the others, so that
    the weight is 0 wherever it is formed: in another wave, another run, the
    prefix or behind it.  infinite_keys: those scores are -inf (e4m3 holds none)."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, lens, nq, prefix, low = case
    n, B = lens[0], len(lens)
    note(f"low scores {case[:-1]} {infinite_keys}")
    rng = np.random.default_rng(len(name) + d)
    kw, okw = {}, {}
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, page, cache, prefix, [n - prefix, lens[1]])
        kw, okw = dict(prefix_pages=_i32(pages), n_prefix=prefix), dict(prefix_pages=pages, n_prefix=prefix)
    else:
        c, pages = Cache(rng, lens, Hkv, d, page, cache), []
    table = c.table
    c.table = table.copy()
    c.table[0, :len(pages)] = pages
    at = np.flatnonzero([low(u) for u in range(n - nq + 1)])
    for run in np.split(at, np.flatnonzero(np.diff(at) > 1) + 1):
        # queries lie along (1, 1, ...): q.k of these keys is about -4.4 * 10 * d, that of the others 10 sqrt(d)
        # at random; at 1 / sqrt(d) 352 (d = 64) to 704 below 0 against 10 at random
        key = np.full((len(run), Hkv, d), -4.4)
        if infinite_keys:
            key[..., 5] = -math.inf
        c.put(0, run[0], key, rng.standard_normal((len(run), Hkv, d)))
    key, bad = np.full((1, Hkv, d), -4.4), rng.standard_normal((1, Hkv, d))
    if infinite_keys:
        key[..., 5] = -math.inf
    bad[..., 3], bad[..., d - 1] = (math.nan if cache == "e4m3" else -math.inf), math.nan
    c.put(0, at[len(at) // 2], key, bad)
    c.table = table
    Q = (10.0 + 0.1 * torch.from_numpy(rng.standard_normal((B, nq, H, d)))).to(TYPE[dtype]).to(DEV)
    lse = torch.empty((B, nq, H), device=DEV)
    call = rr.prefix_attention if prefix else rr.paged_attention
    O = call(Q, *c.args(), lse=lse, **kw, **c.kw())
    torch.cuda.synchronize()
    assert not O[0, ..., [3, d - 1]].isfinite().any()
    with np.errstate(invalid="ignore"):
        exact, elog, W, S = c.oracle(Q, **okw)
    keep = [f for f in range(d) if f not in (3, d - 1)]
    if infinite_keys:  # (the largest sum of |q_i k_i| over the finite keys: theirs is at most 4.5 |q|_1)
        S = np.minimum(S, 4.5 * 11 * d / math.sqrt(d))
    ref = exact[..., keep], elog, W[..., keep], S
    _check(O[..., keep], lse, ref, d, n, dtype, nq * H // Hkv * (B if prefix else 1))
    assert prefix or O[1:].isfinite().all()


NONE = [
    # name, H, Hkv, d, dtype, cache, lengths, n_q, prefix
    ("rows_144_bf16", 16, 1, 128, "bf16", "bf16", [3, 200], 9, 0),
    ("rows_144_e4m3", 16, 1, 64, "bf16", "e4m3", [3, 200], 9, 0),
    ("rows_40_d256", 8, 1, 256, "bf16", "bf16", [2, 70], 5, 0),
    ("rows_40_d256_e4m3", 8, 1, 256, "bf16", "e4m3", [2, 70], 5, 0),
    ("rows_24", 8, 1, 128, "bf16", "bf16", [2, 70], 3, 0),
    ("rows_12", 4, 1, 128, "bf16", "bf16", [1, 70], 3, 0),
    ("rows_24_f32", 8, 1, 64, "f32", "f32", [2, 70], 3, 0),
    ("cut_rows_256", 64, 1, 64, "bf16", "bf16", [2], 4, 0),
    ("prefix_rows_288", 16, 1, 128, "bf16", "bf16", [3, 200], 9, 60),
    ("prefix_rows_f32", 8, 1, 64, "f32", "f32", [2, 200], 3, 60),
]


@pytest.mark.parametrize("case", NONE, ids=[c[0] for c in NONE])
def test_queries_before_the_first_token_among_others(case):
    """More new queries than tokens: those before the first token get zeros
    and a logarithm of -inf, whatever values the others see."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, lens, nq, prefix = case
    note(f"queries before the first token {case}")
    rng = np.random.default_rng(len(name) + d)
    kw, at = {}, None
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, 16, cache, prefix, [max(x - prefix, 0) for x in lens])
        c.lens = list(lens)
        kw = dict(prefix_pages=_i32(pages), n_prefix=prefix)
        at = c.table, c.lens
        c.table = np.tile(np.concatenate([pages, [-1]]), (len(lens), 1))
    else:
        c = Cache(rng, lens, Hkv, d, 16, cache)
    bad = rng.standard_normal((1, Hkv, d))
    bad[..., 1], bad[..., 7] = (math.nan if cache == "e4m3" else math.inf), math.nan
    c.put(0, 0, rng.standard_normal((1, Hkv, d)), bad)
    if at:
        c.table, c.lens = at
    Q = _values(rng, (len(lens), nq, H, d), dtype)
    lse = torch.full((len(lens), nq, H), 7.0, device=DEV)
    call = rr.prefix_attention if prefix else rr.paged_attention
    O = call(Q, *c.args(), lse=lse, **kw, **c.kw())
    torch.cuda.synchronize()
    none = nq - lens[0]
    assert none > 0 and not O[0, :none].any()
    assert (lse[0, :none] == -math.inf).all() and lse[0, none:].isfinite().all()
    assert not O[0, none:][..., [1, 7]].isfinite().any()
    keep = [f for f in range(d) if f not in (1, 7)]
    assert O[0][..., keep].isfinite().all()


@pytest.mark.parametrize("H,Hkv,nq,dtype", [(8, 2, 1, "bf16"), (8, 1, 3, "bf16"), (4, 2, 2, "f32")])
def test_routes_without_slots(H, Hkv, nq, dtype):
    """Routes of no slots name no page: zeros, not attention over everything;
    with first or last pages besides, those alone."""
    rr = rrmod()
    note(f"routes without slots {H} {Hkv} {nq} {dtype}")
    rng = np.random.default_rng(nq)
    c = Cache(rng, [100, 1, 0, 333], Hkv, 64, 16, dtype)
    Q = _values(rng, (4, nq, H, 64), dtype)
    none = torch.empty((4 * H * nq, 0), dtype=torch.int32, device=DEV)
    lse = torch.full((4, nq, H), 7.0, device=DEV)
    side = torch.cuda.Stream()
    for stream in (None, side):
        for ws in (None, rr.paged_workspace(Q, c.K, _i32(c.table), routes=none)):
            out = torch.full_like(Q, 7.0)
            args = c.args()
            torch.cuda.synchronize()
            rr.paged_attention(Q, *args, routes=none, lse=lse, out=out, workspace=ws, stream=stream)
            torch.cuda.synchronize()
            assert not out.any() and (lse == -math.inf).all()
    O = rr.paged_attention(Q, *c.args(), routes=none, n_sink=1, n_recent=2, lse=lse)
    torch.cuda.synchronize()
    _check(O, lse, c.oracle(Q, n_sink=1, n_recent=2), 64, 333, dtype)
    assert torch.equal(O, rr.paged_attention(Q, *c.args(), n_sink=1, n_recent=2))


FINE = [
    # name, H, Hkv, d, dtype, cache, page, lengths, n_q, prefix
    ("rows_17", 17, 1, 128, "bf16", "bf16", 16, [3000, 700], 1, 0),
    ("rows_32", 32, 1, 64, "bf16", "bf16", 16, [3000, 700], 1, 0),
    ("rows_64", 16, 2, 128, "bf16", "bf16", 64, [3000, 700], 8, 0),
    ("rows_40_e4m3", 8, 1, 128, "bf16", "e4m3", 64, [2000, 900, 3], 5, 0),
    ("rows_64_d256", 8, 1, 256, "bf16", "bf16", 64, [1500], 8, 0),
    ("rows_64_d256_e4m3", 8, 1, 256, "bf16", "e4m3", 64, [1500], 8, 0),
    ("rows_32_many", 8, 2, 64, "bf16", "bf16", 64, [400 + i for i in range(40)], 8, 0),
    ("prefix_rows_64", 8, 2, 128, "bf16", "bf16", 16, [1200 + 20 * i for i in range(16)], 1, 1008),
    ("prefix_rows_60", 20, 1, 64, "bf16", "e4m3", 16, [1500, 1009, 1100], 1, 1008),
]


@pytest.mark.parametrize("case", FINE, ids=[c[0] for c in FINE])
def test_weights_of_up_to_64_rows_are_not_rounded_to_one_bf16(case):
    """Outputs of up to 64 rows a key head are as near as those of 16."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, lens, nq, prefix = case
    note(f"fine weights {case}")
    rng = np.random.default_rng(len(name) + d)
    kw, okw = {}, {}
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, page, cache, prefix, [x - prefix for x in lens])
        kw, okw = dict(prefix_pages=_i32(pages), n_prefix=prefix), dict(prefix_pages=pages, n_prefix=prefix)
    else:
        c = Cache(rng, lens, Hkv, d, page, cache)
    # (scores of a standard deviation of 0.3: every token counts, and outputs are small beside the values)
    Q = _values(rng, (len(lens), nq, H, d), dtype, 0.3)
    lse = torch.empty((len(lens), nq, H), device=DEV)
    call = rr.prefix_attention if prefix else rr.paged_attention
    O = call(Q, *c.args(), lse=lse, **kw, **c.kw())
    torch.cuda.synchronize()
    _check(O, lse, c.oracle(Q, **okw), d, max(lens), dtype, rows=16)


def _reference(c, Q, pages, prefix):
    """oracle.paged.attention without routes, on the device, a sequence at a time."""
    B, nq, H, d = Q.shape
    g, page = H // c.Hkv, c.page
    O, W = (torch.zeros(Q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, S = torch.full((B, nq, H), -math.inf, dtype=torch.float64, device=DEV), torch.zeros((B, nq, H), device=DEV)
    for b, n in enumerate(c.lens):
        if n == 0:
            continue
        u = np.arange(n)
        ids = c.table[b, u // page]
        if prefix:
            ids = np.where(u < prefix, np.asarray(pages)[np.minimum(u // page, len(pages) - 1)], ids)
        ids, at = torch.from_numpy(ids).to(DEV), torch.from_numpy(u % page).to(DEV)
        k, v = ((p.view(torch.uint8)[ids, :, at].view(p.dtype) if c.scales[0] is not None else p[ids, :, at]).double()
                for p in (c.K, c.V))
        if c.scales[0] is not None:
            k, v = (x * torch.from_numpy(s).to(DEV).double()[:, None] for x, s in zip((k, v), c.scales))
        k, v = k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()  # [H_kv, n, d]
        q = Q[b].double().view(nq, c.Hkv, g, d).transpose(0, 1).reshape(c.Hkv, nq * g, d)
        kt = k.transpose(1, 2).contiguous()
        s = q @ kt / math.sqrt(d)
        last = n - nq + torch.arange(nq, device=DEV).repeat_interleave(g)
        seen = torch.arange(n, device=DEV) <= last[:, None]
        s = s.masked_fill(~seen, -math.inf)
        sums = torch.logsumexp(s, -1)
        w = torch.where(seen, (s - sums[..., None]).exp(), 0.0)
        size = ((q.abs() @ kt.abs()).masked_fill(~seen, 0.0)).amax(-1) / math.sqrt(d)

        def rows(x):  # [H_kv, nq * g, ...] -> [nq, H, ...]
            return x.unflatten(1, (nq, g)).transpose(0, 1).flatten(1, 2)

        O[b], W[b], lse[b], S[b] = rows(w @ v), rows(w @ v.abs()), rows(sums), rows(size)
    return tuple(x.double().cpu().numpy() for x in (O, lse, W, S))


@pytest.mark.parametrize("case", MANY, ids=[c[0] for c in MANY])
def test_every_row_of_large_batches(case):
    """Every output and logarithm of batches of many sequences, items, rows and
    splits, each within its own tolerance."""
    rr = rrmod()
    name, H, Hkv, d, dtype, cache, page, B, nq, longest, prefix = case
    note(f"every row {case}")
    rng = np.random.default_rng(B + d + nq + 1)
    lens = rng.integers(0, longest, size=B)
    lens[rng.random(B) < 0.2] = 0
    lens[-1], lens[B // 2] = longest, 1
    kw, pages = {}, None
    if prefix:
        c, pages = _prefix_cache(rng, Hkv, d, page, cache, prefix, lens.tolist())
        kw = dict(prefix_pages=_i32(pages), n_prefix=prefix)
    else:
        c = Cache(rng, lens.tolist(), Hkv, d, page, cache)
    Q = _values(rng, (B, nq, H, d), dtype, 2.0)
    lse = torch.full((B, nq, H), 7.0, device=DEV)
    call = rr.prefix_attention if prefix else rr.paged_attention
    O = call(Q, *c.args(), lse=lse, **kw, **c.kw())
    torch.cuda.synchronize()
    _check(O, lse, _reference(c, Q, pages, prefix), d, max(c.lens), dtype, nq * H // Hkv * (B if prefix else 1))


def test_calls_at_once():
    """Calls of different shapes on two streams with a workspace each, not
    waiting for each other, give what they give alone."""
    rr = rrmod()
    note("calls at once")
    rng = np.random.default_rng(41)
    calls = []
    shapes = ((32, 8, 128, "bf16", [20000, 3, 700], 1, 0), (16, 2, 128, "bf16", [9000] * 3, 8, 0),
              (8, 2, 64, "e4m3", [1300 + i for i in range(20)], 1, 1008), (4, 2, 64, "f32", [6000, 40], 2, 0))
    for H, Hkv, d, cache, lens, nq, prefix in shapes:
        if prefix:
            c, pages = _prefix_cache(rng, Hkv, d, 16, cache, prefix, [x - prefix for x in lens])
        else:
            c, pages = Cache(rng, lens, Hkv, d, 16, cache), None
        Q = _values(rng, (len(lens), nq, H, d), "f32" if cache == "f32" else "bf16", 2.0)
        more = dict(prefix_pages=_i32(pages), n_prefix=prefix) if prefix else {}
        more.update(c.kw())
        ws = rr.paged_workspace(Q, c.K, _i32(c.table), n_prefix=prefix)
        call = rr.prefix_attention if prefix else rr.paged_attention
        args = c.args()
        calls.append((functools.partial(call, Q, *args, workspace=ws, **more), torch.empty_like(Q)))
    want = [call() for call, _ in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for (call, out), s in zip(calls, streams):
            call(out=out, stream=s)
    torch.cuda.synchronize()
    for (_, out), w in zip(calls, want):
        assert torch.equal(out, w)
