"""GPU parity of the calls on page tables (cache_fork, cache_resize,
cache_compact) against the oracle, entry by entry: whole numbers and copied
bytes, equal."""
import sys

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
BAD = [-1, -7, 2 ** 31 - 1, -2 ** 31]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)
    yield


def rrmod():
    from paper_2609_07306_amd import routerelay
    return routerelay


def note(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _i32(x):
    return torch.tensor(np.array(x, np.int64), dtype=torch.int32, device=DEV)


def _state(rng, B, width, n_pages, page, shared=0.3, full=0.7, bad=True):
    """A table whose rows hold pages of their own and of earlier rows', as counted."""
    order = list(rng.permutation(n_pages))
    table, lengths, refs = [], [], [0] * n_pages
    for b in range(B):
        n = int(rng.integers(0, int(width * full) + 1))
        row = [int(rng.choice(BAD)) if bad else -1 for _ in range(width)]
        if b and rng.random() < shared:
            o = int(rng.integers(0, b))
            n = min(n, -(-lengths[o] // page))
            row[:n] = table[o][:n]
        else:
            n = min(n, max(0, len(order) - 2 * B))
            row[:n] = [int(order.pop()) for _ in range(n)]
        for e in row[:n]:
            refs[e] += 1
        table.append(row)
        lengths.append(max(0, n * page - int(rng.integers(0, page))) if n else 0)
    for p in order[:len(order) // 4]:
        refs[p] += int(rng.integers(0, 3))  # held apart from any sequence
    return table, lengths, refs


def _pools(rng, n, shape, dtype):
    bits = torch.from_numpy(rng.integers(0, 256, size=(n, int(np.prod(shape)) * TYPE[dtype].itemsize), dtype=np.uint8)).to(DEV)
    return [x.clone().view(TYPE[dtype]).view(shape) for x in bits]


def _bits(t):
    return t.view(torch.uint8).cpu().numpy()


# ------------------------------------------------------------------- fork

@pytest.mark.parametrize("B,width,n_pages", [(1, 1, 1), (1, 9, 20), (2, 3, 10), (16, 33, 300), (65, 7, 400), (300, 129, 9000),
                                             (1100, 5, 4000), (4096, 3, 9000)])
@pytest.mark.parametrize("kind", ["any", "groups", "ends", "stay", "swap"])
def test_fork(B, width, n_pages, kind):
    rr = rrmod()
    note("fork", B, width, n_pages, kind)
    rng = np.random.default_rng(B * width)
    table, lengths, refs = _state(rng, B, width, n_pages, 16)
    parent = {"any": rng.integers(0, B, B), "groups": np.arange(B) // 4 * 4, "stay": np.arange(B),
              "ends": np.where(rng.random(B) < 0.5, np.arange(B), rng.choice([-1, B, 2 ** 31 - 1, -2 ** 31], B)),
              "swap": np.arange(B)[::-1].copy()}[kind]
    t, n, r = _i32(table), _i32(lengths), _i32(refs)
    rr.cache_fork(t, n, r, _i32(parent))
    want = serving.fork(table, lengths, refs, [int(p) for p in parent])
    for got, exact in zip((t, n, r), want):
        assert got.tolist() == exact
    if kind == "stay":
        assert t.tolist() == table and r.tolist() == refs


@pytest.mark.parametrize("B,width,n_pages", [(5, 2049, 12000), (1, 2048, 2100), (64, 2500, 60000), (130, 2065, 90000),
                                             (1638, 2051, 400000), (1639, 2051, 400000), (2731, 65, 40000)])
@pytest.mark.parametrize("kind", ["any", "groups", "ends", "stay", "swap"])
def test_fork_of_wide_tables(B, width, n_pages, kind):
    """Eight columns a workgroup where they are many, with some left over and numbers
    of workgroups that the XCDs do not share evenly; the most sequences that eight and
    four columns take, and one more."""
    rr = rrmod()
    note("fork wide", B, width, n_pages, kind)
    rng = np.random.default_rng(B * width)
    # rows of their own pages or an earlier row's, of any length, as counted
    table, lengths = np.full((B, width), -1, np.int64), np.zeros(B, np.int64)
    order, at = rng.permutation(n_pages), 0
    for b in range(B):
        n = int(rng.integers(0, width + 1)) if b % 7 else width
        if b and rng.random() < 0.6:
            o = int(rng.integers(max(0, b - 3), b))
            n = min(n, int(lengths[o]))
            table[b, :n] = table[o, :n]
        else:
            n = min(n, n_pages - at, max(width // 9, n_pages // B))
            table[b, :n] = order[at:at + n]
            at += n
        lengths[b] = n
        if n < width:
            table[b, n] = rng.choice(BAD)
    counts = np.bincount(table[(table >= 0) & (table < n_pages)], minlength=n_pages)
    parent = {"any": rng.integers(0, B, B), "groups": np.arange(B) // 4 * 4, "stay": np.arange(B),
              "ends": np.where(rng.random(B) < 0.5, np.arange(B), rng.choice([-1, B, 2 ** 31 - 1, -2 ** 31], B)),
              "swap": np.arange(B)[::-1].copy()}[kind]
    there = (parent >= 0) & (parent < B)
    rows = np.where(there[:, None], table[np.where(there, parent, 0)], -1)
    refs = np.bincount(rows[(rows >= 0) & (rows < n_pages)], minlength=n_pages) + 3  # (three held apart)
    t, n, r = _i32(table), _i32(lengths * 5), _i32(counts + 3)
    rr.cache_fork(t, n, r, _i32(parent))
    assert np.array_equal(t.cpu().numpy(), rows)
    assert np.array_equal(n.cpu().numpy(), np.where(there, 5 * lengths[np.where(there, parent, 0)], 0))
    assert np.array_equal(r.cpu().numpy(), refs)
    if B * width < 20000:
        want = serving.fork(table.tolist(), (5 * lengths).tolist(), (counts + 3).tolist(), [int(p) for p in parent])
        assert want[0] == rows.tolist() and want[2] == refs.tolist()


# ----------------------------------------------------------------- resize

def _resize(rr, table, lengths, refs, new, pools, page, missing=True, workspace=None):
    t, n, r = _i32(table), _i32(lengths), _i32(refs)
    before = [_bits(p).copy() for p in pools]
    handle = rr.Pools(pools[0::2], pools[1::2])
    out = rr.cache_resize(handle, t, n, r, _i32(new) if not isinstance(new, int) else new, workspace=workspace)
    news = [new] * len(lengths) if isinstance(new, int) else [int(x) for x in new]
    wt, wr, wm, copies = serving.resize(table, lengths, refs, news, page)
    assert t.tolist() == wt
    assert r.tolist() == wr
    assert out.tolist() == wm
    assert n.tolist() == lengths
    shape = pools[0].shape
    for p, old in zip(pools, before):
        exact = old.copy().reshape(*shape[:3], -1)
        for src, dst, places in copies:
            exact[dst, :, :places] = old.reshape(exact.shape)[src, :, :places]
        assert np.array_equal(_bits(p).reshape(exact.shape), exact)
    return wt, wr, wm, copies


@pytest.mark.parametrize("dtype,Hkv,page,d,n_pools", [("bf16", 2, 16, 64, 2), ("f32", 1, 7, 8, 4), ("e4m3", 3, 5, 8, 2),
                                                      ("e4m3", 2, 64, 128, 6), ("bf16", 1, 1, 8, 2), ("bf16", 8, 64, 128, 2),
                                                      ("bf16", 1, 3, 8, 130)])
@pytest.mark.parametrize("B,width", [(1, 1), (3, 8), (40, 12), (130, 5)])
@pytest.mark.parametrize("what", ["one", "some", "all", "none"])
def test_resize(dtype, Hkv, page, d, n_pools, B, width, what):
    rr = rrmod()
    note("resize", dtype, Hkv, page, d, n_pools, B, width, what)
    if B * width * n_pools * Hkv * page * d > 1 << 25:
        B = 3
    rng = np.random.default_rng(B * width + page)
    n_pages = 2 * B * width + 9
    table, lengths, refs = _state(rng, B, width, n_pages, page)
    cap = width * page
    if what == "one":
        new = 1
        lengths = [min(n + 1, cap) for n in lengths]
    elif what == "some":  # fewer or more tokens than before, some rows ended
        new = rng.integers(-2, 3 * page, B)
        lengths = [int(max(0, min(cap, n + rng.integers(-2 * page, 2 * page)))) * int(rng.random() < 0.9) for n in lengths]
    elif what == "all":
        lengths = [int(rng.integers(0, cap + 1)) for _ in lengths]
        new = np.array(lengths)
    else:
        new = 0
    pools = _pools(rng, n_pools, (n_pages, Hkv, page, d), dtype)
    _resize(rr, table, lengths, refs, new, pools, page)


@pytest.mark.parametrize("seed", range(6))
def test_resize_with_too_few_pages(seed):
    """Pages run out among missing and shared entries: who comes later is counted
    and keeps what it had; the call made again after pages came free provides."""
    rr = rrmod()
    note("resize too few", seed)
    rng = np.random.default_rng(100 + seed)
    B, width, page = 60, 6, 4
    table = [[-1] * width for _ in range(B)]
    lengths, refs, n_pages = [0] * B, [0] * 70, 70
    for g in range(0, B, 5):  # groups of five that share two pages, the second one partly filled
        a, b = 2 * (g // 5), 2 * (g // 5) + 1
        for i in range(g, g + 5):
            table[i][:2] = [a, b]
            lengths[i] = 7
            refs[a] += 1
            refs[b] += 1
    new = rng.integers(0, 7, B)
    lengths = [n + int(m) for n, m in zip(lengths, new)]
    for p in range(24 + 10 + 5 * seed, n_pages):
        refs[p] = 1  # (held apart)
    pools = _pools(rng, 2, (n_pages, 1, page, 8), "bf16")
    wt, wr, wm, _ = _resize(rr, table, lengths, refs, new, pools, page)
    assert sum(wm) > 0
    pools = _pools(rng, 2, (200, 1, page, 8), "bf16")
    _, _, wm, _ = _resize(rr, wt, lengths, wr + [0] * 130, new, pools, page)
    assert sum(wm) == 0


@pytest.mark.parametrize("B,width,n_new,page", [(3000, 2, 1, 16), (2, 1500, 5000, 4), (1025, 4, 9, 4), (64, 40, 100, 3),
                                                (1, 5000, 5000, 1), (2000, 6, 3, 2), (4, 9000, 20000, 3), (1200, 1100, 20, 8)])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("spare", [0.5, 1.0])
def test_resize_of_many(B, width, n_new, page, group, spare):
    """More sequences, entries and pages than a round of the workgroup takes;
    groups that share every page; enough free pages, and half of them."""
    rr = rrmod()
    note("resize many", B, width, n_new, page, group, spare)
    rng = np.random.default_rng(B + width)
    B = -(-B // group) * group
    held = width * page // 3 // page
    need = B * (-(-n_new // page) + 1)
    n_pages = int((B // group) * held + need * spare) + 3
    order = rng.permutation(n_pages)
    base = [[int(x) for x in order[i * held:(i + 1) * held]] for i in range(B // group)]
    table = [base[b // group] + [-1] * (width - held) for b in range(B)]
    refs = [0] * n_pages
    for row in table:
        for e in row[:held]:
            refs[e] += 1
    old = max(0, held * page - page // 2)
    lengths = [min(width * page, old + n_new)] * B
    pools = _pools(rng, 2, (n_pages, 1, page, 8), "e4m3")
    _resize(rr, table, lengths, refs, n_new, pools, page)


def test_resize_beyond_the_table():
    """Lengths below zero and past what the table can hold: as many entries as
    there are; counts of new tokens past everything."""
    rr = rrmod()
    note("resize beyond")
    rng = np.random.default_rng(8)
    page, width = 4, 3
    lengths = [-5, 13, 12, 2 ** 31 - 1, -2 ** 31, 100, 7, 7]
    new = [3, 2, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 87, -1, -2 ** 31]
    table = [[2 * b, 2 * b + 1, -1] for b in range(8)]
    refs = [1] * 16 + [0] * 20
    _resize(rr, table, lengths, refs, new, _pools(rng, 2, (36, 2, page, 16), "bf16"), page)


def test_resize_keeps_the_rest_of_a_copied_page():
    """The places from the first new token on hold what the page held."""
    rr = rrmod()
    note("resize places")
    rng = np.random.default_rng(9)
    for places in (1, 5, 15):
        pools = _pools(rng, 4, (6, 3, 16, 24), "bf16")
        _, _, _, copies = _resize(rr, [[3, -1], [3, -1]], [places + 1] * 2, [0, 0, 0, 2, 0, 0], 1, pools, 16)
        assert copies == [(3, 0, places)]
    pools = _pools(rng, 4, (6, 3, 16, 24), "bf16")  # a shared page that is written from its first place on
    assert _resize(rr, [[3, -1], [3, -1]], [4, 4], [0, 0, 0, 2, 0, 0], 4, pools, 16)[3] == []


# ---------------------------------------------------------------- compact

@pytest.mark.parametrize("n_pages", [1, 2, 5, 63, 64, 1000, 4096, 4097, 16384, 16385, 20000, 49152, 100003])
@pytest.mark.parametrize("used", [0.0, 0.02, 0.5, 0.97, 1.0])
def test_compact(n_pages, used):
    rr = rrmod()
    note("compact", n_pages, used)
    rng = np.random.default_rng(n_pages)
    refs = [int(x) for x in (rng.random(n_pages) < used) * rng.integers(1, 5, n_pages)]
    held = [p for p in range(n_pages) if refs[p]]
    width = 7
    table = [[int(rng.choice(held)) if held and rng.random() < 0.7 else int(rng.choice(BAD)) for _ in range(width)]
             for _ in range(30)]
    pools = _pools(rng, 2, (n_pages, 1, 3, 8), "e4m3") if n_pages > 4000 else _pools(rng, 4, (n_pages, 2, 5, 16), "bf16")
    before = [_bits(p).copy() for p in pools]
    t, r = _i32(table), _i32(refs)
    ids, n = rr.cache_compact(rr.Pools(pools[0::2], pools[1::2]), t, r)
    wt, wr, wids, wn = serving.compact(table, refs)
    assert n.tolist() == [wn] and ids.tolist() == wids and t.tolist() == wt and r.tolist() == wr
    for p, old in zip(pools, before):
        exact = old.copy()
        for src, dst in enumerate(wids):
            if dst >= 0 and dst != src:
                exact[dst] = old[src]
        assert np.array_equal(_bits(p), exact)
    # again: nothing moves
    ids, n = rr.cache_compact(rr.Pools(pools[0::2], pools[1::2]), t, r)
    assert n.tolist() == [wn] and t.tolist() == wt and r.tolist() == wr
    assert ids.tolist() == list(range(wn)) + [-1] * (n_pages - wn)


def test_compact_of_large_pages():
    """Pages past 2^31 bytes into the pools, in layers of one tensor each."""
    rr = rrmod()
    note("compact large")
    n_pages, Hkv, page, d = 300, 8, 4096, 128  # 8 MiB a page, 2.4 GiB a pool
    g = torch.Generator(device=DEV).manual_seed(3)
    pools = [torch.empty((n_pages, Hkv, page, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2)]
    marks = [[p[i, -1, -1].clone() for i in range(n_pages)] for p in pools]
    first = [[p[i, 0, 0].clone() for i in range(n_pages)] for p in pools]
    refs = [0] * n_pages
    for p in (0, 5, 298, 299, 297, 150):
        refs[p] = 1
    t, r = _i32([[299, 0, 5, 298, 297, 150]]), _i32(refs)
    ids, n = rr.cache_compact(rr.Pools(pools[0], pools[1]), t, r)
    assert t.tolist() == [[4, 0, 5, 3, 2, 1]] or t.tolist() == serving.compact([[299, 0, 5, 298, 297, 150]], refs)[0]
    for p, m, f in zip(pools, marks, first):
        for old, new in enumerate(ids.tolist()):
            if new >= 0:
                assert torch.equal(p[new, -1, -1], m[old]) and torch.equal(p[new, 0, 0], f[old])


def _random_pools(seed, n_pools, shape, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    size = int(np.prod(shape)) * TYPE[dtype].itemsize
    return [torch.empty(size, dtype=torch.uint8, device=DEV).random_(0, 256, generator=g).view(TYPE[dtype]).view(shape)
            for _ in range(n_pools)]


@pytest.mark.parametrize("dtype,Hkv,page,d,n_pages,n_pools", [
    ("bf16", 1, 16, 128, 90, 2),      # 256 pieces of 16 bytes: two pages a turn of a workgroup's threads
    ("bf16", 1, 17, 128, 90, 2),      # just over that: a page a turn
    ("f32", 2, 16, 64, 90, 4),        # a whole turn
    ("f32", 2, 16, 72, 90, 4),        # a turn and a part of one
    ("bf16", 3, 43, 136, 90, 6),      # some of them and a part
    ("e4m3", 2, 15, 72, 90, 2),       # rows of an odd number of 8 bytes: the same in pieces of these
    ("e4m3", 4, 16, 72, 90, 2),
    ("e4m3", 8, 64, 72, 40, 4),
    ("e4m3", 3, 50, 200, 40, 66),     # more pools than a launch takes
    ("bf16", 3, 43, 136, 40, 130),
    ("bf16", 1, 3, 8, 300, 130),
    ("bf16", 1, 17, 128, 20000, 2),   # more pages than a workgroup counts
    ("e4m3", 2, 31, 72, 33000, 4),
    ("bf16", 1, 17, 128, 17000, 66),
    ("bf16", 8, 4096, 128, 300, 2),   # past 2^31 bytes into a pool
])
@pytest.mark.parametrize("used", [0.05, 0.5, 0.9])
def test_compact_moves_whole_pages(dtype, Hkv, page, d, n_pages, n_pools, used):
    """Every byte of every pool, pages of all sizes of the copies."""
    rr = rrmod()
    note("compact whole", dtype, Hkv, page, d, n_pages, n_pools, used)
    rng = np.random.default_rng(n_pages + page)
    refs = (rng.random(n_pages) < used) * rng.integers(1, 5, n_pages)
    refs[-1] = 2
    held = np.nonzero(refs)[0]
    table = rng.choice(held, (25, 9))
    table[rng.random(table.shape) < 0.3] = -1
    pools = _random_pools(page, n_pools, (n_pages, Hkv, page, d), dtype)
    t, r = _i32(table), _i32(refs)
    handle = rr.Pools(pools[0::2], pools[1::2])
    before = [p.view(torch.uint8).clone() for p in pools]
    ids, n = rr.cache_compact(handle, t, r)
    wt, wr, wids, wn = serving.compact(table.tolist(), refs.tolist())
    assert n.tolist() == [wn] and ids.tolist() == wids and t.tolist() == wt and r.tolist() == wr
    src = [p for p, to in enumerate(wids) if to >= 0 and to != p]
    assert src
    dst = torch.tensor([wids[p] for p in src], device=DEV)
    for p, old in zip(pools, before):
        old[dst] = old[torch.tensor(src, device=DEV)]  # (sources lie behind all destinations)
        assert torch.equal(p.view(torch.uint8), old)


@pytest.mark.parametrize("dtype,Hkv,page,d,n_pools", [
    ("e4m3", 2, 28, 72, 2), ("e4m3", 2, 29, 72, 2),    # 504 and 522 pieces of 8 bytes: pages together, and one a unit
    ("e4m3", 8, 64, 72, 4), ("e4m3", 16, 64, 72, 2),   # three units, five
    ("bf16", 3, 61, 136, 66), ("bf16", 2, 16, 128, 130), ("f32", 8, 64, 128, 2), ("bf16", 1, 33, 128, 2),
])
@pytest.mark.parametrize("group", [2, 5])
def test_resize_copies_parts_of_large_pages(dtype, Hkv, page, d, n_pools, group):
    """Groups just forked write their first tokens behind any number of places."""
    rr = rrmod()
    note("resize parts", dtype, Hkv, page, d, n_pools, group)
    rng = np.random.default_rng(page * group)
    places = [1, page - 1, page // 2, page, 3, 2 * page, page + 1, 2 * page - 1]  # tokens of the groups
    B, width = group * len(places), 4
    table, refs, at = [], [], 0
    for n in places:
        held = -(-n // page)
        row = list(range(at, at + held)) + [-1] * (width - held)
        at += held
        refs += [group] * held
        table += [list(row) for _ in range(group)]
    n_pages = at + 2 * B
    refs += [0] * (n_pages - at)
    new = rng.integers(1, page + 2, B)
    lengths = [n + int(m) for n, m in zip(np.repeat(places, group), new)]
    pools = _random_pools(page, n_pools, (n_pages, Hkv, page, d), dtype)
    copies = _resize(rr, table, lengths, refs, new, pools, page)[3]
    assert len(copies) == 6 * (group - 1)  # (of the groups whose last page is not full)


# -------------------------------------------------------------- all of it

def test_a_long_life_of_a_cache():
    """Forks, growth, rejected drafts, ends and compactions one after the other on
    one table and workspace, every step as the oracle's; at the end everything
    ends and every page is free."""
    rr = rrmod()
    note("a long life")
    rng = np.random.default_rng(77)
    B, width, page, n_pages = 24, 10, 8, 400
    pools = _pools(rng, 2, (n_pages, 2, page, 16), "bf16")
    handle = rr.Pools(pools[0::2], pools[1::2])
    ws = rr.pages_workspace(handle)
    table, lengths, refs = [[-1] * width for _ in range(B)], [0] * B, [0] * n_pages
    t, n, r = _i32(table), _i32(lengths), _i32(refs)
    for step in range(40):
        if step % 7 == 3:
            parent = np.where(rng.random(B) < 0.6, np.arange(B), rng.integers(-1, B, B))
            rr.cache_fork(t, n, r, _i32(parent))
            table, lengths, refs = serving.fork(table, lengths, refs, [int(p) for p in parent])
        if step % 9 == 8:
            old = [_bits(p).copy() for p in pools]
            ids, used = rr.cache_compact(handle, t, r, workspace=ws)
            table, refs, wids, wn = serving.compact(table, refs)
            assert ids.tolist() == wids and used.tolist() == [wn]
            for p, o in zip(pools, old):
                exact = o.copy()
                for src, dst in enumerate(wids):
                    if dst >= 0:
                        exact[dst] = o[src]
                assert np.array_equal(_bits(p), exact)
        new = rng.integers(0, 12, B)
        lengths = [int(max(0, x - rng.integers(0, 6))) for x in lengths]
        lengths = [min(width * page, x + int(m)) if rng.random() < 0.95 else 0 for x, m in zip(lengths, new)]
        if step == 39:
            lengths = [0] * B
        n.copy_(_i32(lengths))
        old = [_bits(p).copy() for p in pools]
        missing = rr.cache_resize(handle, t, n, r, _i32(new), workspace=ws)
        table, refs, wm, copies = serving.resize(table, lengths, refs, [int(x) for x in new], page)
        assert missing.tolist() == wm and sum(wm) == 0
        assert (t.tolist(), n.tolist(), r.tolist()) == (table, lengths, refs)
        for p, o in zip(pools, old):
            for src, dst, places in copies:
                o.reshape(n_pages, 2, page, -1)[dst, :, :places] = o.reshape(n_pages, 2, page, -1)[src, :, :places]
            assert np.array_equal(_bits(p), o)
        # counts and tables agree
        count = [0] * n_pages
        for row in table:
            for e in row:
                if e >= 0:
                    count[e] += 1
        assert count == refs
    assert refs == [0] * n_pages
