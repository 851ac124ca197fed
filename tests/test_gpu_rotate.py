"""GPU parity of the rotation by positions of several axes (rotate, and
cache_append with positions) against the binary64 oracle.

Tolerance, from the arithmetic (u = half a step of the output's type): the angle
is reduced in binary64 and rounded to binary32 in turns (at most 2^-26 turns
off: pi 2^-25 radians), sine and cosine and the two products and their sum round
to 2^-24 relative each or twice that: 8 * 2^-24 * (|x| + |y|) for partners x, y,
then u relative (e4m3: 2^-4, or half its smallest step, 2^-10)."""
import sys

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
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


def note(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _np(t):
    return t.double().cpu().numpy()


def _freqs(half):
    return 10000.0 ** (-np.arange(half) / max(1, half))


def _positions(rng, axes, n, real, top=50000):
    p = rng.integers(-20, top, size=(axes, n))
    return (p + rng.random(p.shape)).astype(np.float32) if real else p.astype(np.int32)


def _partners(x, rot, inter):
    """|x| + |partner| of every feature."""
    a = np.abs(x)
    out = a.copy()
    half = rot // 2
    i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if inter else (np.arange(half), np.arange(half, rot))
    out[..., i] = out[..., j] = a[..., i] + a[..., j]
    return out


def _check(got, x, exact, rot, inter, dtype):
    tol = 8 * 2.0 ** -24 * _partners(x, rot, inter) + 1.01 * HALF[dtype] * np.abs(exact) + 1e-30
    off = np.abs(got - exact)
    bad = np.argwhere(~(off <= tol))
    assert len(bad) == 0, f"{len(bad)} beyond tolerance, first {bad[0].tolist()}: {got[tuple(bad[0])]} vs " \
                          f"{exact[tuple(bad[0])]}"
    # what is not rotated is as it was
    assert np.array_equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,d,rot,inter,axes,real,tokens", [
    (1, 1, 8, 8, False, 1, False, 0), (1, 5, 64, 64, False, 3, False, 1), (37, 6, 64, 64, True, 2, False, 0),
    (37, 6, 64, 64, True, 2, True, 1), (300, 8, 128, 128, False, 3, False, 1), (300, 8, 128, 64, False, 3, True, 0),
    (65, 3, 256, 256, True, 4, False, 0), (65, 3, 40, 24, False, 2, False, 1), (65, 3, 40, 6, True, 2, False, 0),
    (33, 2, 1024, 1024, False, 3, False, 0), (33, 2, 1024, 2, False, 1, False, 1), (9, 70, 96, 94, False, 3, False, 0),
    (2500, 40, 128, 128, False, 3, False, 1), (7, 3, 128, 0, False, 1, False, 0),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate(dtype, n, H, d, rot, inter, axes, real, tokens, inverse):
    rr = rrmod()
    note("rotate", dtype, n, H, d, rot, inter, axes, real, tokens, inverse)
    rng = np.random.default_rng(n * d + rot + axes)
    shape = (n, H, d) if tokens == 0 else (H, n, d)
    X = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPE[dtype]).to(DEV)
    pos, f = _positions(rng, axes, n, real), _freqs(rot // 2)
    axis = rng.integers(0, axes, rot // 2).astype(np.int32)
    dev = [torch.from_numpy(a).to(DEV) for a in (pos, f, axis)]
    x = _np(X) if tokens == 0 else _np(X).transpose(1, 0, 2)
    exact = serving.rotate(x, pos, f, axis, inter, inverse)
    got = rr.rotate(X, dev[0], dev[1], axis=dev[2], tokens=tokens, interleaved=inter, inverse=inverse)
    _check(_np(got) if tokens == 0 else _np(got).transpose(1, 0, 2), x, exact, rot, inter, dtype)
    # in place: the same bits
    Y = X.clone()
    assert rr.rotate(Y, dev[0], dev[1], axis=dev[2], tokens=tokens, interleaved=inter, inverse=inverse, out=Y) is Y
    assert torch.equal(Y, got)
    # on one axis, without a list of them
    one = rr.rotate(X, dev[0][0].contiguous(), dev[1], tokens=tokens, interleaved=inter, inverse=inverse)
    exact = serving.rotate(x, pos[:1], f, None, inter, inverse)
    _check(_np(one) if tokens == 0 else _np(one).transpose(1, 0, 2), x, exact, rot, inter, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_axis_that_is_not_there_rotates_nothing(dtype):
    rr = rrmod()
    note("rotate axes outside", dtype)
    rng = np.random.default_rng(3)
    n, H, d = 40, 4, 64
    X = torch.from_numpy(rng.standard_normal((n, H, d)).astype(np.float32)).to(TYPE[dtype]).to(DEV)
    pos, f = _positions(rng, 2, n, False), _freqs(32)
    axis = rng.choice([0, 1, 2, 7, -1, 2 ** 31 - 1, -2 ** 31], 32).astype(np.int32)
    got = rr.rotate(X, torch.from_numpy(pos).to(DEV), torch.from_numpy(f).to(DEV), axis=torch.from_numpy(axis).to(DEV))
    _check(_np(got), _np(X), serving.rotate(_np(X), pos, f, axis), 64, False, dtype)
    still = np.isin(axis, [0, 1], invert=True)
    assert np.array_equal(_np(got)[..., :32][..., still], _np(X)[..., :32][..., still])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_views_and_rows_around_them(dtype, shift):
    """Rows of a fused projection into a part of a larger tensor, one input row
    for all heads; what lies between the rows of the output stays."""
    rr = rrmod()
    note("rotate views", dtype, shift)
    rng = np.random.default_rng(4)
    n, H, d = 130, 5, 64
    wide = torch.from_numpy(rng.standard_normal((n, 2 * H + 1, d + 8 * (1 + shift) + shift)).astype(np.float32))
    wide = wide.to(TYPE[dtype]).to(DEV)
    X = wide[:, 1:H + 1, shift:shift + d]
    pos, f = _positions(rng, 3, n, False), _freqs(32)
    axis = rng.integers(0, 3, 32).astype(np.int32)
    dev = [torch.from_numpy(a).to(DEV) for a in (pos, f, axis)]
    into = torch.full_like(wide, 77.0)
    out = into[:, H + 1:, shift:shift + d]
    rr.rotate(X, dev[0], dev[1], axis=dev[2], out=out)
    _check(_np(out), _np(X), serving.rotate(_np(X), pos, f, axis), 64, False, dtype)
    rest = into.clone()
    rest[:, H + 1:, shift:shift + d] = 77.0
    assert bool((rest == 77.0).all())
    same = X[:, :1].expand(n, H, d)
    got = rr.rotate(same, dev[0], dev[1], axis=dev[2])
    assert torch.equal(got, got[:, :1].expand(n, H, d).contiguous())
    assert torch.equal(got[:, 0], rr.rotate(X, dev[0], dev[1], axis=dev[2])[:, 0])


def test_far_positions_and_values_that_are_not_finite():
    rr = rrmod()
    note("rotate far positions")
    rng = np.random.default_rng(5)
    d = 64
    pos = np.array([[0, 1, 2 ** 20, 2 ** 24 + 1, 2 ** 30 + 7, -2 ** 31, 2 ** 31 - 1]], np.int32)
    n = pos.shape[1]
    X = torch.from_numpy(rng.standard_normal((n, 3, d)).astype(np.float32)).to(DEV)
    f = _freqs(32)
    got = rr.rotate(X, torch.from_numpy(pos).to(DEV), torch.from_numpy(f).to(DEV))
    # (position times frequency rounds to 2^-53 relative in either: 2^31 radians to 2^-22)
    exact = serving.rotate(_np(X), pos, f)
    more = 2 * 2.0 ** -52 * np.abs(pos[0].astype(np.float64))[:, None, None] * _partners(_np(X), d, False)
    assert np.all(np.abs(_np(got) - exact) <= 8 * 2.0 ** -24 * _partners(_np(X), d, False) + 2.0 ** -24 * np.abs(exact) + more)
    assert torch.equal(got[0], X[0])
    X[2, 1, 5] = float("inf")
    X[3, 0, 40] = float("nan")
    again = rr.rotate(X, torch.from_numpy(pos).to(DEV), torch.from_numpy(f).to(DEV))
    changed = ~((again == got) | (again.isnan() & got.isnan()))
    assert changed.nonzero().tolist() == [[2, 1, 5], [2, 1, 37], [3, 0, 8], [3, 0, 40]]


def test_gradient():
    """The inverse is the rotation's gradient: against autograd of the formula in
    binary64, and against differences of the rotation itself (linear, so a
    difference over a whole unit is off by its roundings alone)."""
    rr = rrmod()
    note("rotate gradient")
    rng = np.random.default_rng(6)
    n, H, d, rot = 19, 3, 64, 48
    pos, f = _positions(rng, 3, n, False), _freqs(rot // 2)
    axis = rng.integers(0, 3, rot // 2).astype(np.int32)
    dev = [torch.from_numpy(a).to(DEV) for a in (pos, f, axis)]
    X = torch.from_numpy(rng.standard_normal((n, H, d)).astype(np.float32))
    G = torch.from_numpy(rng.standard_normal((n, H, d)).astype(np.float32))
    x = X.double().requires_grad_()
    angle = torch.from_numpy(pos[axis].astype(np.float64).T * f)[:, None]
    a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    y = torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin(), x[..., rot:]), -1)
    (y * G.double()).sum().backward()
    got = rr.rotate(G.to(DEV), dev[0], dev[1], axis=dev[2], inverse=True)
    _check(_np(got), _np(G), x.grad.numpy(), rot, False, "f32")
    forward = _np(rr.rotate(X.to(DEV), dev[0], dev[1], axis=dev[2]))
    for i in range(0, d, 5):
        E = X.clone()
        E[:, :, i] += 1.0
        step = (E.double() - X.double())[:, :, i].numpy()  # (one, but for the rounding of the sum)
        diff = ((_np(rr.rotate(E.to(DEV), dev[0], dev[1], axis=dev[2])) - forward) * G.double().numpy()).sum(-1)
        tol = 2 * 9 * 2.0 ** -24 * (np.abs(G.double().numpy()) * (_partners(np.abs(_np(X)) + 1, rot, False))).sum(-1)
        assert np.all(np.abs(diff - step * _np(got)[:, :, i]) <= tol)


def test_more_than_2_31_elements():
    rr = rrmod()
    note("rotate 2^31 elements")
    n, H, d = 132000, 64, 256
    X = torch.empty((H, n, d), dtype=torch.bfloat16, device=DEV)
    assert X.numel() > 2 ** 31
    X.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    pos = torch.stack((torch.arange(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV) % 97))
    f = _freqs(d // 2)
    axis = (np.arange(d // 2) % 2).astype(np.int32)
    rows = [(0, 0), (0, n - 1), (31, 77777), (H - 1, 0), (H - 1, n - 1), (62, 131071)]
    before = {r: _np(X[r]) for r in rows}
    rr.rotate(X, pos, torch.from_numpy(f).to(DEV), axis=torch.from_numpy(axis).to(DEV), tokens=1, out=X)
    p = pos.cpu().numpy()
    for h, i in rows:
        x = before[h, i][None, None]
        _check(_np(X[h, i])[None, None], x, serving.rotate(x, p[:, i:i + 1], f, axis), d, False, "bf16")


# ------------------------------------------------------------ the append

@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("d,rot,inter,axes,real,page", [
    (128, 128, False, 3, False, 16), (64, 32, True, 2, True, 7), (40, 24, False, 4, False, 5), (128, 0, False, 1, False, 16),
])
def test_append_by_axes(dtype, cache, d, rot, inter, axes, real, page):
    rr = rrmod()
    note("append axes", dtype, cache, d, rot, inter, axes, real, page)
    rng = np.random.default_rng(d + rot)
    H, Hkv = 6, 2
    lens, new = [1, 50, 0, 33, 7], [1, 20, 0, 33, 3]
    n = sum(new)
    starts = np.concatenate(([0], np.cumsum(new)))
    held = [-(-x // page) for x in lens]
    n_pages = sum(held) + 2
    order, table, at = rng.permutation(n_pages), np.full((5, max(held) + 1), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    K, V, Q = (torch.from_numpy(rng.standard_normal((n, h, d)).astype(np.float32)).to(TYPE[dtype]).to(DEV)
               for h in (Hkv, Hkv, H))
    pools = [torch.zeros((n_pages, Hkv, page, d), dtype=TYPE[cache], device=DEV) for _ in range(2)]
    scales = {}
    if cache == "e4m3":
        scales = {k: torch.from_numpy((0.01 + 0.02 * rng.random(Hkv)).astype(np.float32)).to(DEV) for k in ("k_scale", "v_scale")}
    pos, f = _positions(rng, axes, n, real), _freqs(rot // 2)
    axis = rng.integers(0, axes, rot // 2).astype(np.int32)
    dev = [torch.from_numpy(a).to(DEV) for a in (pos, f, axis)]
    i32 = [torch.from_numpy(np.asarray(a, np.int32)).to(DEV) for a in (table, lens, starts)]
    out = rr.cache_append(K, V, *pools, i32[0], i32[1], seq_start=i32[2], freqs=dev[1], interleaved=inter, Q=Q,
                          positions=dev[0], axis=dev[2], **scales)
    exact = serving.rotate(_np(Q), pos, f, axis, inter)
    _check(_np(out), _np(Q), exact, rot, inter, dtype)
    exact, k, got = serving.rotate(_np(K), pos, f, axis, inter), _np(K), np.zeros((n, Hkv, d))
    for b in range(5):
        for i in range(new[b]):
            u = lens[b] - new[b] + i
            got[starts[b] + i] = _np(pools[0][table[b, u // page], :, u % page].float())
            v = _np(pools[1][table[b, u // page], :, u % page].float())
            if cache != "e4m3":
                assert np.array_equal(v, _np(V[starts[b] + i]))
    if cache == "e4m3":
        ks = _np(scales["k_scale"])[:, None]
        k, exact = k / ks, exact / ks
        tol = 9 * 2.0 ** -24 * _partners(k, rot, inter) + 1.01 * np.maximum(2.0 ** -4 * np.abs(exact), 2.0 ** -10)
        assert np.all(np.abs(got - np.clip(exact, -448, 448)) <= tol)
    else:
        _check(got, k, exact, rot, inter, cache)


def test_positions_of_the_places_are_the_append():
    """Tokens whose positions are their places: what cache_append does without."""
    rr = rrmod()
    note("append axes as places")
    rng = np.random.default_rng(9)
    B, H, Hkv, d, page = 3, 8, 2, 128, 16
    lens = torch.tensor([40, 9, 100], dtype=torch.int32, device=DEV)
    table = torch.arange(3 * 7, dtype=torch.int32, device=DEV).view(3, 7)
    n = 2 * B
    K, V, Q = (torch.from_numpy(rng.standard_normal((n, h, d)).astype(np.float32)).bfloat16().to(DEV) for h in (Hkv, Hkv, H))
    f = torch.from_numpy(_freqs(d // 2)).to(DEV)
    pos = torch.stack((lens - 2, lens - 1), 1).flatten().to(torch.int32)
    got = []
    for more in ({}, dict(positions=pos), dict(positions=pos.float()),
                 dict(positions=torch.stack((pos, pos)), axis=(torch.arange(64, device=DEV) % 2).to(torch.int32))):
        pools = [torch.zeros((21, Hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        out = rr.cache_append(K, V, *pools, table, lens, freqs=f, Q=Q, **more)
        got.append((out, *pools))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("scale", [1.0, 0.02, 3.1e-3, float.fromhex("0x1.fffffep-7"), 1e-30, 2e30, 7.0 / 3])
def test_values_of_an_8_bit_cache_are_quotients(scale):
    """What an e4m3 cache holds is x / scale, rounded to binary32 and then once
    more, as a division gives it: bits equal, for values that are not finite, past
    448, and near every border of the type too."""
    rr = rrmod()
    note("append e4m3 quotients", scale)
    rng = np.random.default_rng(11)
    s = np.float32(scale)
    borders = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    mid = ((borders[:-1] + borders[1:]) / 2).nan_to_num(0.0)
    x = torch.cat((borders.nan_to_num(0.0) * s, mid * s, torch.from_numpy(rng.standard_normal(40000).astype(np.float32) * 60 * s),
                   torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38, -3e38, 1e-38, 0.0, -0.0]) * 1.0))
    x = torch.cat((x, -x))
    n, d = -(-x.numel() // 128), 64
    rows = torch.zeros(n * 128)
    rows[:x.numel()] = x
    K = rows.view(n, 2, d).bfloat16().to(DEV)
    pools = [torch.zeros((n, 2, 1, d), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
    table = torch.arange(n, dtype=torch.int32, device=DEV).view(1, n)
    scales = torch.tensor([s, s], device=DEV)
    rr.cache_append(K, K, *pools, table, torch.tensor([n], dtype=torch.int32, device=DEV), k_scale=scales, v_scale=scales)
    y = (K.float().cpu() / torch.tensor(s))
    y = torch.where(y.isnan(), y, y.clamp(-448, 448)).to(torch.float8_e4m3fn).view(torch.uint8)
    for pool in pools:
        got = pool.view(torch.uint8).cpu()[:, :, 0]
        nan = K.isnan().cpu()
        assert torch.equal(got[~nan], y[~nan])
        assert bool(((got[nan] & 0x7f) == 0x7f).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [0, 1])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("heads,d,rot", [(17, 128, 128), (5, 256, 128), (3, 1024, 1024)])
def test_large_rotations_are_small_ones(dtype, tokens, inter, heads, d, rot):
    """What does not fit the last cache goes past it: every bit as a few tokens at a
    time give it, in place too."""
    rr = rrmod()
    note("rotate large", dtype, tokens, inter, heads, d, rot)
    g = torch.Generator(device=DEV).manual_seed(heads)
    n = (260 << 20) // (heads * d * dtype.itemsize) + 3
    shape = (n, heads, d) if tokens == 0 else (heads, n, d)
    X = torch.randn(shape, generator=g, device=DEV).to(dtype)
    positions = torch.randint(0, 9000, (2, n), generator=g, device=DEV).to(torch.int32)
    axis = torch.randint(0, 2, (rot // 2,), generator=g, device=DEV).to(torch.int32)
    freqs = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / (rot // 2))
    kw = dict(axis=axis, tokens=tokens, interleaved=inter)
    whole = rr.rotate(X, positions, freqs, **kw)
    parts = torch.empty_like(X)
    step = n // 5 + 1
    for i in range(0, n, step):
        j = min(i + step, n)
        rr.rotate(X.narrow(tokens, i, j - i), positions[:, i:j].contiguous(), freqs, out=parts.narrow(tokens, i, j - i), **kw)
    assert torch.equal(whole, parts)
    rr.rotate(X, positions, freqs, out=X, **kw)
    assert torch.equal(whole, X)


NOT_THERE = [2, 7, -1, 2 ** 31 - 1, -2 ** 31]


def _without_axes(rng, half, n):
    """Axes of frequencies, some of them not there, whose frequencies are whatever they are."""
    axis = rng.integers(0, 2, half).astype(np.int32)
    still = rng.random(half) < 0.5
    still[:5] = True
    axis[still] = rng.choice(NOT_THERE, int(still.sum()))
    f = _freqs(half)
    f[still] = rng.choice([np.nan, np.inf, -np.inf, 0.0, 1e300, 1.0], int(still.sum()))
    return axis, f, still


def _any_values(rng, shape, still, rot, inter, dtype):
    """Rows that are ordinary but for the features that stay: infinities, NaN, zeros of both signs, the largest there are."""
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPE[dtype])
    at = np.nonzero(still)[0]
    both = np.concatenate((2 * at, 2 * at + 1) if inter else (at, at + rot // 2))
    big = torch.finfo(TYPE[dtype]).max
    some = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0, 0.0, big, -big, 1.0], dtype=torch.float32).to(TYPE[dtype])
    x[..., both] = some[torch.from_numpy(rng.integers(0, len(some), (*shape[:-1], len(both))))]
    return x.to(DEV), both


def _same_bits(a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16 if a.dtype == torch.bfloat16 else torch.uint8
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,d,rot,tokens", [(1, 1, 64, 64, 0), (40, 4, 64, 64, 0), (40, 4, 64, 32, 1), (40, 4, 72, 72, 0),
                                              (40, 4, 72, 72, 1), (9001, 64, 128, 128, 0), (9001, 64, 128, 128, 1)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_an_axis_that_is_not_there_leaves_its_partners(dtype, n, H, d, rot, tokens, inter, inverse):
    """Whatever they are, and whatever its frequency is, by bits: a partner of an
    infinity or a NaN, zeros below 0.  (The largest go past the caches.)"""
    rr = rrmod()
    note("rotate no axis", dtype, n, H, d, rot, tokens, inter, inverse)
    rng = np.random.default_rng(n + rot)
    axis, f, still = _without_axes(rng, rot // 2, n)
    X, both = _any_values(rng, (n, H, d) if tokens == 0 else (H, n, d), still, rot, inter, dtype)
    dev = [torch.from_numpy(a).to(DEV) for a in (_positions(rng, 2, n, False), f, axis)]
    got = rr.rotate(X, dev[0], dev[1], axis=dev[2], tokens=tokens, interleaved=inter, inverse=inverse)
    assert _same_bits(got[..., both], X[..., both])
    assert _same_bits(got[..., rot:], X[..., rot:])
    others = np.setdiff1d(np.arange(rot), both)
    assert bool(got[..., others].isfinite().all())
    assert len(others) == 0 or n == 1 or not _same_bits(got[..., others], X[..., others])
    Y = X.clone()
    rr.rotate(Y, dev[0], dev[1], axis=dev[2], tokens=tokens, interleaved=inter, inverse=inverse, out=Y)
    assert _same_bits(Y, got)


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("H,Hkv,d,rot,n", [(6, 2, 64, 64, 50), (6, 2, 72, 72, 50), (3, 1, 1024, 1024, 33), (60, 4, 128, 128, 9001)])
@pytest.mark.parametrize("inter", [False, True])
def test_append_by_an_axis_that_is_not_there(dtype, cache, H, Hkv, d, rot, n, inter):
    rr = rrmod()
    note("append no axis", dtype, cache, H, Hkv, d, rot, n, inter)
    rng = np.random.default_rng(n + rot)
    axis, f, still = _without_axes(rng, rot // 2, n)
    X, both = _any_values(rng, (n, H + 2 * Hkv, d), still, rot, inter, dtype)
    Q, K, V = X[:, :H], X[:, H:H + Hkv], X[:, H + Hkv:]
    pools = [torch.zeros((n, Hkv, 1, d), dtype=TYPE[cache], device=DEV) for _ in range(2)]
    scales = {}
    if cache == "e4m3":
        scales = {k: torch.full((Hkv,), 0.0625, device=DEV) for k in ("k_scale", "v_scale")}
    dev = [torch.from_numpy(a).to(DEV) for a in (_positions(rng, 2, n, False), f, axis)]
    table = torch.randperm(n, generator=torch.Generator().manual_seed(n)).to(torch.int32).to(DEV)
    out = rr.cache_append(K, V, *pools, table.view(1, n), torch.tensor([n], dtype=torch.int32, device=DEV), freqs=dev[1],
                          interleaved=inter, Q=Q, positions=dev[0], axis=dev[2], **scales)
    assert _same_bits(out[..., both], Q[..., both])
    got, values = (p[table.long(), :, 0] if cache != "e4m3" else p.view(torch.uint8)[table.long(), :, 0] for p in pools)
    want, values_want = K[..., both], V
    if cache == "e4m3":  # (16 x is exact, NaN is any of that type's two)
        want, values_want = ((16 * x.float()).clamp(-448.0, 448.0).to(TYPE[cache]).view(torch.uint8) for x in (want, values_want))
        k_nan, v_nan = K[..., both].isnan(), V.isnan()
        assert bool(((got[..., both][k_nan] & 0x7f) == 0x7f).all()) and bool(((values[v_nan] & 0x7f) == 0x7f).all())
        assert torch.equal(got[..., both][~k_nan], want[~k_nan]) and torch.equal(values[~v_nan], values_want[~v_nan])
    else:
        assert _same_bits(got[..., both], want) and _same_bits(values, values_want)
    others = np.setdiff1d(np.arange(rot), both)
    assert bool(out[..., others].isfinite().all()) and bool((got.float() if cache != "e4m3" else got.view(TYPE[cache]).float())
                                                            [..., others].isfinite().all())


def _either(x):
    """What binary32 may hold of a sum of two numbers that binary64 has rounded to x."""
    return [torch.from_numpy((x * (1 + e)).astype(np.float32)) for e in (-2.0 ** -52, 2.0 ** -52)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot,shift", [(64, 64, 0), (128, 64, 0), (72, 40, 0), (64, 64, 1)])
@pytest.mark.parametrize("heads", [3, 40])
def test_every_call_rounds_the_same_product_first(dtype, inter, d, rot, shift, heads):
    """x c - (q s rounded), and the partner's own product last of two halves, first
    of two neighbours: the same bits from the rotation of either layout, from the
    append by place and by axes, of few tokens and (40 heads) of what goes past the
    caches.  Cosines and sines are those that the rotation gives 1 and 0."""
    rr = rrmod()
    note("rotate product", dtype, inter, d, rot, shift, heads)
    rng = np.random.default_rng(d + rot)
    few = 70
    n = few if heads == 3 else (260 << 20) // (heads * d * TYPE[dtype].itemsize) + 1
    half = rot // 2
    a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if inter else (np.arange(half), np.arange(half, rot))
    wide = torch.zeros((n, heads, d + 8 * shift), dtype=TYPE[dtype], device=DEV)
    wide.normal_(generator=torch.Generator(device=DEV).manual_seed(d))
    X = wide[:, :, shift:shift + d]
    f = torch.from_numpy(_freqs(half)).to(DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    one = torch.zeros((few, 1, d), device=DEV)
    one[..., a] = 1.0
    turn = _np(rr.rotate(one, pos[:few].contiguous(), f, interleaved=inter))
    c, s, x = turn[..., a], turn[..., b], _np(X[:few])
    p, q = x[..., a], x[..., b]

    def once(v):
        return v.astype(np.float32).astype(np.float64)

    first = _either(p * c - once(q * s))
    second = _either(p * s + once(q * c) if inter else q * c + once(p * s))
    got = rr.rotate(X, pos, f, interleaved=inter)
    for at, want in ((a, first), (b, second)):
        y = got[:few].cpu()[..., at]
        assert bool(((y == want[0].to(TYPE[dtype])) | (y == want[1].to(TYPE[dtype]))).all())
    turned = rr.rotate(wide.transpose(0, 1).contiguous()[:, :, shift:shift + d], pos, f, tokens=1, interleaved=inter)
    assert torch.equal(turned.transpose(0, 1), got)
    del turned
    assert torch.equal(rr.rotate(X[:few], pos[:few].contiguous(), f, interleaved=inter), got[:few])
    table, lens = pos.view(1, n), torch.tensor([n], dtype=torch.int32, device=DEV)
    flat = X.contiguous() if not shift else None
    if shift:  # (rows of a token lie together: as many elements off as a vector has not)
        flat = torch.empty(n * heads * d + 1, dtype=TYPE[dtype], device=DEV)[1:].view(n, heads, d)
        flat.copy_(X)
    for more in ({}, dict(positions=pos)):
        pools = [torch.zeros((n, 1, 1, d), dtype=TYPE[dtype], device=DEV) for _ in range(2)]
        out = rr.cache_append(flat[:, :1], flat[:, :1], *pools, table, lens, freqs=f, interleaved=inter, Q=flat, **more)
        assert torch.equal(out, got)
        assert torch.equal(pools[0][:, :, 0], got[:, :1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [0, 1])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("heads,d,rot", [(17, 128, 64), (9, 256, 128), (5, 512, 128), (40, 96, 32), (3, 1024, 0)])
def test_large_rotations_of_a_part_of_each_row(dtype, tokens, inter, heads, d, rot):
    """What is not rotated is copied past the last cache too, and left where it is
    in place."""
    rr = rrmod()
    note("rotate large, a part", dtype, tokens, inter, heads, d, rot)
    g = torch.Generator(device=DEV).manual_seed(heads + d)
    n = (260 << 20) // (heads * d * dtype.itemsize) + 3
    shape = (n, heads, d) if tokens == 0 else (heads, n, d)
    X = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    positions = torch.randint(0, 9000, (2, n), generator=g, device=DEV).to(torch.int32)
    axis = torch.randint(0, 2, (rot // 2,), generator=g, device=DEV).to(torch.int32)
    freqs = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / max(1, rot // 2))
    kw = dict(axis=axis, tokens=tokens, interleaved=inter)
    whole = rr.rotate(X, positions, freqs, **kw)
    parts = torch.empty_like(X)
    step = n // 5 + 1
    for i in range(0, n, step):
        j = min(i + step, n)
        rr.rotate(X.narrow(tokens, i, j - i), positions[:, i:j].contiguous(), freqs, out=parts.narrow(tokens, i, j - i), **kw)
    assert torch.equal(whole, parts)
    assert torch.equal(whole[..., rot:], X[..., rot:])
    assert rot == 0 or not torch.equal(whole[..., :rot], X[..., :rot])
    back = rr.rotate(whole, positions, freqs, inverse=True, **kw)
    assert torch.equal(back[..., rot:], X[..., rot:])
    rr.rotate(X, positions, freqs, out=X, **kw)
    assert torch.equal(whole, X)


def _at_borders(rng, x):
    """Scales, one for each number of x, that bring it to a border between two e4m3
    numbers or as near as binary32 comes: three for each of some borders."""
    values = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    t = rng.choice((values[:-1].astype(np.float64) + values[1:]) / 2, x.shape)
    s = (np.abs(x) / t).astype(np.float32)
    way = rng.integers(-1, 2, x.shape)
    return np.where(way < 0, np.nextafter(s, np.float32(0)), np.where(way > 0, np.nextafter(s, np.float32(np.inf)), s))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("axes", [False, True])
@pytest.mark.parametrize("d,size", [(64, 1.0), (72, 1e-6), (128, 3e4)])
def test_quotients_at_the_borders_of_8_bits(inter, axes, d, size):
    """Keys that are rotated (all 24 bits of a numerator) and values, under scales
    that bring one of each row next to a border: the bits of a division.  (What a
    key is before its quotient is what the rotation gives in binary32.)"""
    rr = rrmod()
    note("append e4m3 borders", inter, axes, d, size)
    rng = np.random.default_rng(d)
    heads, n = 3000, 5
    K, V = (torch.from_numpy(rng.standard_normal((n, heads, d)).astype(np.float32) * size).bfloat16().to(DEV) for _ in range(2))
    f = torch.from_numpy(_freqs(d // 2)).to(DEV)
    pos = torch.arange(100, 100 + n, dtype=torch.int32, device=DEV)
    keys = rr.rotate(K.float(), pos, f, interleaved=inter).cpu()
    scales = [torch.from_numpy(_at_borders(rng, x[rng.integers(0, n, heads), np.arange(heads), rng.integers(0, d, heads)].numpy()))
              for x in (keys, V.float().cpu())]
    assert bool((torch.cat(scales) > 2.0 ** -60).all())
    pools = [torch.zeros((105, heads, 1, d), dtype=TYPE["e4m3"], device=DEV) for _ in range(2)]
    table = torch.arange(105, dtype=torch.int32, device=DEV).view(1, 105)
    rr.cache_append(K, V, *pools, table, torch.tensor([100 + n], dtype=torch.int32, device=DEV), freqs=f, interleaved=inter,
                    positions=pos if axes else None, k_scale=scales[0].to(DEV), v_scale=scales[1].to(DEV))
    for pool, x, s in zip(pools, (keys, V.float().cpu()), scales):
        want = (x / s[:, None]).clamp(-448.0, 448.0).to(TYPE["e4m3"]).view(torch.uint8)
        assert torch.equal(pool.view(torch.uint8)[100:, :, 0].cpu(), want)
