"""GPU parity of the verification of drafted tokens against the binary64 oracle.

Everything is compared as whole numbers: products of binary32 numbers are exact
in binary64, and sums of V terms in another order are off by at most V 2^-53 of
the whole, so that a drawn token may differ only where a border lies that near
to a sum: the oracle says how near the nearest one came (`near`), and the test
asserts that it is farther than 2 V 2^-53."""
import sys

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


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


def _probabilities(g, shape, dtype, sharp=2.0, kept=0.0):
    p = (torch.randn(shape, generator=g, device=DEV) * sharp).softmax(-1)
    p = torch.where(p >= kept * p.amax(-1, keepdim=True), p, torch.zeros_like(p))
    return (p / p.sum(-1, keepdim=True)).to(TYPE[dtype])


def _inputs(seed, B, n, V, dtype, kept=0.0, close=0.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    P = _probabilities(g, (B, n + 1, V), dtype, kept=kept)
    Q = P[:, :n].float() * (torch.randn((B, n, V), generator=g, device=DEV) * close).exp()
    Q = (Q / Q.sum(-1, keepdim=True)).to(TYPE[dtype])
    wait = torch.empty((B, n, V), device=DEV).exponential_(generator=g)
    drafts = (Q.float() / wait).argmax(-1).to(torch.int32) if n else torch.zeros((B, 0), dtype=torch.int32, device=DEV)
    return P, Q, drafts, torch.rand((B, n + 1), generator=g, device=DEV)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _check(rr, P, Q, drafts, u, count=None, **kw):
    accepted, tokens = rr.verify_drafts(P, drafts, u, draft_probs=Q, n_drafts=count, **kw)
    a, t, near = serving.verify(_np(P), _np(Q), drafts.cpu().numpy(), _np(u), None if count is None else count.cpu().numpy())
    assert near > 2 * P.shape[-1] * 2.0 ** -53, "inputs at a border"
    assert accepted.tolist() == a.tolist()
    assert tokens.tolist() == t.tolist()
    return accepted, tokens


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,V", [(1, 0, 1), (1, 1, 2), (5, 3, 3), (7, 4, 255), (3, 2, 256), (3, 5, 257), (2, 70, 40),
                                   (64, 4, 1000), (1, 4, 32000), (3, 2, 50001), (2, 1, 131072), (40, 3, 20011),
                                   (2, 2, 300001), (30, 1, 131071)])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("ragged", [False, True])
def test_verify(dtype, B, n, V, given, ragged):
    rr = rrmod()
    note("verify", dtype, B, n, V, given, ragged)
    P, Q, drafts, u = _inputs(B + V, B, n, V, dtype)
    count = torch.randint(-1, n + 3, (B,), device=DEV).to(torch.int32) if ragged else None
    a, t = _check(rr, P, Q if given else None, drafts, u, count)
    if not given and n and V > 2 and not ragged:  # looked-up drafts are taken as often as the target says
        assert int(a.max()) <= n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_workspace_for_every_shape(dtype):
    rr = rrmod()
    note("verify one workspace", dtype)
    shapes = [(4, 3, 131072), (300, 2, 33), (1, 0, 7), (2, 5, 65537), (500, 1, 100), (4, 3, 131072)]
    ws = max((rr.verify_workspace(torch.empty((B, n + 1, V), dtype=TYPE[dtype], device=DEV)) for B, n, V in shapes),
             key=lambda w: w.numel())
    for i, (B, n, V) in enumerate(shapes):
        P, Q, drafts, u = _inputs(50 + i, B, n, V, dtype)
        _check(rr, P, Q, drafts, u, workspace=ws)
    assert int(ws[:65536].sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (1, 1), (7, 3), (32, 0)])
def test_rows_that_lie_apart(dtype, pad, shift):
    """Views of padded rows, from any element on; what lies between is NaN."""
    rr = rrmod()
    note("verify views", dtype, pad, shift)
    B, n, V = 6, 3, 4003
    P, Q, drafts, u = _inputs(7, B, n, V, dtype)
    wide = [torch.full((B, x.shape[1] + 2, V + pad), float("nan"), dtype=x.dtype, device=DEV) for x in (P, Q)]
    views = [w[:, 1:1 + x.shape[1], shift:shift + V] for w, x in zip(wide, (P, Q))]
    for v, x in zip(views, (P, Q)):
        v.copy_(x)
    got = _check(rr, *views, drafts, u)
    want = rr.verify_drafts(P, drafts, u, draft_probs=Q)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # one target row for all sequences
    same = P[:1].expand(B, n + 1, V)
    _check(rr, same, Q, drafts, u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_truncated_distributions(dtype):
    rr = rrmod()
    note("verify truncated", dtype)
    P, Q, drafts, u = _inputs(11, 50, 4, 9001, dtype, kept=0.05, close=1.5)
    assert float((P == 0).float().mean()) > 0.9
    _check(rr, P, Q, drafts, u)
    _check(rr, P, None, drafts, u)


def test_borders():
    """Probabilities that are sums of powers of two: every sum is exact, and a
    uniform number on a border belongs to the token behind it; uniform numbers
    of 0, below 1, 1, past it, below 0 and NaN."""
    rr = rrmod()
    note("verify borders")
    p = [0.0, 0.25, 0.0, 0.5, 0.125, 0.125, 0.0]
    us = [0.0, 0.125, 0.25, 0.5, 0.75, 0.875, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan")]
    want = [1, 1, 3, 3, 4, 5, 5, 5, 5, 1, 5]
    B = len(us)
    for dtype in ("f32", "bf16"):
        P = torch.tensor(p, device=DEV).to(TYPE[dtype]).expand(B, 1, 7)
        u = torch.tensor(us, device=DEV).view(B, 1)
        a, t = rr.verify_drafts(P, torch.zeros((B, 0), dtype=torch.int32, device=DEV), u)
        assert a.tolist() == [0] * B and t.flatten().tolist() == want
        # a draft is taken below p / q, not at it
        P = torch.tensor([p, p], device=DEV).to(TYPE[dtype]).expand(4, 2, 7)
        Q = torch.tensor([0.0, 0.0, 0.0, 1.0, 0.0, 0.0, 0.0], device=DEV).to(TYPE[dtype]).expand(4, 1, 7)
        u = torch.tensor([[0.5, 0.3], [0.5 - 2.0 ** -24, 0.3], [0.0, 0.9], [float("nan"), 0.3]], device=DEV)
        drafts = torch.full((4, 1), 3, dtype=torch.int32, device=DEV)
        a, t = rr.verify_drafts(P, drafts, u, draft_probs=Q)
        # (not taken: 0.25, 0.125 and 0.125 are left, 0.3 of 0.5 lies in the first)
        assert a.tolist() == [0, 1, 1, 0] and t.tolist() == [[1, -1], [3, 3], [3, 5], [1, -1]]
        assert rr.verify_drafts(P, drafts, u)[1].tolist() == t.tolist()


@pytest.mark.parametrize("V", [3000, 300001])
def test_nothing_left_and_no_probabilities(V):
    rr = rrmod()
    note("verify nothing left", V)
    inf, nan = float("inf"), float("nan")
    last = V - 1

    def row(**at):
        x = torch.zeros(V)
        for k, v in at.items():
            x[int(k[1:])] = v
        return x

    rows = [  # target, drafts' probabilities, draft, uniform numbers, token, taken
        (row(v5=0.5, v2000=0.5), row(v5=0.5, v2000=0.5, v7=0.1), 7, [0.0, 0.2], 5, 0),   # q covers p: from the target
        (row(v5=0.5, v2000=0.5), row(v5=0.6, v2000=0.6, v7=0.1), 7, [0.9, 0.6], 2000, 0),
        (row(), row(v5=1.0), 5, [0.0, 0.5], -1, 0),                                      # the target has none
        (row(v3=nan, v4=inf, v9=-1.0), row(v5=1.0), 5, [0.0, 0.5], -1, 0),               # ... that counts
        (row(v3=nan, v4=inf, v9=-1.0, **{f"v{last}": 0.1}), row(v5=1.0), 5, [0.0, 0.0], last, 0),
        (row(v8=1.0), row(v8=nan), 8, [0.0, 0.5], 8, 0),                                 # p - NaN: nothing, so from p
        (row(v8=1.0, v9=0.5), row(v8=1.0), -1, [0.0, 0.5], 9, 0),                        # no such draft
        (row(v8=1.0, v9=0.5), row(v8=1.0), V, [0.0, 0.5], 9, 0),
        (row(v8=1.0, v9=0.5), row(v9=0.5), 2 ** 31 - 1, [0.0, 0.5], 8, 0),
        (row(v4=inf), row(v4=1.0), 4, [0.5, 0.5], 4, 1),
    ]
    P = torch.stack([torch.stack((r[0], row(v4=0.25))) for r in rows]).to(DEV)
    Q = torch.stack([r[1][None] for r in rows]).to(DEV)
    drafts = torch.tensor([[r[2]] for r in rows], dtype=torch.int32, device=DEV)
    u = torch.tensor([r[3] for r in rows], device=DEV)
    for dtype in ("f32", "bf16"):
        a, t = rr.verify_drafts(P.to(TYPE[dtype]), drafts, u, draft_probs=Q.to(TYPE[dtype]))
        assert a.tolist() == [r[5] for r in rows]
        assert t.tolist() == [[4, 4] if r[5] else [r[4], -1] for r in rows]
    # a looked-up draft that is all the target has
    one = row(v6=0.5).expand(1, 2, V).contiguous().to(DEV)
    a, t = rr.verify_drafts(one, torch.tensor([[6]], dtype=torch.int32, device=DEV), torch.tensor([[0.7, 0.1]], device=DEV))
    assert a.tolist() == [0] and t.tolist() == [[6, -1]]


def test_lengths_and_outputs_given():
    rr = rrmod()
    note("verify lengths")
    B, n, V = 33, 5, 700
    P, Q, drafts, u = _inputs(21, B, n, V, "f32")
    count = (torch.arange(B, device=DEV) % (n + 1)).to(torch.int32)
    lengths = (100 + torch.arange(B, device=DEV)).to(torch.int32)
    accepted, tokens = torch.full((B,), 9, dtype=torch.int32, device=DEV), torch.full((B, n + 1), 9, dtype=torch.int32, device=DEV)
    got = _check(rr, P, Q, drafts, u, count, lengths=lengths, accepted=accepted, tokens=tokens)
    assert got[0] is accepted and got[1] is tokens
    assert lengths.tolist() == [100 + b - (int(c) - int(a)) for b, (c, a) in enumerate(zip(count, accepted))]


def test_more_sequences_than_counters():
    rr = rrmod()
    note("verify many sequences")
    B, n, V = 40000, 2, 9
    P, Q, drafts, u = _inputs(22, B, n, V, "f32")
    count = torch.randint(0, n + 1, (B,), device=DEV).to(torch.int32)
    lengths = torch.full((B,), 50, dtype=torch.int32, device=DEV)
    a, _ = _check(rr, P, Q, drafts, u, count, lengths=lengths)
    assert torch.equal(lengths, 50 - count + a)


def test_drawn_as_from_the_target():
    """First tokens of many drafted pairs are distributed as the target's: each
    frequency within six standard deviations of its probability."""
    rr = rrmod()
    note("verify distribution")
    B, V = 1 << 16, 8
    g = torch.Generator(device=DEV).manual_seed(5)
    p = _probabilities(g, (1, 2, V), "f32", sharp=1.0)
    q = _probabilities(g, (1, 1, V), "f32", sharp=1.0)
    wait = torch.empty((B, 1, V), device=DEV).exponential_(generator=g)
    drafts = (q / wait).argmax(-1).to(torch.int32)
    u = torch.rand((B, 2), generator=g, device=DEV)
    _, t = rr.verify_drafts(p.expand(B, 2, V), drafts, u, draft_probs=q.expand(B, 1, V))
    f = torch.bincount(t[:, 0].long(), minlength=V).double() / B
    want = p[0, 0].double()
    assert bool(((f - want).abs() <= 6 * (want * (1 - want) / B).sqrt()).all())


def test_rows_past_2_31_elements():
    rr = rrmod()
    note("verify 2^31 elements")
    B, n, V = 17, 1, 1 << 20
    wide = torch.zeros((B, 130, V), dtype=torch.bfloat16, device=DEV)  # rows of P and Q 65 apart: 2.3e9 elements
    assert wide.numel() > 2 ** 31
    P, Q, drafts, u = _inputs(31, B, n, V, "bf16")
    wide[:, 0::65][:, :2].copy_(P)
    wide[:, 64:65].copy_(Q)
    got = rr.verify_drafts(wide[:, 0::65], drafts, u, draft_probs=wide[:, 64:65])
    want = rr.verify_drafts(P, drafts, u, draft_probs=Q)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    _check(rr, P[-2:], Q[-2:], drafts[-2:], u[-2:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("given", [True, False])
def test_large_batches_are_small_ones(dtype, given):
    """Probabilities that do not fit the last cache are read past it."""
    rr = rrmod()
    note("verify large", dtype, given)
    n, V = 3, 50003
    B = (270 << 20) // ((2 * n + 1 if given else n + 1) * V * (4 if dtype == "f32" else 2)) + 1
    P, Q, drafts, u = _inputs(31, B, n, V, dtype)
    Q = Q if given else None
    accepted, tokens = rr.verify_drafts(P, drafts, u, draft_probs=Q)
    step = B // 3 + 1
    for i in range(0, B, step):
        s = slice(i, min(i + step, B))
        a, t = rr.verify_drafts(P[s], drafts[s], u[s], draft_probs=None if Q is None else Q[s])
        assert torch.equal(a, accepted[s])
        assert torch.equal(t, tokens[s])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,V", [(33, 1, 131071), (90, 1, 100003), (170, 1, 100500), (340, 1, 100500), (60, 1, 300001),
                                   (700, 2, 20011), (1100, 1, 9000)])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("ragged", [False, True])
def test_waves_that_sum_several_parts(dtype, B, n, V, given, ragged):
    """Two to sixteen parts a wave, the last waves with fewer or none, of one, two
    and four steps; and the same sequences in calls of one part a wave."""
    rr = rrmod()
    note("verify several parts", dtype, B, n, V, given, ragged)
    P, Q, drafts, u = _inputs(B + V, B, n, V, dtype)
    count = torch.randint(-1, n + 3, (B,), device=DEV).to(torch.int32) if ragged else None
    Q = Q if given else None
    accepted, tokens = _check(rr, P, Q, drafts, u, count)
    step = max(1, 8000 // max(1, -(-V // 256)))
    for i in range(0, B, step):
        s = slice(i, min(i + step, B))
        a, t = rr.verify_drafts(P[s], drafts[s], u[s], draft_probs=None if Q is None else Q[s],
                                n_drafts=None if count is None else count[s])
        assert torch.equal(a, accepted[s]) and torch.equal(t, tokens[s])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_past_the_last_cache_as_one_part_a_wave(dtype):
    rr = rrmod()
    note("verify past the last cache", dtype)
    n, V = 3, 50003
    B = (270 << 20) // ((2 * n + 1) * V * (4 if dtype == "f32" else 2)) + 1
    P, Q, drafts, u = _inputs(32, B, n, V, dtype)
    accepted, tokens = rr.verify_drafts(P, drafts, u, draft_probs=Q)
    for i in range(0, B, 40):  # (of 196 parts, or 98)
        s = slice(i, min(i + 40, B))
        a, t = rr.verify_drafts(P[s], drafts[s], u[s], draft_probs=Q[s])
        assert torch.equal(a, accepted[s]) and torch.equal(t, tokens[s])
    _check(rr, P[-9:], Q[-9:], drafts[-9:], u[-9:])


def test_looked_up_drafts_are_taken_as_often_as_the_target_says():
    """Each within six standard deviations of its probability."""
    rr = rrmod()
    note("verify looked up")
    B, V = 1 << 17, 8
    g = torch.Generator(device=DEV).manual_seed(6)
    p = _probabilities(g, (1, 2, V), "f32", sharp=1.0)
    drafts = (torch.arange(B, device=DEV) % V).to(torch.int32)
    u = torch.rand((B, 2), generator=g, device=DEV)
    a, t = rr.verify_drafts(p.expand(B, 2, V), drafts[:, None].contiguous(), u)
    for x in range(V):
        want, k = float(p[0, 0, x]), B // V
        assert abs(float(a[drafts == x].double().mean()) - want) <= 6 * (want * (1 - want) / k) ** 0.5
        assert not bool((t[(drafts == x) & (a == 0), 0] == x).any())
