"""The calls around the paged cache together, as a program that answers makes
them: fork, resize, append by axes, attention, verification, resize again; step by
step against the oracles, captured into graphs and replayed, on streams of their
own and side by side."""
import sys

import numpy as np
import pytest
import torch

from oracle import paged, serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
LAYERS, H, HKV, D, PAGE, VOCAB, DRAFTS = 2, 4, 2, 64, 8, 311, 3


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


class Server:
    """A batch's cache and a step's buffers, as a program keeps them."""

    def __init__(self, B=6, width=12, n_pages=120):
        rr = rrmod()
        self.B = B
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table = torch.full((B, width), -1, **i32)
        self.lengths, self.refs = torch.zeros(B, **i32), torch.zeros(n_pages, **i32)
        self.K = [torch.zeros((n_pages, HKV, PAGE, D), dtype=torch.bfloat16, device=DEV) for _ in range(LAYERS)]
        self.V = [torch.zeros_like(k) for k in self.K]
        self.pools = rr.Pools(self.K, self.V)
        self.pages_ws = rr.pages_workspace(self.pools)
        n = DRAFTS + 1
        self.new = torch.full((B,), n, **i32)
        self.missing, self.accepted = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.tokens, self.drafts = torch.zeros((B, n), **i32), torch.zeros((B, DRAFTS), **i32)
        self.qkv = torch.zeros((LAYERS, B * n, H + 2 * HKV, D), dtype=torch.bfloat16, device=DEV)
        self.Q = torch.zeros((LAYERS, B * n, H, D), dtype=torch.bfloat16, device=DEV)
        self.O = torch.zeros((LAYERS, B, n, H, D), dtype=torch.bfloat16, device=DEV)
        self.positions = torch.zeros((3, B * n), **i32)
        self.axis = (torch.arange(D // 2, device=DEV) * 3 // (D // 2)).to(torch.int32)
        self.freqs = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) / (D // 2))
        self.P = torch.zeros((B, n, VOCAB), device=DEV)
        self.Qd = torch.zeros((B, DRAFTS, VOCAB), device=DEV)
        self.u = torch.zeros((B, n), device=DEV)
        self.attn_ws = rr.paged_workspace(self.Q[0].view(B, n, H, D), self.K[0], self.table)
        self.verify_ws = rr.verify_workspace(self.P)

    def feed(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.qkv.normal_(generator=g)
        self.positions.random_(0, 3000, generator=g)
        self.P.copy_((torch.randn(self.P.shape, generator=g, device=DEV) * 2).softmax(-1))
        self.Qd.copy_((self.P[:, :-1] * torch.randn(self.Qd.shape, generator=g, device=DEV).exp()))
        self.Qd.div_(self.Qd.sum(-1, keepdim=True))
        wait = torch.empty(self.Qd.shape, device=DEV).exponential_(generator=g)
        self.drafts.copy_((self.Qd / wait).argmax(-1))
        self.u.uniform_(generator=g)

    def step(self):
        """A token and three drafts of every sequence (of `new` of them)."""
        rr = rrmod()
        n = DRAFTS + 1
        self.lengths.add_(self.new)
        rr.cache_resize(self.pools, self.table, self.lengths, self.refs, self.new, missing=self.missing, workspace=self.pages_ws)
        for l in range(LAYERS):
            q, k, v = self.qkv[l].split((H, HKV, HKV), 1)
            rr.cache_append(k, v, self.K[l], self.V[l], self.table, self.lengths, freqs=self.freqs, Q=q, Q_out=self.Q[l],
                            positions=self.positions, axis=self.axis)
            rr.paged_attention(self.Q[l].view(self.B, n, H, D), self.K[l], self.V[l], self.table, self.lengths, out=self.O[l],
                               workspace=self.attn_ws)
        rr.verify_drafts(self.P, self.drafts, self.u, draft_probs=self.Qd, lengths=self.lengths, accepted=self.accepted,
                         tokens=self.tokens, workspace=self.verify_ws)

    def state(self):
        return [self.table, self.lengths, self.refs, self.missing, self.accepted, self.tokens, self.Q, self.O, *self.K, *self.V]

    def copy_from(self, other):
        for a, b in zip(self.state(), other.state()):
            a.copy_(b)


def _np(t):
    return t.float().cpu().numpy()


def test_steps_against_the_oracles():
    """Eight steps with forks between them.  Tables, counts, drafts and tokens are
    equal; rotated rows and attention within what tests of those calls allow, here
    on the cache as the step left it."""
    rr = rrmod()
    note("serving steps")
    s = Server()
    table, lengths, refs = s.table.tolist(), s.lengths.tolist(), s.refs.tolist()
    rng = np.random.default_rng(1)
    for step in range(8):
        s.feed(step)
        if step in (2, 3, 6):
            parent = [0, 0, 0, 3, 3, 5] if step == 2 else [int(p) for p in rng.integers(-1, 6, 6)]
            rr.cache_fork(s.table, s.lengths, s.refs, torch.tensor(parent, dtype=torch.int32, device=DEV))
            table, lengths, refs = serving.fork(table, lengths, refs, parent)
        held = [k.clone() for k in (*s.K, *s.V)]
        before = [list(row) for row in table]
        s.step()
        lengths = [n + DRAFTS + 1 for n in lengths]
        old = list(lengths)
        table, refs, missing, copies = serving.resize(table, lengths, refs, [DRAFTS + 1] * 6, PAGE)
        assert s.table.tolist() == table and s.refs.tolist() == refs and s.missing.tolist() == missing == [0] * 6
        # what the step appended: the queries and keys by their axes, into pages that no other sequence writes
        pos = s.positions.cpu().numpy()
        written = {}
        for l in range(LAYERS):
            q, k, v = (_np(x) for x in s.qkv[l].split((H, HKV, HKV), 1))
            exact = serving.rotate(k, pos, s.freqs.cpu().numpy(), s.axis.cpu().numpy())
            tol = 8 * 2.0 ** -24 * (np.abs(k) + np.abs(np.roll(k, D // 2, -1))) + 1.01 * 2.0 ** -8 * np.abs(exact)
            for b in range(6):
                for t in range(DRAFTS + 1):
                    u = old[b] - DRAFTS - 1 + t
                    at = (table[b][u // PAGE], u % PAGE)
                    assert written.setdefault((l, *at), (b, t)) == (b, t)
                    i = b * (DRAFTS + 1) + t
                    assert np.all(np.abs(_np(s.K[l][at[0], :, at[1]]) - exact[i]) <= tol[i])
                    assert np.array_equal(_np(s.V[l][at[0], :, at[1]]), v[i])
                # earlier tokens are those that the sequence had
                for u in range(old[b] - DRAFTS - 1):
                    for now, was in ((s.K[l], held[l]), (s.V[l], held[LAYERS + l])):
                        assert torch.equal(now[table[b][u // PAGE], :, u % PAGE], was[before[b][u // PAGE], :, u % PAGE])
            O, _, W, S = paged.attention(_np(s.Q[l].view(6, DRAFTS + 1, H, D)), _np(s.K[l]), _np(s.V[l]), np.array(table), old)
            err = 2 * (D + 8) * 2.0 ** -24 * S + (max(old) + 8) * 2.0 ** -24 + 2.0 ** -16
            assert np.all(np.abs(_np(s.O[l]) - O) <= 1.01 * (err[..., None] * W + 2.0 ** -8 * np.abs(O)) + 1e-30)
        a, t, near = serving.verify(s.P.double().cpu().numpy(), s.Qd.double().cpu().numpy(), s.drafts.cpu().numpy(),
                                    s.u.double().cpu().numpy())
        assert near > 2 * VOCAB * 2.0 ** -53
        assert s.accepted.tolist() == a.tolist() and s.tokens.tolist() == t.tolist()
        lengths = [n - DRAFTS + int(x) for n, x in zip(lengths, a)]
        assert s.lengths.tolist() == lengths
    # compacted: every sequence still has its tokens
    held = [k.clone() for k in (*s.K, *s.V)]
    rr.cache_compact(s.pools, s.table, s.refs, workspace=s.pages_ws)
    now, refs, _, used = serving.compact(table, refs)
    assert s.table.tolist() == now and s.refs.tolist() == refs and max(max(row) for row in now) < used
    for b in range(6):
        for u in range(lengths[b]):
            for x, y in zip((*s.K, *s.V), held):
                assert torch.equal(x[now[b][u // PAGE], :, u % PAGE], y[table[b][u // PAGE], :, u % PAGE])


def test_a_captured_step():
    """A step in a graph, replayed with other inputs and with eager steps, forks and
    compactions of another server between the replays, is the eager step, bit by bit."""
    rr = rrmod()
    note("serving captured")
    eager, graphed = Server(), Server()
    eager.feed(100)
    eager.step()
    graphed.copy_from(eager)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = Server()
        other.feed(5)
        other.step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    saved = [x.clone() for x in graphed.state()]
    with torch.cuda.graph(graph):
        graphed.step()
    for x, y in zip(graphed.state(), saved):
        assert torch.equal(x, y)  # (captured, not run)
    for step in range(5):
        eager.feed(step)
        graphed.feed(step)
        if step == 2:
            parent = torch.tensor([1, 1, 2, -1, 4, 4], dtype=torch.int32, device=DEV)
            for s in (eager, graphed):
                rr.cache_fork(s.table, s.lengths, s.refs, parent)
        eager.step()
        graph.replay()
        other.step()
        if step == 3:
            for s in (eager, graphed):
                rr.cache_compact(s.pools, s.table, s.refs, workspace=s.pages_ws)
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(eager.state(), graphed.state())):
            assert torch.equal(x, y), f"replay {step}: state {i} differs"


def test_captured_page_calls():
    """Forks and compactions in a graph of their own, replayed."""
    rr = rrmod()
    note("serving captured pages")
    a, b = Server(), Server()
    for s in (a, b):
        for step in range(3):
            s.feed(step)
            s.step()
    parent = torch.tensor([0, 0, 2, 2, -1, 5], dtype=torch.int32, device=DEV)
    ids, used = torch.zeros(120, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def change(s, ids, used):
        rr.cache_fork(s.table, s.lengths, s.refs, parent)
        rr.cache_resize(s.pools, s.table, s.lengths, s.refs, 0, missing=s.missing, workspace=s.pages_ws)
        rr.cache_compact(s.pools, s.table, s.refs, new_ids=ids, n_used=used, workspace=s.pages_ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        change(b, ids, used)
    ids2, used2 = ids.clone(), used.clone()
    for turn in ([0, 0, 2, 2, -1, 5], [5, 4, 3, 2, 1, 0], [0, 1, 2, 3, 4, 5], [-1, 0, 0, 0, 0, 0]):
        parent.copy_(torch.tensor(turn, dtype=torch.int32))
        a.feed(9)
        a.step()
        b.feed(9)
        b.step()
        graph.replay()
        change(a, ids2, used2)
        torch.cuda.synchronize()
        for x, y in zip((*a.state(), ids2, used2), (*b.state(), ids, used)):
            assert torch.equal(x, y)


def test_two_graphs_with_workspaces_of_their_own_side_by_side():
    note("serving two graphs")
    want, servers, graphs = Server(), [Server(), Server()], []
    streams = [torch.cuda.Stream() for _ in servers]
    for s in (want, *servers):
        s.feed(3)
        s.step()
    for s in servers:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
        graphs.append(graph)
    for turn in range(4):
        for s in (want, *servers):
            s.feed(turn)
        want.step()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s in servers:
            for x, y in zip(want.state(), s.state()):
                assert torch.equal(x, y)


def test_calls_on_a_stream_that_is_given():
    """The calls take a stream as the append and the attention do, with workspaces
    and outputs of their own where none are given."""
    rr = rrmod()
    note("serving streams")
    a, b = Server(), Server()
    for s in (a, b):
        s.feed(1)
        s.step()
        s.feed(2)
    stream = torch.cuda.Stream()
    parent = torch.tensor([0, 0, 2, 3, 4, 4], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    got = []
    for s, st in ((a, None), (b, stream)):
        rr.cache_fork(s.table, s.lengths, s.refs, parent, stream=st)
        missing = rr.cache_resize(s.pools, s.table, s.lengths, s.refs, 1, stream=st)
        accepted, tokens = rr.verify_drafts(s.P, s.drafts, s.u, draft_probs=s.Qd, stream=st)
        x = s.qkv[0][:, :H]
        y = rr.rotate(x, s.positions, s.freqs, axis=s.axis, stream=st)
        ids, used = rr.cache_compact(s.pools, s.table, s.refs, stream=st)
        (st or torch.cuda.current_stream()).synchronize()
        got.append([missing, accepted, tokens, y, ids, used, *s.state()])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    with pytest.raises(ValueError, match="stream"):
        class Other:
            device_index, device, cuda_stream = 7, "cuda:7", 0
        rr.cache_fork(a.table, a.lengths, a.refs, parent, stream=Other())


def test_tensors_of_two_devices_are_refused():
    rr = rrmod()
    note("serving devices")
    s = Server()
    cpu = torch.zeros(6, dtype=torch.int32)
    with pytest.raises(ValueError, match="one device"):
        rr.cache_fork(s.table, s.lengths, s.refs, cpu)
    with pytest.raises(ValueError, match="one device"):
        rr.cache_resize(s.pools, s.table, s.lengths, s.refs, cpu)
    with pytest.raises(ValueError, match="one device"):
        rr.verify_drafts(s.P, s.drafts, s.u.cpu())
    with pytest.raises(ValueError, match="one device"):
        rr.rotate(s.Q[0], s.positions, s.freqs.cpu())
    with pytest.raises(ValueError, match="one device"):
        rr.cache_compact(s.pools, s.table.cpu(), s.refs)


def test_profiled_kinds_of_these_calls():
    rr = rrmod()
    note("serving kinds")
    s = Server()
    s.feed(1)
    rr.profile_start()
    s.step()
    rr.cache_fork(s.table, s.lengths, s.refs, torch.arange(6, dtype=torch.int32, device=DEV))
    rr.cache_compact(s.pools, s.table, s.refs, workspace=s.pages_ws)
    rr.rotate(s.Q[0], s.positions, s.freqs, axis=s.axis)
    got = {k: n for k, (ms, n) in rr.profile_stop().items() if n}
    join = got.pop("join", 0)
    assert got == {"append": LAYERS, "paged": LAYERS, "verify": 1, "pages": 3, "copy": 2, "rotate": 1} and join <= LAYERS


@pytest.mark.parametrize("heads,kv,d,rot", [(32, 8, 128, 128), (24, 4, 160, 96), (5, 3, 1024, 1024), (6, 2, 1024, 0),
                                            (40, 1, 72, 48)])
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("by_axes", [False, True])
def test_large_appends_are_small_ones(heads, kv, d, rot, dtype, cache, inter, by_axes):
    """A call that writes more than the caches hold goes past them: every bit as a
    call for each sequence gives it, in place too; behind the last sequence and
    beyond the table nothing is written."""
    rr = rrmod()
    note("append large", heads, kv, d, rot, dtype, cache, inter, by_axes)
    T = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
    g = torch.Generator(device=DEV).manual_seed(heads + d)
    token = 2 * d * ((heads + kv) * T[dtype].itemsize + kv * T[cache].itemsize)  # read and written
    # (the last sequence has some tokens beyond its pages, and some follow it)
    n0 = 260 * (1 << 20) // token // 2 + 9
    n, page = 2 * n0 + 40, 16
    width = -(-(n0 + 30) // page)
    beyond = n0 + 30 + 10 - width * page
    start = torch.tensor([0, n0 + 10, 2 * n0 + 20], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([n0 + 17, n0 + 40], dtype=torch.int32, device=DEV)
    table = torch.randperm(2 * width, generator=g, device=DEV).to(torch.int32).view(2, width)
    qkv = torch.randn((n, heads + 2 * kv, d), generator=g, device=DEV).to(T[dtype])
    Q, K, V = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    scales = [torch.rand(kv, generator=g, device=DEV) + 0.1 for _ in range(2)] if cache == "e4m3" else [None, None]
    freqs = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / max(1, rot // 2))
    positions = axis = None
    if by_axes:
        positions = torch.randint(0, 5000, (3, n), generator=g, device=DEV).to(torch.int32)
        axis = torch.randint(0, 3, (rot // 2,), generator=g, device=DEV).to(torch.int32)
    pools = [[torch.zeros((2 * width, kv, page, d), device=DEV).to(T[cache]) for _ in range(2)] for _ in range(2)]
    outs = [torch.full((n, heads, d), 7.0, dtype=T[dtype], device=DEV) for _ in range(3)]
    common = dict(freqs=freqs, interleaved=inter, k_scale=scales[0], v_scale=scales[1])
    rr.cache_append(K, V, *pools[0], table, lengths, seq_start=start, Q=Q, Q_out=outs[0], positions=positions, axis=axis, **common)
    step = n0 // 6
    for b in range(2):
        i0, i1 = int(start[b]), int(start[b + 1])
        for i in range(i0, i1, step):
            j = min(i + step, i1)
            part = None if positions is None else positions[:, i:j].contiguous()
            rr.cache_append(K[i:j], V[i:j], *pools[1], table[b:b + 1], lengths[b:b + 1] - (i1 - j), Q=Q[i:j],
                            Q_out=outs[1][i:j], positions=part, axis=axis, **common)
    bits = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])
    assert torch.equal(bits(outs[0]), bits(outs[1]))
    for a, b in zip(*pools):
        assert torch.equal(bits(a), bits(b))
    kept = int(start[2])
    assert bool((outs[0][kept:] == 7.0).all()) and bool((outs[0][kept - max(0, beyond):kept] == 7.0).all())
    assert float(outs[0][:kept - max(0, beyond)].float().std()) > 0.5
    outs[2].copy_(Q)
    rr.cache_append(K, V, *pools[1], table, lengths, seq_start=start, Q=outs[2], Q_out=outs[2], positions=positions, axis=axis,
                    **common)
    assert torch.equal(bits(outs[2][:kept - max(0, beyond)]), bits(outs[0][:kept - max(0, beyond)]))


@pytest.mark.parametrize("heads,kv,d,rot", [(32, 8, 128, 128), (9, 4, 256, 128), (5, 3, 1024, 1024), (6, 2, 1024, 0),
                                            (40, 3, 64, 64), (24, 4, 160, 96)])
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("by_axes", [False, True])
def test_appends_past_the_last_cache(heads, kv, d, rot, dtype, cache, inter, by_axes):
    """More than the last cache holds, read and written together: what is made of
    whole lines goes past it, and every bit is as calls for a part of the tokens
    give it; rows behind the last sequence are left, tokens beyond the table too."""
    rr = rrmod()
    note("append past the last cache", heads, kv, d, rot, dtype, cache, inter, by_axes)
    T = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
    g = torch.Generator(device=DEV).manual_seed(heads + d)
    n0 = (270 << 20) // (2 * d * ((heads + kv) * T[dtype].itemsize + kv * T[cache].itemsize)) // 2 + 7
    n, page = 2 * n0 + 40, 16
    width = -(-(n0 + 30) // page)
    start = torch.tensor([0, n0 + 10, 2 * n0 + 20], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([n0 + 17, n0 + 40], dtype=torch.int32, device=DEV)  # (the second passes its pages)
    table = torch.randperm(2 * width, generator=g, device=DEV).to(torch.int32).view(2, width)
    qkv = torch.empty((n, heads + 2 * kv, d), dtype=T[dtype], device=DEV).normal_(generator=g)
    Q, K, V = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    scales = [torch.rand(kv, generator=g, device=DEV) + 0.1 for _ in range(2)] if cache == "e4m3" else [None, None]
    freqs = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / max(1, rot // 2))
    positions = axis = None
    if by_axes:
        positions = torch.randint(0, 5000, (3, n), generator=g, device=DEV).to(torch.int32)
        axis = torch.randint(-1, 4, (rot // 2,), generator=g, device=DEV).to(torch.int32)
    pools = [[torch.zeros((2 * width, kv, page, d), device=DEV).to(T[cache]) for _ in range(2)] for _ in range(2)]
    outs = [torch.full((n, heads, d), 7.0, dtype=T[dtype], device=DEV) for _ in range(2)]
    common = dict(freqs=freqs, interleaved=inter, k_scale=scales[0], v_scale=scales[1])
    rr.cache_append(K, V, *pools[0], table, lengths, seq_start=start, Q=Q, Q_out=outs[0], positions=positions, axis=axis, **common)
    step = n0 // 3
    for b in range(2):
        i0, i1 = int(start[b]), int(start[b + 1])
        for i in range(i0, i1, step):
            j = min(i + step, i1)
            part = None if positions is None else positions[:, i:j].contiguous()
            rr.cache_append(K[i:j], V[i:j], *pools[1], table[b:b + 1], lengths[b:b + 1] - (i1 - j), Q=Q[i:j],
                            Q_out=outs[1][i:j], positions=part, axis=axis, **common)
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
    for a, b in ((outs[0], outs[1]), *zip(*pools)):
        assert torch.equal(a.view(bits[a.element_size()]), b.view(bits[b.element_size()]))
    assert bool((outs[0][2 * n0 + 20:] == 7.0).all())
    assert not bool((outs[0][0] == 7.0).all()) and bool(pools[0][0].float().any())
    # in place, where rows of queries follow each other
    q = Q.contiguous()
    again = [torch.zeros_like(p) for p in pools[0]]
    rr.cache_append(K, V, *again, table, lengths, seq_start=start, Q=q, Q_out=q, positions=positions, axis=axis, **common)
    end = 2 * n0 + 10  # (the last ones of the second sequence's tokens have no pages, and keep what Q_out held)
    assert torch.equal(q[:end].view(bits[q.element_size()]), outs[0][:end].view(bits[q.element_size()]))
    for a, b in zip(again, pools[0]):
        assert torch.equal(a.view(bits[a.element_size()]), b.view(bits[b.element_size()]))
