"""Numbers past 32 bits, to which ctypes would cut them without a word, are
refused by the binding before any call: a chunk of 2^32 + 5 tokens was taken as
one of 5, beyond the outputs that the binding had made for the former.  (Without
a GPU: large tensors are views of one element or have no memory at all.)"""
import pytest
import torch

BF, I32, F64 = torch.bfloat16, torch.int32, torch.float64
MANY = 2 ** 32 + 1


@pytest.fixture
def rr(monkeypatch):
    from paper_2609_07306_amd import routerelay
    monkeypatch.setattr(routerelay, "_device_of", lambda tensors: 0)
    monkeypatch.setattr(routerelay, "_launch", lambda *a: pytest.fail("launched"))
    monkeypatch.setattr(routerelay, "_ptr", lambda t: pytest.fail("taken"))
    return routerelay


def refused():
    return pytest.raises(ValueError, match="32 bits")


def _no_memory(*shape, dtype=I32):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("n", [MANY, 2 ** 31, -2 ** 31 - 1, 1 - 2 ** 32])
def test_new_tokens(rr, n):
    pool = torch.zeros((10, 2, 16, 64), dtype=BF)
    table, lens, refs = torch.zeros((2, 4), dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(10, dtype=I32)
    with refused():
        rr.cache_resize(rr.Pools(pool, pool), table, lens, refs, n, workspace=torch.zeros(4096, dtype=torch.uint8))


@pytest.mark.parametrize("name", ["n_sink", "n_recent", "n_prefix"])
@pytest.mark.parametrize("n", [MANY, 2 ** 31, 1 - 2 ** 32])
def test_pages_that_a_query_sees_besides(rr, name, n):
    Q, pool = torch.zeros((2, 1, 4, 64), dtype=BF), torch.zeros((10, 2, 16, 64), dtype=BF)
    table = torch.zeros((2, 4), dtype=I32)
    with refused():
        rr.paged_workspace(Q, pool, table, **{name: n})
    with refused():
        lens = torch.zeros(2, dtype=I32)
        if name == "n_prefix":
            rr.prefix_attention(Q, pool, pool, table, lens, torch.zeros(1, dtype=I32), n)
        else:
            rr.paged_attention(Q, pool, pool, table, lens, **{name: n})


def test_chunks(rr):
    with refused():
        rr.pool_chunks(torch.zeros((2, 100, 64)), MANY)
    with refused():
        rr.expand_tokens(torch.zeros((2, 0), dtype=I32), MANY, 100)
    with refused():
        rr.expand_tokens(torch.zeros((2, 3), dtype=I32), 5, MANY)
    x = torch.zeros((2, 100, 64), dtype=BF)
    with refused():
        rr.sparse_attention(x, x, x, torch.zeros((2, 3), dtype=I32), MANY, True)


def test_configurations_and_layers(rr):
    base = dict(n_heads=2, n_kv_heads=1, n_q=8, n_k=8, d=64, k=4)
    rr.Config(**base).c()
    for name in [*base, "m", "r", "n_sink", "n_recent", "min_reuse"]:
        with refused():
            rr.Config(**dict(base, **{name: MANY})).c()
    cfg, x = rr.Config(**base), torch.zeros((2, 8, 64))
    with refused():
        rr.relay_static(cfg, MANY, x, x[:1], {})
    ledger = object.__new__(rr.Ledger)
    ledger.cfg, ledger._h = cfg, None
    for call in (ledger.anchor, ledger.relay):
        with refused():
            call(MANY, x, x[:1])
    with refused():
        ledger.import_(MANY, None, None, None, None)
    with refused():
        rr.set_sweep_cap(MANY)


def test_tensors_of_the_paged_cache(rr):
    one, pool = torch.zeros((1, 2, 64), dtype=BF), torch.zeros((10, 2, 16, 64), dtype=BF)
    table, lens = torch.zeros((2, 4), dtype=I32), torch.zeros(2, dtype=I32)
    many = one.expand(MANY, 2, 64)
    with refused():
        rr.cache_append(many, many, pool, pool, table, lens)
    with refused():
        rr.cache_append(one, one, pool, pool, _no_memory(1, MANY), lens[:1])
    large = _no_memory(MANY, 2, 16, 64, dtype=BF)
    with refused():
        rr.cache_append(one, one, large, large, table, lens)
    Q = torch.zeros((2, 1, 4, 64), dtype=BF)
    with refused():
        rr.paged_attention(Q, large, large, table, lens)
    with refused():
        rr.paged_attention(Q, pool, pool, _no_memory(2, MANY), lens)
    with refused():
        rr.paged_attention(Q, pool, pool, table, lens, routes=_no_memory(8, MANY))
    with refused():
        rr.Pools(large, large)


def test_rows_and_drafts(rr):
    one, f = torch.zeros((1, 1, 8), dtype=BF), torch.zeros(4, dtype=F64)
    many, out = one.expand(MANY, 1, 8), _no_memory(MANY, 1, 8, dtype=BF)
    with refused():
        rr.rotate(many, _no_memory(1, MANY), f, out=out)
    with refused():
        rr.rotate(many, torch.zeros((1, 1), dtype=I32), f, tokens=1, out=out)
    with refused():
        rr.rotate(one, _no_memory(MANY, 1), f, out=torch.zeros_like(one))
    P = torch.zeros((1, 2, 5))
    with refused():
        rr.verify_drafts(P.expand(MANY, 2, 5), _no_memory(MANY, 1), _no_memory(MANY, 2, dtype=torch.float32))
    with refused():
        rr.verify_workspace(P.expand(MANY, 2, 5))


def test_page_tables(rr):
    table, lens, refs = torch.zeros((2, 4), dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(10, dtype=I32)
    with refused():
        rr.cache_fork(table, lens, _no_memory(MANY), lens)
    with refused():
        rr.cache_fork(_no_memory(2, MANY), lens, refs, lens)
    pool = torch.zeros((10, 2, 16, 64), dtype=BF)
    pools = rr.Pools(pool, pool)
    for new in (1, lens):
        with refused():
            rr.cache_resize(pools, _no_memory(2, MANY), lens, refs, new)
    with refused():
        rr.cache_compact(pools, _no_memory(2, MANY), refs)
