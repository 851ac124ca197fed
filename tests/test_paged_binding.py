"""The paged cache's binding without a GPU: what the library refuses reaches the
caller as it was refused."""
import pytest
import torch


def _rr():
    from paper_2609_07306_amd import routerelay
    return routerelay


@pytest.mark.parametrize("kw,shape,status", [
    ({}, (2, 1, 4, 96), "UNSUPPORTED"),                 # a width that no kernel has
    (dict(n_prefix=8), (2, 1, 4, 96), "UNSUPPORTED"),
    (dict(routes=(8, 3)), (2, 1, 4, 96), "UNSUPPORTED"),
    ({}, (2, 1, 3, 64), "INVALID"),                     # heads that key heads do not divide
    (dict(n_sink=257), (2, 1, 4, 64), "INVALID"),
    (dict(n_prefix=-1), (2, 1, 4, 64), "INVALID"),
    (dict(n_prefix=8, n_recent=1), (2, 1, 4, 64), "INVALID"),
    (dict(n_prefix=8, routes=(8, 3)), (2, 1, 4, 64), "INVALID"),
])
def test_workspace_refusals_carry_their_status(kw, shape, status):
    rr = _rr()
    B, nq, H, d = shape
    Q = torch.zeros(shape, dtype=torch.bfloat16)
    pool, table = torch.zeros((10, 2, 16, d), dtype=torch.bfloat16), torch.zeros((B, 4), dtype=torch.int32)
    if "routes" in kw:
        kw = dict(kw, routes=torch.zeros(kw["routes"], dtype=torch.int32))
    with pytest.raises(rr.RRError) as e:
        rr.paged_workspace(Q, pool, table, **kw)
    assert e.value.status == getattr(rr, "RR_ERR_" + status)
