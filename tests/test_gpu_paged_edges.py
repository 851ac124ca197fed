"""The paged cache at its edges: queries before their sequence's first token
beside others that see values which are not finite."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import DEV, Cache, _i32, _prefix_cache, _values, note, rrmod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)
    yield


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
