"""The paged cache's operators as cases to be timed: what a program that answers with a model calls at each layer of
each step.

Kinds of case (``case["kind"]``):

* ``append``  the new tokens' keys and values go into the pages of their sequences, keys (and the queries beside
  them) rotated by their positions on the way;
* ``paged``   one or a few new tokens of every sequence attend to their sequence's cache, to all of it or
  (``k`` > 0) along routes of pages, with the first and the last pages besides;
* ``prefix``  the same for a batch whose sequences begin with the same tokens, which the cache holds once.

Where ``own`` is false, `run` computes them in elementary torch operations in binary32 (angles, and what is next to
a border of 8 bits, in binary64), where it is true through the public binding.  Sequence lengths follow from the case
alone, so that its work does; the seed makes values, pages and routes.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


def listed():
    return [
        # one token of one sequence, the smallest call: latency alone
        _append("append one token", 32, 8, 128, "bf16", "bf16", 256, 1, 1, 1, 700, 128),
        # a decode step of a large batch of young sequences into an 8-bit cache
        _append("append decode batch e4m3", 32, 8, 128, "bf16", "e4m3", 16, 192, 1, 1, 64, 128),
        # a long prompt, rows of a fused projection, chunks of the benchmark's prefill point
        _append("append prompt", 32, 8, 128, "bf16", "bf16", 256, 1, 32768, 32768, 32768, 128, fused=True),
        # prompts of odd lengths with rows left over, binary32, a quarter of each row rotated in neighbour pairs
        _append("append ragged f32", 6, 2, 64, "f32", "f32", 48, 24, 0, 1, 700, 32, inter=True, left=37),
        # one sequence's decode step: the key axis has to be split to fill the card
        _paged("decode one sequence", 32, 8, 128, "bf16", "bf16", 64, 1, 1, 8192, 8192),
        # a decode step of a batch whose lengths differ a hundredfold
        _paged("decode ragged batch", 32, 8, 128, "bf16", "bf16", 64, 64, 1, 300, 32768),
        # 8-bit cache, small pages
        _paged("decode batch e4m3", 32, 8, 128, "bf16", "e4m3", 16, 128, 1, 100, 16384),
        # five draft tokens to verify, binary32, pages of an odd size
        _paged("draft tokens f32", 6, 2, 64, "f32", "f32", 48, 7, 5, 5, 5000),
        # long contexts along routes: the benchmark's prefill context and route width
        _paged("decode along routes", 32, 8, 128, "bf16", "bf16", 256, 8, 1, 100000, 131072, 32, 1, 2),
        # a few answers to one prompt, sampled side by side
        _prefix("few after a prompt", 8, 2, 64, "bf16", "bf16", 32, 6, 1, 2000, 1, 130),
        # a batch behind one system prompt
        _prefix("batch after a prompt", 32, 8, 128, "bf16", "bf16", 64, 64, 1, 8192, 16, 1024),
        # the largest: two draft tokens each of a large batch behind a long document
        _prefix("drafts after a document", 32, 8, 128, "bf16", "bf16", 64, 160, 2, 32768, 64, 2048),
    ]


def _append(name, heads, kv, d, dtype, cache, page, batch, new, shortest, longest, rot, inter=False, fused=False,
            left=0):
    """new = 0: every sequence's tokens are all new, `left` rows follow the last one's."""
    c = dict(kind="append", heads=heads, kv_heads=kv, d=d, dtype=dtype, cache=cache, page=page, batch=batch, new=new,
             shortest=shortest, longest=longest, rot=rot, inter=inter, fused=fused, left=left)
    return dict(c, name=name) if name else c


def _paged(name, heads, kv, d, dtype, cache, page, batch, nq, shortest, longest, k=0, sinks=0, recent=0):
    c = dict(kind="paged", heads=heads, kv_heads=kv, d=d, dtype=dtype, cache=cache, page=page, batch=batch, nq=nq,
             shortest=shortest, longest=longest, k=k, sinks=sinks, recent=recent)
    return dict(c, name=name) if name else c


def _prefix(name, heads, kv, d, dtype, cache, page, batch, nq, prefix, shortest, longest):
    """shortest, longest: of what follows the shared tokens."""
    c = dict(kind="prefix", heads=heads, kv_heads=kv, d=d, dtype=dtype, cache=cache, page=page, batch=batch, nq=nq,
             prefix=prefix, shortest=shortest, longest=longest)
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "paged", "paged", "paged", "prefix", "prefix"])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
    kv = rng.choice([1, 2, 3, 4, 8, 8])
    heads = kv * rng.choice([1, 2, 4, 4, 7, 8])
    d = rng.choice([64, 128, 128, 256] if dtype == "bf16" else [64, 128])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256, _log(rng, 5, 300)])
    row = kv * d * BYTES[cache]  # bytes of a token's keys
    if kind == "append":
        rot = rng.choice([d, d, d // 2, 0])
        inter = rng.random() < 0.3
        if rng.random() < 0.5:  # a decode step, drafts among them
            batch, new = _log(rng, 1, 256), rng.choice([1, 1, 1, 2, 5])
            return _append("", heads, kv, d, dtype, cache, page, batch, new, new, new + _log(rng, 1, 100), rot, inter,
                           rng.random() < 0.5)
        longest = _log(rng, 20, 8192)
        batch = _log(rng, 1, max(1, min(64, (1 << 25) // (longest * row))))
        return _append("", heads, kv, d, dtype, cache, page, batch, 0, max(1, longest // 20), longest, rot, inter,
                       rng.random() < 0.5, rng.choice([0, 5]))
    nq = rng.choice([1, 1, 1, 1, 2, 4, 7])
    batch = _log(rng, 1, 128)
    if kind == "prefix":
        batch = max(2, batch)
        while batch * nq * heads > 4096:
            batch = max(2, batch // 2)
            nq = max(1, nq // 2)
        prefix = min(_log(rng, 100, 16384), (1 << 26) // row)
        longest = nq + min(_log(rng, 1, 1024), max(1, (1 << 28) // (row * batch)))
        return _prefix("", heads, kv, d, dtype, cache, page, batch, nq, prefix, nq, longest)
    longest = nq + min(_log(rng, 10, 32768), (1 << 29) // (row * batch))
    shortest = min(longest, nq + longest // 50)
    if rng.random() < 0.3 and longest >= 8 * page:
        k = min(_log(rng, 2, 48), longest // page)
        while batch * nq * heads * k * page * d > 1 << 30:  # (the plain form's copies)
            batch, k = max(1, batch // 2), max(2, k // 2)
        return _paged("", heads, kv, d, dtype, cache, page, batch, nq, shortest, longest, k, rng.choice([0, 1]),
                      rng.choice([1, 2]))
    return _paged("", heads, kv, d, dtype, cache, page, batch, nq, shortest, longest)


def _lengths(c):
    """Every sequence's tokens, the new ones (and a shared prefix) counted: spread between shortest and longest over
    their logarithm, the last one the longest."""
    lo, hi = math.log(c["shortest"]), math.log(c["longest"])
    n = [int(round(math.exp(lo + (hi - lo) * ((i + 1) * 0.6180339887498949 % 1.0)))) for i in range(c["batch"] - 1)]
    return [c.get("prefix", 0) + x for x in n + [c["longest"]]]


def _new(c):
    """New tokens of every sequence of an append."""
    return [c["new"] or n for n in _lengths(c)]


def _frequencies(c):
    return 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / max(1, c["rot"]))


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    H, Hkv, d, page, B = c["heads"], c["kv_heads"], c["d"], c["page"], c["batch"]
    dt = TYPES[c["dtype"]]
    lens = _lengths(c)
    shared = c.get("prefix", 0)
    # whole pages of the shared tokens are held once; a page that they end in is every sequence's own
    held = shared // page
    own_pages = [max(1, -(-n // page)) - held for n in lens]
    n_shared = -(-shared // page)
    n_pages = n_shared + sum(own_pages) + 3
    width = held + max(own_pages) + 2

    def randn(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=DEV) * scale

    # keys and values as the cache holds them: 8 bits hold them over a scale per head
    pools, scales = [], (None, None)
    if c["cache"] == "e4m3":
        scales = tuple(0.01 + 0.02 * torch.rand(Hkv, generator=g, device=DEV) for _ in range(2))
        for s in scales:
            x = randn(n_pages, Hkv, page, d) / s[:, None, None]
            pools.append(x.clamp_(-448.0, 448.0).to(E4M3))
    else:
        pools = [randn(n_pages, Hkv, page, d).to(TYPES[c["cache"]]) for _ in range(2)]
    # pages in any order; entries past a sequence's last page are empty
    order = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = n_shared
    for b, n in enumerate(own_pages):
        table[b, :held] = order[:held]
        table[b, held:held + n] = order[at:at + n]
        at += n
    s = dict(case=c, K_cache=pools[0], V_cache=pools[1], table=table, k_scale=scales[0], v_scale=scales[1],
             lengths=torch.tensor(lens, dtype=torch.int32, device=DEV))
    if c["kind"] == "append":
        new = _new(c)
        n = sum(new) + c["left"]
        starts = [0] + torch.tensor(new).cumsum(0).tolist()
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        s["freqs"] = _frequencies(c)
        if c["fused"]:
            qkv = randn(n, H + 2 * Hkv, d).to(dt)
            s["Q"], s["K"], s["V"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        else:
            s["Q"], s["K"], s["V"] = (randn(n, h, d).to(dt) for h in (H, Hkv, Hkv))
        # (rows past the last sequence's stay what they are)
        s["Q_out"] = torch.zeros((n, H, d), dtype=dt, device=DEV)
        return s
    # scores of a standard deviation of two: some tokens stand out, as they do in a trained model
    s["Q"] = randn(B, c["nq"], H, d, scale=2.0).to(dt)
    if c["kind"] == "prefix":
        s["pages"] = order[:n_shared].clone()
        if held < n_shared:  # the page that the shared tokens end in: every copy begins with them
            tail = shared - held * page
            src, dst = order[held].long(), table[:, held].long()
            for p in pools:
                bits = p.view(torch.uint8) if p.dtype == E4M3 else p
                bits[dst, :, :tail] = bits[src, :, :tail]
    elif c["k"]:
        n_rows, most = B * H * c["nq"], width
        pick = torch.rand((n_rows, most), generator=g, device=DEV)
        chunks = -(-s["lengths"].long() // page)
        rows = torch.arange(n_rows, device=DEV) // (H * c["nq"])
        pick.masked_fill_(torch.arange(most, device=DEV)[None] >= chunks[rows][:, None], -1.0)
        top = pick.topk(c["k"], dim=1)
        ids = torch.where(top.values >= 0, top.indices, torch.full_like(top.indices, most))
        ids = ids.sort(dim=1).values
        s["routes"] = torch.where(ids < most, ids, torch.full_like(ids, -1)).to(torch.int32)
    return s


def run(state):
    kind = state["case"]["kind"]
    if kind == "append":
        return _run_append(state)
    return {"O": _run_paged(state) if kind == "paged" else _run_prefix(state)}


def _keep(s, **more):
    """The workspace that a program keeps for the calls of one shape."""
    from paper_2609_07306_amd import routerelay as rr
    if "workspace" not in s:
        s["workspace"] = rr.paged_workspace(s["Q"], s["K_cache"], s["table"], **more)
    return rr, s["workspace"]


# ------------------------------------------------------------------ append

def _rotated(x, angle, inter, wide):
    """Rows [n, heads, d] rotated by [n, rot / 2] angles, in binary32 (wide: binary64)."""
    t = torch.float64 if wide else torch.float32
    cos, sin = angle.cos().to(t)[:, None], angle.sin().to(t)[:, None]
    r = 2 * angle.shape[1]
    x = x.to(t)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if inter else (x[..., :r // 2], x[..., r // 2:r])
    y, z = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((y, z), -1).flatten(-2) if inter else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _run_append(s):
    c = s["case"]
    if own:
        from paper_2609_07306_amd import routerelay as rr
        rr.cache_append(s["K"], s["V"], s["K_cache"], s["V_cache"], s["table"], s["lengths"],
                        seq_start=s["starts"] if c["new"] == 0 else None, freqs=s["freqs"] if c["rot"] else None,
                        interleaved=c["inter"], Q=s["Q"], Q_out=s["Q_out"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {"K_cache": s["K_cache"], "V_cache": s["V_cache"], "Q": s["Q_out"]}
    n = s["K"].shape[0] - c["left"]
    i = torch.arange(n, device=DEV)
    b = torch.searchsorted(s["starts"][1:].long(), i, right=True)
    pos = s["lengths"][b].long() - s["starts"][b + 1] + i
    phys = s["table"][b, pos // c["page"]].long()
    off = pos % c["page"]
    angle = pos.double()[:, None] * s["freqs"]
    wide = c["cache"] == "e4m3"
    for x, pool, scale in ((_rotated(s["K"][:n], angle, c["inter"], wide), s["K_cache"], s["k_scale"]),
                           (s["V"][:n], s["V_cache"], s["v_scale"])):
        if wide:
            x = (x.double() / scale.double()[:, None]).clamp(-448.0, 448.0).float().to(E4M3)
            pool.view(torch.uint8)[phys, :, off] = x.view(torch.uint8)
        else:
            pool[phys, :, off] = x.to(pool.dtype)
    s["Q_out"][:n] = _rotated(s["Q"][:n], angle, c["inter"], False).to(s["Q"].dtype)
    return {"K_cache": s["K_cache"], "V_cache": s["V_cache"], "Q": s["Q_out"]}


# --------------------------------------------------------------- attention

def _pages(pool, ids):
    """The values of the pages `ids` [..., n] as [..., kv heads, n * page, d] in binary32, before any scale."""
    ids = ids.clamp(min=0).long()
    x = pool.view(torch.uint8)[ids].view(pool.dtype) if pool.dtype == E4M3 else pool[ids]
    return x.transpose(-4, -3).flatten(-3, -2).float()


def _grouped(s):
    """Queries [B, kv heads, nq * group, d] in binary32, scaled; row t * group + j."""
    c = s["case"]
    g = c["heads"] // c["kv_heads"]
    q = s["Q"].float().view(c["batch"], c["nq"], c["kv_heads"], g, c["d"]) / math.sqrt(c["d"])
    if s["k_scale"] is not None:
        q = q * s["k_scale"][:, None, None]
    return q.transpose(1, 2).flatten(2, 3)


def _ungrouped(s, o):
    c = s["case"]
    if s["v_scale"] is not None:
        o = o * s["v_scale"][:, None, None]
    return o.unflatten(2, (c["nq"], -1)).transpose(1, 2).flatten(2, 3).to(s["Q"].dtype)


def _last_seen(s):
    """The last token that each row of _grouped sees, [B, nq * group]."""
    c = s["case"]
    t = torch.arange(c["nq"], device=DEV).repeat_interleave(c["heads"] // c["kv_heads"])
    return s["lengths"].long()[:, None] - c["nq"] + t


def _softmax_parts(scores, seen):
    w = scores.masked_fill(~seen, -math.inf)
    top = w.amax(-1, keepdim=True).clamp(min=-1e30)
    return (w - top).exp()


def _run_paged(s):
    c = s["case"]
    if own:
        more = dict(routes=s["routes"], n_sink=c["sinks"], n_recent=c["recent"]) if c["k"] else {}
        rr, ws = _keep(s, **more)
        return rr.paged_attention(s["Q"], s["K_cache"], s["V_cache"], s["table"], s["lengths"], workspace=ws,
                                  k_scale=s["k_scale"], v_scale=s["v_scale"], **more)
    if c["k"]:
        return _routed_plain(s)
    q, last = _grouped(s), _last_seen(s)
    k, v = _pages(s["K_cache"], s["table"]), _pages(s["V_cache"], s["table"])
    u = torch.arange(k.shape[2], device=DEV)
    seen = u <= last[:, None, :, None]
    w = _softmax_parts(q @ k.transpose(-1, -2), seen)
    v = v.masked_fill(~(u[:, None] <= last.amax(1)[:, None, None, None]), 0.0)
    return _ungrouped(s, (w @ v) / w.sum(-1, keepdim=True).clamp(min=1e-30))


def _routed_plain(s):
    """Every (sequence, head, query) row over its own pages: the routes, the first and the last ones, each once."""
    c = s["case"]
    B, H, nq, page, g = c["batch"], c["heads"], c["nq"], c["page"], c["heads"] // c["kv_heads"]
    routes = s["routes"].long().view(B, H, nq, c["k"])
    last = (s["lengths"].long()[:, None] - nq + torch.arange(nq, device=DEV))[:, None, :, None].expand(B, H, nq, 1)
    here = last.div(page, rounding_mode="floor")
    sinks = torch.arange(c["sinks"], device=DEV).expand(B, H, nq, -1)
    recent = here - torch.arange(c["recent"], device=DEV)
    ids = torch.cat((sinks, recent, routes), -1)
    ids = torch.where((ids >= 0) & (ids <= here), ids, torch.full_like(ids, -1)).sort(-1).values
    again = torch.cat((torch.zeros_like(ids[..., :1], dtype=torch.bool), ids[..., 1:] == ids[..., :-1]), -1)
    ids = torch.where(again, torch.full_like(ids, -1), ids)
    b, h = torch.arange(B, device=DEV)[:, None, None, None], torch.arange(H, device=DEV)[:, None, None]
    phys = s["table"][b, ids.clamp(min=0)].long().clamp(min=0)
    kv = (h // g).expand_as(phys)

    def tokens(pool):  # [B, H, nq, pages * page, d]
        bits = pool.view(torch.uint8) if pool.dtype == E4M3 else pool
        x = bits[phys, kv]
        return (x.view(E4M3) if pool.dtype == E4M3 else x).float().flatten(3, 4)

    u = (ids[..., None] * page + torch.arange(page, device=DEV)).flatten(3, 4)
    seen = (u <= last) & (ids >= 0).repeat_interleave(page, -1)
    q = s["Q"].float().transpose(1, 2) / math.sqrt(c["d"])
    if s["k_scale"] is not None:
        q = q * s["k_scale"].repeat_interleave(g)[:, None, None]
    w = _softmax_parts((tokens(s["K_cache"]) @ q[..., None]).squeeze(-1), seen)
    o = (w[..., None, :] @ tokens(s["V_cache"])).squeeze(-2) / w.sum(-1, keepdim=True).clamp(min=1e-30)
    if s["v_scale"] is not None:
        o = o * s["v_scale"].repeat_interleave(g)[:, None, None]
    return o.transpose(1, 2).to(s["Q"].dtype)


def _run_prefix(s):
    c = s["case"]
    n, B, R = c["prefix"], c["batch"], c["nq"] * (c["heads"] // c["kv_heads"])
    if own:
        rr, ws = _keep(s, n_prefix=n)
        return rr.prefix_attention(s["Q"], s["K_cache"], s["V_cache"], s["table"], s["lengths"], s["pages"], n,
                                   workspace=ws, k_scale=s["k_scale"], v_scale=s["v_scale"])
    q, last = _grouped(s), _last_seen(s)
    flat = q.transpose(0, 1).flatten(1, 2)  # every row of a key head against the shared tokens
    k0, v0 = _pages(s["K_cache"], s["pages"])[:, :n], _pages(s["V_cache"], s["pages"])[:, :n]
    shared = (flat @ k0.transpose(-1, -2)).unflatten(1, (B, R)).transpose(0, 1)
    held = n // c["page"]  # each sequence's table from the page that the shared tokens end in
    k1, v1 = _pages(s["K_cache"], s["table"][:, held:]), _pages(s["V_cache"], s["table"][:, held:])
    u = torch.cat((torch.arange(n, device=DEV), held * c["page"] + torch.arange(k1.shape[2], device=DEV)))
    seen = (u <= last[:, None, :, None]) & ((torch.arange(u.numel(), device=DEV) < n) | (u >= n))
    w = _softmax_parts(torch.cat((shared, q @ k1.transpose(-1, -2)), -1), seen)
    w0 = w[..., :n].transpose(0, 1).flatten(1, 2)
    o = (w0 @ v0).unflatten(1, (B, R)).transpose(0, 1) + w[..., n:] @ v1
    return _ungrouped(s, o / w.sum(-1, keepdim=True).clamp(min=1e-30))


# -------------------------------------------------------------------- work

def work(case):
    c = case
    H, Hkv, d, lens = c["heads"], c["kv_heads"], c["d"], _lengths(c)
    e, ce = BYTES[c["dtype"]], BYTES[c["cache"]]
    if c["kind"] == "append":
        n = sum(_new(c))
        return {"bytes": n * d * (2 * H * e + 2 * Hkv * (e + ce)) + 8 * c["batch"],
                "flops": 3 * n * (H + Hkv) * c["rot"] + (n * 2 * Hkv * d if ce == 1 else 0)}
    qo = 2 * c["batch"] * c["nq"] * H * d * e
    # (query, token) pairs of a head: query t of n sees n - nq + t + 1
    pairs = sum(max(0, n - c["nq"] + t + 1) for n in lens for t in range(c["nq"]))
    if c.get("k"):
        slots = c["k"] + c["sinks"] + c["recent"]
        rows = c["nq"] * (H // Hkv)
        pairs = sum(min(slots * c["page"], n) * c["nq"] for n in lens)
        # pages of a key head that at least one of its rows takes
        taken = [n / c["page"] * (1 - max(0.0, 1 - slots * c["page"] / n) ** rows) for n in lens]
        return {"bytes": int(sum(taken) * c["page"] * Hkv * d * 2 * ce + qo + 4 * c["batch"] * H * c["nq"] * c["k"]),
                "flops": 4 * d * H * pairs}
    n = c.get("prefix", 0)
    tokens = n + sum(max(0, x - n) for x in lens)
    return {"bytes": tokens * Hkv * d * 2 * ce + qo, "flops": 4 * d * H * pairs}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """The same from the definitions in binary64, a sequence at a time."""
    c, s = case, prepare(case, seed)
    Hkv, d, page, nq = c["kv_heads"], c["d"], c["page"], c.get("nq", 0)
    table, lens = s["table"].cpu(), _lengths(c)

    def value(x, scale=None):
        x = x.to(torch.float64)
        return x if scale is None else x * scale.double()[:, None, None]

    if c["kind"] == "append":
        K, V, Q = value(s["K_cache"]), value(s["V_cache"]), torch.zeros_like(s["Q_out"], dtype=torch.float64)
        at, half = 0, c["rot"] // 2
        first = torch.arange(half, device=DEV) * (2 if c["inter"] else 1)
        second = first + (1 if c["inter"] else half)
        for b, n in enumerate(_new(c)):
            place = torch.arange(lens[b] - n, lens[b], device=DEV)
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                               place.double()[:, None, None] * s["freqs"])
            rows = slice(at, at + n)
            at += n
            for x, y in ((s["K"][rows], None), (s["Q"][rows], Q[rows])):
                x = x.double()
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
                if y is not None:
                    y.copy_(x)
                    continue
                v = s["V"][rows].double()
                if c["cache"] == "e4m3":
                    x = (x / s["k_scale"].double()[:, None]).clamp(-448, 448)
                    v = (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
                phys = s["table"][b].long()[place // page]
                K[phys, :, place % page] = x
                V[phys, :, place % page] = v
        return {"K_cache": K, "V_cache": V, "Q": Q}

    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    g = c["heads"] // Hkv

    def attend(q, k, v):  # [rows, d] x [tokens, d]
        x = (k @ q.T) * (1.0 / math.sqrt(d))
        p = torch.exp(x - x.max(0).values)
        return (p / p.sum(0)).T @ v

    for b, n in enumerate(lens):
        u = torch.arange(n, device=DEV)
        phys = s["table"][b].long()[u // page]
        if c.get("k"):
            rows = s["routes"].view(c["batch"], c["heads"], nq, c["k"])[b].cpu().tolist()
            for t in range(nq):
                last = n - nq + t
                more = set(range(c["sinks"])) | {last // page - i for i in range(c["recent"])}
                for h in range(c["heads"]):
                    ids = sorted(j for j in more | set(rows[h][t]) if 0 <= j <= last // page)
                    if not ids:
                        continue
                    at = (torch.tensor(ids, device=DEV)[:, None] * page + torch.arange(page, device=DEV)).flatten()
                    at = at[at <= last]
                    k, v = (value(p[phys[at], h // g, at % page]) for p in (s["K_cache"], s["V_cache"]))
                    if s["k_scale"] is not None:
                        k, v = k * s["k_scale"][h // g].double(), v * s["v_scale"][h // g].double()
                    O[b, t, h] = attend(s["Q"][b, t, h].double()[None], k, v)[0]
            continue
        if c["kind"] == "prefix":
            phys = torch.where(u < c["prefix"], s["pages"].long()[(u // page).clamp(max=len(s["pages"]) - 1)], phys)
        for h in range(Hkv):
            k, v = (value(p.view(torch.uint8)[phys, h, u % page].view(E4M3) if p.dtype == E4M3 else
                          p[phys, h, u % page]) for p in (s["K_cache"], s["V_cache"]))
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            for t in range(nq):
                m = n - nq + t + 1
                if m > 0:
                    O[b, t, h * g:(h + 1) * g] = attend(s["Q"][b, t, h * g:(h + 1) * g].double(), k[:m], v[:m])
    return {"O": O}
