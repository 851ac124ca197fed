"""More operators around the paged cache as cases to be timed: what a program that answers with a model calls beside the
append and the attention.

Kinds of case (``case["kind"]``):

* ``rotate``   queries or keys that no cache holds (yet) are rotated by positions of several axes (time, height and width
  of an image's or a film's token; a text token has the same position on all of them), or back, as gradients are;
* ``append``   the same on the way into the pages of a cache;
* ``verify``   drafted tokens are checked against the target's probabilities, one more token is drawn;
* ``fork``     sequences go on from others: samples of one prompt, the beams of a search;
* ``resize``   page tables follow the sequences' lengths: pages past the end are freed, new tokens get pages, and a page
  that other sequences hold too is copied before it is written;
* ``compact``  used pages move together, so that the rest of the pools can be given away.

Where ``own`` is false, `run` computes them in elementary torch operations (in binary64 what is next to a border: angles,
probabilities), where it is true through the public binding.  What a case has to move follows from the case alone; the
seed makes values, the order of pages and what is drawn.  The three calls on page tables change them in place, so a pass
begins by setting them back, in one copy.
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
        # the gradient of a small picture's queries, a few heads in binary32, neighbours rotated: latency
        _rotate("rotate picture gradient f32", 6, 64, "f32", 196, 2, 64, inter=True, inverse=True),
        # a film's queries on their way to chunk pooling and routing: the benchmark's prefill heads and context
        _rotate("rotate film", 32, 128, "bf16", 32768, 3, 128, heads_first=True),
        # a decode step of a batch whose prompts held pictures
        _append("append decode axes", 32, 8, 128, "bf16", "bf16", 64, 64, 1, 1, 2000, 3, 128),
        # prompts with pictures of odd lengths, rows of a fused projection, an 8-bit cache
        _append("append prompts axes e4m3", 32, 8, 128, "bf16", "e4m3", 64, 24, 0, 30, 4000, 3, 128, fused=True),
        # one sequence's drafts: the vocabulary has to be split to fill the card
        _verify("verify one sequence", 1, 4, 32000, "f32"),
        # the drafts of a large batch, a large vocabulary
        _verify("verify batch", 192, 5, 131072, "f32"),
        # four answers each to a few prompts: latency
        _fork("fork samples", 16, 128, 64, 4, 100, 6000, beams=False),
        # beams of a large batch go on from the best ones
        _fork("fork beams", 512, 1024, 16, 8, 500, 16000, beams=True),
        # drafts after one token: a decode step's bookkeeping, nobody shares a page that is written
        _resize("resize decode", 8, 128, "bf16", 64, 64, 256, 1, 5, 300, 12000, 8),
        # samples just forked write their first token: every group's last page is copied for all but one
        _resize("resize after fork", 8, 128, "bf16", 64, 128, 128, 4, 1, 100, 4000, 16),
        # a small 8-bit pool after a few sequences ended
        _compact("compact small e4m3", 2, 64, "e4m3", 16, 300, 0.7, 12, 4),
        # a large pool, half of which has fallen free
        _compact("compact pool", 8, 128, "bf16", 64, 2400, 0.5, 64, 4),
    ]


def _named(name, c):
    return dict(c, name=name) if name else c


def _rotate(name, heads, d, dtype, tokens, axes, rot, heads_first=False, inter=False, inverse=False, fractions=False):
    """fractions: positions are binary32 numbers (seconds of a film), otherwise int32."""
    return _named(name, dict(kind="rotate", heads=heads, d=d, dtype=dtype, tokens=tokens, axes=axes, rot=rot,
                             heads_first=heads_first, inter=inter, inverse=inverse, fractions=fractions))


def _append(name, heads, kv, d, dtype, cache, page, batch, new, shortest, longest, axes, rot, inter=False, fused=False,
            fractions=False):
    """new = 0: every sequence's tokens are all new."""
    return _named(name, dict(kind="append", heads=heads, kv_heads=kv, d=d, dtype=dtype, cache=cache, page=page,
                             batch=batch, new=new, shortest=shortest, longest=longest, axes=axes, rot=rot, inter=inter,
                             fused=fused, fractions=fractions))


def _verify(name, batch, drafts, vocab, dtype, given=True, ragged=False, kept=0.0, pad=0):
    """given: the drafts come with the probabilities that they were drawn with (otherwise they were looked up); kept: the
    least probability that a truncated distribution keeps, 0: all; pad: columns behind the vocabulary's."""
    return _named(name, dict(kind="verify", batch=batch, drafts=drafts, vocab=vocab, dtype=dtype, given=given,
                             ragged=ragged, kept=kept, pad=pad))


def _fork(name, batch, max_pages, page, group, shortest, longest, beams):
    return _named(name, dict(kind="fork", batch=batch, max_pages=max_pages, page=page, group=group, shortest=shortest,
                             longest=longest, beams=beams))


def _resize(name, kv, d, cache, page, batch, max_pages, group, new, shortest, longest, pools):
    """group: sequences that were one until now; new = 0: every sequence's tokens are all new; pools: of all layers."""
    return _named(name, dict(kind="resize", kv_heads=kv, d=d, cache=cache, page=page, batch=batch, max_pages=max_pages,
                             group=group, new=new, shortest=shortest, longest=longest, pools=pools))


def _compact(name, kv, d, cache, page, n_pages, used, batch, pools):
    return _named(name, dict(kind="compact", kv_heads=kv, d=d, cache=cache, page=page, n_pages=n_pages, used=used,
                             batch=batch, pools=pools))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "append", "verify", "verify", "verify", "fork", "fork", "resize",
                       "resize", "resize", "compact", "compact"])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
    kv = rng.choice([1, 2, 3, 4, 8, 8])
    heads = kv * rng.choice([1, 2, 4, 4, 7, 8])
    d = rng.choice([64, 128, 128, 256] if dtype == "bf16" else [64, 128])
    page = rng.choice([16, 16, 32, 64, 64, 128, _log(rng, 5, 200)])
    axes, inter, fractions = rng.choice([1, 2, 3, 3, 4]), rng.random() < 0.3, rng.random() < 0.25
    rot = rng.choice([d, d, d // 2])
    if kind == "rotate":
        tokens = min(_log(rng, 1, 32768), (1 << 28) // (heads * d * BYTES[dtype]))
        return _rotate("", heads, d, dtype, tokens, axes, rot, rng.random() < 0.5, inter, rng.random() < 0.4, fractions)
    if kind == "append":
        if rng.random() < 0.5:
            batch, new = _log(rng, 1, 256), rng.choice([1, 1, 1, 2, 5])
            return _append("", heads, kv, d, dtype, cache, page, batch, new, new, new + _log(rng, 1, 300), axes, rot,
                           inter, rng.random() < 0.5, fractions)
        longest = _log(rng, 20, 6000)
        batch = _log(rng, 1, max(1, min(48, (1 << 25) // (longest * (heads + 2 * kv) * d // 4))))
        return _append("", heads, kv, d, dtype, cache, page, batch, 0, max(1, longest // 20), longest, axes, rot, inter,
                       rng.random() < 0.5, fractions)
    if kind == "verify":
        vocab, drafts = _log(rng, 500, 131072), rng.choice([0, 1, 2, 3, 4, 5, 8])
        batch = min(_log(rng, 1, 256), (1 << 27) // (vocab * (drafts + 1)))
        return _verify("", batch, drafts, vocab, rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.7,
                       rng.random() < 0.4, rng.choice([0.0, 0.0, 1e-4]), rng.choice([0, 0, 1, 32]))
    if kind == "fork":
        group = rng.choice([2, 3, 4, 8])
        batch, max_pages = group * _log(rng, 1, 512 // group), _log(rng, 4, 1024)
        longest = max(1, max_pages * page - 1)
        return _fork("", batch, max_pages, page, group, 1 + longest // 30, longest, rng.random() < 0.5)
    row = kv * d * page * BYTES[cache]  # bytes of a page
    if kind == "resize":
        group = rng.choice([1, 1, 2, 4])
        batch = group * _log(rng, 1, 128 // group)
        pools = 2 * rng.choice([1, 2, 4, 8])
        new = rng.choice([0, 1, 1, 1, 6, 40]) if group == 1 else rng.choice([1, 1, 6, 40])
        most = (1 << 30) // (row * pools * batch // group)  # pages of a sequence
        longest = min(_log(rng, 5, 12000), max(1, most * page // 2))
        return _resize("", kv, d, cache, page, batch, -(-(longest + new) // page) + rng.choice([1, 3, 50]), group, new,
                       1 + longest // 30, longest, pools)
    pools = 2 * rng.choice([1, 2, 4])
    n_pages = min(_log(rng, 20, 100000), (1 << 30) // (row * pools))
    return _compact("", kv, d, cache, page, max(4, n_pages), round(rng.uniform(0.05, 0.98), 2), _log(rng, 1, 64), pools)


def _spread(n, shortest, longest):
    """n numbers spread between the two over their logarithm, the last one the longest."""
    lo, hi = math.log(shortest), math.log(longest)
    got = [int(round(math.exp(lo + (hi - lo) * ((i + 1) * 0.6180339887498949 % 1.0)))) for i in range(n - 1)]
    return got + [longest]


def _lengths(c):
    """An append: every sequence's tokens, the new ones counted in.  Page tables: of every group before the call."""
    return _spread(c["batch"] // c.get("group", 1), c["shortest"], c["longest"])


def _int32(x):
    return torch.as_tensor(x, dtype=torch.int32)


# ----------------------------------------------------------------- prepare

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    return {"rotate": _prepare_rotate, "append": _prepare_append, "verify": _prepare_verify, "fork": _prepare_fork,
            "resize": _prepare_resize, "compact": _prepare_compact}[kind](case, g)


def _randn(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV) * scale


def _angles(c, n, g, at=None):
    """Frequencies, the axis of each, and positions [axes, n] as a prompt of pictures has them: the first axis runs with
    the token (from `at`), the others over rows and columns of a picture of odd sizes."""
    half = c["rot"] // 2
    freqs = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    # sections of the frequencies, one an axis
    axis = (torch.arange(half, device=DEV) * c["axes"] // half).to(torch.int32)
    time = torch.arange(n, device=DEV) if at is None else at
    wide = 20 + torch.randint(0, 9, (), generator=g, device=DEV)
    rows = [time, time // wide % 31, time % wide, time // 7 % 5][:c["axes"]]
    pos = torch.stack(rows)
    if c["fractions"]:
        return freqs, axis, pos.to(torch.float32) + torch.rand(pos.shape, generator=g, device=DEV)
    return freqs, axis, pos.to(torch.int32)


def _prepare_rotate(c, g):
    shape = (c["heads"], c["tokens"], c["d"]) if c["heads_first"] else (c["tokens"], c["heads"], c["d"])
    x = _randn(g, *shape).to(TYPES[c["dtype"]])
    freqs, axis, pos = _angles(c, c["tokens"], g)
    return dict(case=c, X=x, freqs=freqs, axis=axis, positions=pos, Y=torch.empty_like(x))


def _pool_values(g, shape, cache):
    x = _randn(g, *shape)
    return x.clamp_(-448.0, 448.0).to(E4M3) if cache == "e4m3" else x.to(TYPES[cache])


def _prepare_append(c, g):
    H, Hkv, d, page, B = c["heads"], c["kv_heads"], c["d"], c["page"], c["batch"]
    dt, lens = TYPES[c["dtype"]], _lengths(c)
    held = [-(-n // page) for n in lens]
    n_pages, width = sum(held) + 3, max(held) + 2
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first = torch.tensor([0] + held).cumsum(0)
    col = torch.arange(width)
    slot = torch.where(col < torch.tensor(held)[:, None], first[:-1, None] + col, -1).to(DEV)
    table = torch.where(slot >= 0, order[slot.clamp(min=0)], torch.full_like(order[:1], -1)).contiguous()
    pools = [_pool_values(g, (n_pages, Hkv, page, d), c["cache"]) for _ in range(2)]
    scales = (None, None)
    if c["cache"] == "e4m3":
        scales = tuple(0.01 + 0.02 * torch.rand(Hkv, generator=g, device=DEV) for _ in range(2))
    new = [c["new"] or n for n in lens]
    n = sum(new)
    starts = torch.tensor([0] + new).cumsum(0)
    b = torch.repeat_interleave(torch.arange(B), torch.tensor(new))
    at = torch.arange(n) - starts[b + 1] + torch.tensor(lens)[b]
    freqs, axis, pos = _angles(c, n, g, at.to(DEV))
    s = dict(case=c, K_cache=pools[0], V_cache=pools[1], table=table, k_scale=scales[0], v_scale=scales[1],
             lengths=_int32(lens).to(DEV), starts=starts.to(torch.int32).to(DEV), freqs=freqs, axis=axis, positions=pos)
    if c["fused"]:
        qkv = _randn(g, n, H + 2 * Hkv, d).to(dt)
        s["Q"], s["K"], s["V"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        s["Q"], s["K"], s["V"] = (_randn(g, n, h, d).to(dt) for h in (H, Hkv, Hkv))
    s["Q_out"] = torch.zeros((n, H, d), dtype=dt, device=DEV)
    return s


def _prepare_verify(c, g):
    B, n, V, dt = c["batch"], c["drafts"], c["vocab"], TYPES[c["dtype"]]
    width = V + c["pad"]  # (rows of a padded vocabulary)
    P = torch.zeros((B, n + 1, width), dtype=dt, device=DEV)
    Qd = torch.zeros((B, max(n, 1), width), dtype=dt, device=DEV)
    drafts = torch.zeros((B, n), dtype=torch.int32, device=DEV)
    for b in range(0, B, 16):
        part = slice(b, min(B, b + 16))
        x = _randn(g, part.stop - b, n + 1, V, scale=3.0)
        for into, logits in ((P, x), (Qd, x[:, :n] + _randn(g, part.stop - b, n, V, scale=0.7))):
            if logits.shape[1]:
                p = logits.softmax(-1)
                p = torch.where(p >= c["kept"], p, torch.zeros_like(p))
                into[part, :logits.shape[1], :V] = (p / p.sum(-1, keepdim=True)).to(dt)
        if n:  # drawn from the drafts' own probabilities: the first of exponential arrivals
            wait = torch.empty((part.stop - b, n, V), device=DEV).exponential_(generator=g)
            drafts[part] = (Qd[part, :n, :V].float() / wait).argmax(-1).to(torch.int32)
    u = torch.rand((B, n + 1), generator=g, device=DEV)
    count = torch.randint(0, n + 1, (B,), generator=g, device=DEV).to(torch.int32) if c["ragged"] else None
    return dict(case=c, P=P[..., :V], Qd=Qd[:, :n, :V] if c["given"] and n else None, drafts=drafts, uniforms=u,
                n_drafts=count)


def _books(c, table, lengths, n_pages):
    """Page table, lengths and holders of every page as a program keeps them, and the same to set them back from: parts
    of one buffer each."""
    refs = torch.bincount(table[table >= 0].long(), minlength=n_pages)
    whole = torch.cat((table.flatten(), lengths, refs)).to(torch.int32).to(DEV)
    s = dict(case=c, book=whole.clone(), begin=whole)
    s["table"], s["lengths"], s["refs"] = (
        x.view(y) for x, y in zip(s["book"].split([table.numel(), lengths.numel(), n_pages]),
                                  (table.shape, lengths.shape, (n_pages,))))
    return s


def _paged_table(c, groups, held, g, spare):
    """A table in which the sequences of a group hold the same pages, held[group] of them, in any order."""
    first = torch.tensor([0] + held).cumsum(0)
    n_pages = int(first[-1]) + spare
    order = torch.randperm(n_pages, generator=g, device=DEV).cpu()
    col = torch.arange(c["max_pages"])
    slot = torch.where(col < torch.tensor(held)[:, None], first[:-1, None] + col, -1)
    rows = torch.where(slot >= 0, order[slot.clamp(min=0)], -1)
    return rows.repeat_interleave(c["batch"] // groups, 0), order[int(first[-1]):], n_pages


def _prepare_fork(c, g):
    B, G, page = c["batch"], c["group"], c["page"]
    lens = [min(n, c["max_pages"] * page) for n in _lengths(c)]
    held = [-(-n // page) for n in lens]
    b = torch.arange(B)
    if c["beams"]:  # every beam has a last page of its own, the rest is the group's
        table, free, n_pages = _paged_table(c, B // G, held, g, B + 8)
        last = torch.tensor(held).repeat_interleave(G) - 1
        table[b, last] = free[:B]
        lengths = torch.tensor(lens).repeat_interleave(G)
        parent = b // G * G + torch.randint(0, G, (B,), generator=g, device=DEV).cpu()
    else:  # the first of a group holds the prompt, the others are empty
        table, free, n_pages = _paged_table(c, B // G, held, g, 8)
        table[b % G != 0] = -1
        lengths = torch.where(b % G == 0, torch.tensor(lens).repeat_interleave(G), 0)
        parent = b // G * G
    s = _books(c, table, lengths, n_pages)
    s["parent"] = parent.to(torch.int32).to(DEV)
    return s


def _prepare_resize(c, g):
    B, G, page, new = c["batch"], c["group"], c["page"], c["new"]
    now = _lengths(c)
    old = [n if new else 0 for n in now]
    after = [n + new for n in now]
    # pages before the call; then every third sequence has one behind its new end (its drafts were not taken)
    held = [-(-n // page) for n in old]
    need = G * sum(-(-m // page) - n // page for n, m in zip(old, after))
    table, free, n_pages = _paged_table(c, B // G, held, g, need + B // 3 + 4)
    lengths = torch.tensor(after).repeat_interleave(G)
    end = (lengths + page - 1) // page
    left = torch.arange(B)[(torch.arange(B) % 3 == 0) & (end < c["max_pages"])]
    table[left, end[left]] = free[:len(left)]
    s = _books(c, table, lengths, n_pages)
    s["new"] = lengths.to(torch.int32).to(DEV) if new == 0 else new
    s["missing"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    s["pools"] = _pool_values(g, (c["pools"], n_pages, c["kv_heads"], page, c["d"]), c["cache"])
    return s


def _prepare_compact(c, g):
    n, B = c["n_pages"], c["batch"]
    used = _used(c)
    order = torch.randperm(n, generator=g, device=DEV).cpu()[:used]
    each = max(1, used // B)
    table = torch.full((B, each + 2), -1, dtype=torch.int64)
    rows = min(B, used // each)
    table[:rows, :each] = order[:rows * each].view(rows, each)
    table[:, each] = order[0]  # a page that every sequence holds
    s = _books(c, table, torch.zeros(B, dtype=torch.int64), n)
    held = torch.zeros(n, dtype=torch.int32, device=DEV)
    held[order[rows * each:].to(DEV)] = 1  # the others are held apart from any sequence, as a shared prefix is
    for book in (s["book"], s["begin"]):
        book[-n:] += held
    s["pools"] = _pool_values(g, (c["pools"], n, c["kv_heads"], c["page"], c["d"]), c["cache"])
    s["new_ids"] = torch.zeros(n, dtype=torch.int32, device=DEV)
    s["n_used"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _used(c):
    return max(1, int(round(c["used"] * c["n_pages"])))


# --------------------------------------------------------------------- run

def run(state):
    return {"rotate": _run_rotate, "append": _run_append, "verify": _run_verify, "fork": _run_fork,
            "resize": _run_resize, "compact": _run_compact}[state["case"]["kind"]](state)


def _rr():
    from paper_2609_07306_amd import routerelay
    return routerelay


def _turned(x, angle, inter, wide):
    """Rows [n, heads, d] rotated by [n, rot / 2] angles, in binary32 (wide: binary64)."""
    t = torch.float64 if wide else torch.float32
    cos, sin = angle.cos().to(t)[:, None], angle.sin().to(t)[:, None]
    r = 2 * angle.shape[1]
    x = x.to(t)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if inter else (x[..., :r // 2], x[..., r // 2:r])
    y, z = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((y, z), -1).flatten(-2) if inter else torch.cat((y, z), -1)
    return torch.cat((y, x[..., r:]), -1)


def _angle(s):
    return (s["positions"].double()[s["axis"].long()] * s["freqs"][:, None]).T


def _run_rotate(s):
    c = s["case"]
    if own:
        return {"Y": _rr().rotate(s["X"], s["positions"], s["freqs"], axis=s["axis"], tokens=1 if c["heads_first"] else 0,
                                  interleaved=c["inter"], inverse=c["inverse"], out=s["Y"])}
    angle = -_angle(s) if c["inverse"] else _angle(s)
    x = s["X"].transpose(0, 1) if c["heads_first"] else s["X"]
    y = _turned(x, angle, c["inter"], False)
    s["Y"].copy_(y.transpose(0, 1) if c["heads_first"] else y)
    return {"Y": s["Y"]}


def _run_append(s):
    c = s["case"]
    if own:
        _rr().cache_append(s["K"], s["V"], s["K_cache"], s["V_cache"], s["table"], s["lengths"],
                           seq_start=s["starts"] if c["new"] == 0 else None, freqs=s["freqs"], interleaved=c["inter"],
                           Q=s["Q"], Q_out=s["Q_out"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                           positions=s["positions"], axis=s["axis"])
        return {"K_cache": s["K_cache"], "V_cache": s["V_cache"], "Q": s["Q_out"]}
    i = torch.arange(s["K"].shape[0], device=DEV)
    b = torch.searchsorted(s["starts"][1:].long(), i, right=True)
    at = s["lengths"][b].long() - s["starts"][b + 1] + i
    phys = s["table"][b, at // c["page"]].long()
    off, angle, wide = at % c["page"], _angle(s), c["cache"] == "e4m3"

    def put(x, pool, scale):
        if wide:
            x = (x.double() / scale.double()[:, None]).clamp(-448.0, 448.0).float().to(E4M3)
            pool.view(torch.uint8)[phys, :, off] = x.view(torch.uint8)
        else:
            pool[phys, :, off] = x.to(pool.dtype)

    put(_turned(s["K"], angle, c["inter"], wide), s["K_cache"], s["k_scale"])
    put(s["V"], s["V_cache"], s["v_scale"])
    s["Q_out"].copy_(_turned(s["Q"], angle, c["inter"], False))
    return {"K_cache": s["K_cache"], "V_cache": s["V_cache"], "Q": s["Q_out"]}


def _run_verify(s):
    P, Qd, drafts, u, count = s["P"], s["Qd"], s["drafts"], s["uniforms"], s["n_drafts"]
    if own:
        rr = _rr()
        if "workspace" not in s:
            s["workspace"] = rr.verify_workspace(P)
        accepted, tokens = rr.verify_drafts(P, drafts, u, draft_probs=Qd, n_drafts=count, workspace=s["workspace"])
        return {"accepted": accepted, "tokens": tokens}
    B, n = drafts.shape
    V = P.shape[-1]
    b, i = torch.arange(B, device=DEV), torch.arange(n, device=DEV)
    x = drafts.long()
    p_x = P[b[:, None], i, x].double()
    q_x = Qd[b[:, None], i, x].double() if Qd is not None else torch.ones_like(p_x)
    took = u[:, :n].double() * q_x < p_x
    if count is not None:
        took &= i < count[:, None]
    a = took.long().cumprod(1).sum(1)  # accepted drafts
    most = count.long() if count is not None else torch.full_like(a, n)
    r = P[b, a].double()
    if n:
        at, rejected = a.clamp(max=n - 1), (a < most)[:, None]
        v = torch.arange(V, device=DEV)
        q_a = Qd[b, at].double() if Qd is not None else torch.where(v == x[b, at][:, None], math.inf, 0.0).double()
        rest = torch.where(rejected, (r - q_a).clamp(min=0), r)
        r = torch.where(rest.sum(1, keepdim=True) > 0, rest, r)  # (nothing is left: the target's own)
    total = r.cumsum(1)
    seen = (total > u[:, n:].double() * total[:, -1:]) & (r > 0)
    token = seen.to(torch.int8).argmax(1)
    j = torch.arange(n + 1, device=DEV)
    tokens = torch.where(j < a[:, None], torch.cat((drafts, drafts.new_zeros(B, 1)), 1).long(), -1)
    tokens = torch.where(j == a[:, None], token[:, None], tokens)
    return {"accepted": a.to(torch.int32), "tokens": tokens.to(torch.int32)}


def _count(refs, ids, there, by):
    """Adds `by` to refs[id] for every id that is there."""
    more = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=DEV)
    at = torch.where(there, ids.long(), refs.numel()).flatten()
    more.index_add_(0, at, by.expand(ids.shape).flatten())
    refs += more[:-1]


def _run_fork(s):
    s["book"].copy_(s["begin"])
    table, lengths, refs, parent = s["table"], s["lengths"], s["refs"], s["parent"]
    if own:
        _rr().cache_fork(table, lengths, refs, parent)
        return {"page_table": table, "lengths": lengths, "refs": refs}
    B = parent.numel()
    there = (parent >= 0) & (parent < B)
    source = parent.long().clamp(0, B - 1)
    rows = torch.where(there[:, None], table[source], -1)
    one = torch.ones((), dtype=torch.int32, device=DEV)
    _count(refs, table, table >= 0, -one)
    _count(refs, rows, rows >= 0, one)
    lengths.copy_(torch.where(there, lengths[source], 0))
    table.copy_(rows)
    return {"page_table": table, "lengths": lengths, "refs": refs}


def _pools(s):
    rr = _rr()
    if "handle" not in s:
        x = s["pools"].unbind(0)
        s["handle"] = rr.Pools(x[0::2], x[1::2])
        s["workspace"] = rr.pages_workspace(s["handle"])
    return rr, s["handle"], s["workspace"]


def _run_resize(s):
    c = s["case"]
    s["book"].copy_(s["begin"])
    table, lengths, refs, new = s["table"], s["lengths"], s["refs"], s["new"]
    if own:
        rr, pools, workspace = _pools(s)
        rr.cache_resize(pools, table, lengths, refs, new, missing=s["missing"], workspace=workspace)
        return {"page_table": table, "refs": refs, "missing": s["missing"], "pools": s["pools"]}
    page, (B, most), n_pages = c["page"], table.shape, refs.numel()
    one = torch.ones((), dtype=torch.int32, device=DEV)
    end = (lengths.long() + page - 1) // page
    col = torch.arange(most, device=DEV)
    past = (col >= end[:, None]) & (table >= 0)
    _count(refs, table, past, -one)
    table.masked_fill_(past, -1)
    # the entries of the newest tokens, in the order of sequences and pages
    begin = lengths.long() - new
    width = -(-(c["new"] or c["longest"]) // page) + 1
    at = begin[:, None] // page + torch.arange(width, device=DEV)
    live = at < end[:, None]
    at = at.clamp(max=most - 1)
    e = table.gather(1, at).long()
    held = live & (e >= 0)
    # how many earlier ones hold the same page: each of those that are copied leaves it to one less
    key = torch.where(held, e, n_pages).flatten()
    by, place = key.sort(stable=True)
    i = torch.arange(by.numel(), device=DEV)
    rank = torch.empty_like(i).scatter_(0, place, i - torch.searchsorted(by, by)).view_as(e)
    copied = held & (refs[e.clamp(min=0)] - rank > 1)
    need = copied | (live & (e < 0))
    order = need.flatten().cumsum(0) - 1
    free = refs == 0
    ids = torch.full((n_pages + 1,), -1, dtype=torch.int64, device=DEV)
    ids.scatter_(0, torch.where(free, free.cumsum(0) - 1, n_pages), torch.arange(n_pages, device=DEV))
    ids[n_pages] = -1
    to = torch.where(need.flatten(), ids[order.clamp(0, n_pages)], -1).view_as(e)
    got = to >= 0
    copied &= got
    _count(refs, to, got, one)
    _count(refs, e, copied, -one)
    b = torch.arange(B, device=DEV)[:, None].expand_as(at)
    table[b[got], at[got]] = to[got].to(torch.int32)
    s["missing"].copy_((need & ~got).sum(1))
    # what the copied pages hold before the new tokens
    kept = (begin[:, None] - at * page)[copied].clamp(0, page)
    src, dst = e[copied], to[copied]
    old = torch.arange(page, device=DEV) < kept[:, None]
    bits = s["pools"].view(torch.uint8) if c["cache"] == "e4m3" else s["pools"]
    bits[:, dst] = torch.where(old[None, :, None, :, None], bits[:, src], bits[:, dst])
    return {"page_table": table, "refs": refs, "missing": s["missing"], "pools": s["pools"]}


def _run_compact(s):
    c = s["case"]
    s["book"].copy_(s["begin"])
    table, refs = s["table"], s["refs"]
    if own:
        rr, pools, workspace = _pools(s)
        rr.cache_compact(pools, table, refs, new_ids=s["new_ids"], n_used=s["n_used"], workspace=workspace)
    else:
        n = refs.numel()
        id_ = torch.arange(n, device=DEV)
        used = refs > 0
        n_used = used.sum()
        low, high = ~used & (id_ < n_used), used & (id_ >= n_used)
        places = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
        places.scatter_(0, torch.where(low, low.cumsum(0) - 1, n), id_)
        to = torch.where(high, places[(high.cumsum(0) - 1).clamp(min=0)], torch.where(used, id_, -1))
        src = id_[high]
        bits = s["pools"].view(torch.uint8) if c["cache"] == "e4m3" else s["pools"]
        bits[:, to[src]] = bits[:, src]
        moved = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
        moved.scatter_(0, torch.where(used, to, n), refs)
        refs.copy_(torch.where(id_ < n_used, moved[:-1], 0))
        table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)].to(torch.int32), table))
        s["new_ids"].copy_(to)
        s["n_used"].copy_(n_used)
    return {"page_table": table, "refs": refs, "new_ids": s["new_ids"], "n_used": s["n_used"], "pools": s["pools"]}


# -------------------------------------------------------------------- work

def work(case):
    c = case
    kind = c["kind"]
    if kind in ("rotate", "append"):
        e, rot = BYTES[c["dtype"]], c["rot"]
        if kind == "rotate":
            rows = c["tokens"] * c["heads"]
            return {"bytes": 2 * rows * c["d"] * e + 4 * c["tokens"] * c["axes"] + 12 * (rot // 2), "flops": 3 * rows * rot}
        H, Hkv, d, ce = c["heads"], c["kv_heads"], c["d"], BYTES[c["cache"]]
        n = sum(c["new"] or x for x in _lengths(c))
        return {"bytes": n * (d * (2 * H * e + 2 * Hkv * (e + ce)) + 4 * c["axes"]) + 8 * c["batch"],
                "flops": 3 * n * (H + Hkv) * rot + (n * 2 * Hkv * d if ce == 1 else 0)}
    if kind == "verify":
        # the target's row, and the drafts' where one was rejected: about one in four of these drafts is
        n = c["drafts"] / (2.0 if c["ragged"] else 1.0)
        rows = 1 + (1 - 0.75 ** n if c["given"] else 0)
        return {"bytes": int(c["batch"] * (rows * c["vocab"] * BYTES[c["dtype"]] + 8 * c["drafts"] * 4)),
                "flops": int(c["batch"] * c["vocab"] * (rows + 1))}
    if kind == "fork":
        # a row that changes: what it held, what it will hold, and that written; every page's holders
        moved = c["batch"] * (c["group"] - 1) / c["group"]
        held = sum(-(-min(n, c["max_pages"] * c["page"]) // c["page"]) for n in _lengths(c))
        return {"bytes": int(moved * c["max_pages"] * 12 + 8 * held + 12 * c["batch"]), "flops": int(moved * c["max_pages"])}
    row = c["kv_heads"] * c["d"] * BYTES[c["cache"]] * c["pools"]  # bytes of a token in all pools
    if kind == "resize":
        B, G, page, new = c["batch"], c["group"], c["page"], c["new"]
        tokens = sum((G - 1) * (n % page) for n in _lengths(c)) if new else 0  # copied
        pages = sum(G * -(-(n + new) // page) + (-(-n // page) if new else 0) for n in _lengths(c)) + B
        return {"bytes": 2 * row * tokens + 4 * (B * c["max_pages"] + pages + 3 * B), "flops": pages}
    n, used = c["n_pages"], _used(c)
    moves = used * (n - used) / n  # the used ones of as many pages as are free, drawn from all
    return {"bytes": int(2 * row * c["page"] * moves + 16 * n + 8 * used), "flops": n}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """The same from the definitions: rotations as complex products in binary64, page tables entry by entry."""
    c, s = case, prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "verify": _exact_verify, "fork": _exact_fork,
            "resize": _exact_resize, "compact": _exact_compact}[c["kind"]](c, s)


def _complex_turn(x, s, inter, rot):
    """Rows [n, heads, d] in binary64, partners as real and imaginary parts."""
    half = rot // 2
    first = torch.arange(half, device=DEV) * (2 if inter else 1)
    second = first + (1 if inter else half)
    turn = torch.stack([s["positions"][int(t)].double() * f for t, f in zip(s["axis"], s["freqs"])], -1)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(turn), turn)[:, None]
    if s["case"].get("inverse"):
        z = torch.complex(x[..., first], x[..., second]) / torch.polar(torch.ones_like(turn), turn)[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rotate(c, s):
    x = s["X"].double()
    y = _complex_turn(x.transpose(0, 1) if c["heads_first"] else x, s, c["inter"], c["rot"])
    return {"Y": y.transpose(0, 1) if c["heads_first"] else y}


def _exact_append(c, s):
    K, V = (x.to(torch.float64) for x in (s["K_cache"], s["V_cache"]))
    k, q = (_complex_turn(s[x].double(), s, c["inter"], c["rot"]) for x in "KQ")
    v, page, at = s["V"].double(), c["page"], 0
    if c["cache"] == "e4m3":
        k = (k / s["k_scale"].double()[:, None]).clamp(-448, 448)
        v = (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
    for b, length in enumerate(_lengths(c)):
        n = c["new"] or length
        place = torch.arange(length - n, length, device=DEV)
        phys = s["table"][b].long()[place // page]
        K[phys, :, place % page], V[phys, :, place % page] = k[at:at + n], v[at:at + n]
        at += n
    return {"K_cache": K, "V_cache": V, "Q": q}


def _exact_verify(c, s):
    import numpy as np
    B, n = s["drafts"].shape
    drafts, u = s["drafts"].cpu().numpy(), s["uniforms"].cpu().numpy().astype(np.float64)
    count = s["n_drafts"].cpu().numpy() if s["n_drafts"] is not None else np.full(B, n)
    accepted, tokens = np.zeros(B, np.int32), np.full((B, n + 1), -1, np.int32)
    for b in range(B):
        p = s["P"][b].double().cpu().numpy()
        q = s["Qd"][b].double().cpu().numpy() if s["Qd"] is not None else None
        rest = p[count[b]]
        for i in range(count[b]):
            x = drafts[b, i]
            if u[b, i] * (q[i, x] if q is not None else 1.0) < p[i, x]:
                tokens[b, i] = x
                accepted[b] += 1
                continue
            rest = p[i] - q[i] if q is not None else p[i] * (np.arange(p.shape[1]) != x)
            rest = np.maximum(rest, 0.0)
            rest = rest if rest.any() else p[i]
            break
        v = np.nonzero(rest)[0]
        below = rest[v].cumsum()
        tokens[b, accepted[b]] = v[min(int((below <= u[b, n] * below[-1]).sum()), len(v) - 1)]
    return {"accepted": torch.from_numpy(accepted), "tokens": torch.from_numpy(tokens)}


def _holders(refs, before, after):
    """Holders of every page where rows of the table change: those held apart stay."""
    refs = list(refs)
    for rows, by in ((before, -1), (after, 1)):
        for row in rows:
            for e in row:
                if e >= 0:
                    refs[e] += by
    return refs


def _exact_fork(c, s):
    table, lengths, refs, parent = (s[k].cpu().tolist() for k in ("table", "lengths", "refs", "parent"))
    rows = [list(table[p]) if 0 <= p < len(table) else [-1] * len(table[0]) for p in parent]
    return {"page_table": _int32(rows), "lengths": _int32([lengths[p] if 0 <= p < len(table) else 0 for p in parent]),
            "refs": _int32(_holders(refs, table, rows))}


def _exact_resize(c, s):
    table, lengths, refs = (s[k].cpu().tolist() for k in ("table", "lengths", "refs"))
    new = s["new"].cpu().tolist() if torch.is_tensor(s["new"]) else [s["new"]] * len(lengths)
    pools, page, missing = s["pools"].double(), c["page"], [0] * len(lengths)
    for row, n in zip(table, lengths):
        for i in range(-(-n // page), len(row)):
            if row[i] >= 0:
                refs[row[i]] -= 1
                row[i] = -1
    free = [p for p, r in enumerate(refs) if r == 0][::-1]
    for b, (row, n) in enumerate(zip(table, lengths)):
        begin = max(0, n - new[b])
        for i in range(begin // page, -(-n // page) if n > begin else 0):
            if row[i] >= 0 and refs[row[i]] <= 1:
                continue
            if not free:
                missing[b] += 1
                continue
            p, e, kept = free.pop(), row[i], max(0, begin - i * page)
            if e >= 0:
                refs[e] -= 1
                pools[:, p, :, :kept] = pools[:, e, :, :kept]
            row[i], refs[p] = p, 1
    return {"page_table": _int32(table), "refs": _int32(refs), "missing": _int32(missing), "pools": pools}


def _exact_compact(c, s):
    table, refs = (s[k].cpu().tolist() for k in ("table", "refs"))
    n_used = sum(r > 0 for r in refs)
    free = [p for p in range(n_used) if refs[p] == 0][::-1]
    pools, to = s["pools"].double(), []
    for p, r in enumerate(refs):
        to.append(-1 if r == 0 else p if p < n_used else free.pop())
    src = [p for p, t in enumerate(to) if t >= 0 and t != p]
    for p in src:
        pools[:, to[p]] = pools[:, p]
        refs[to[p]], refs[p] = refs[p], 0
    return {"page_table": _int32([[to[e] if e >= 0 else e for e in row] for row in table]), "refs": _int32(refs),
            "new_ids": _int32(to), "n_used": _int32([n_used]), "pools": pools}
