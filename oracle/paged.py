"""Oracle of the paged cache -- TEST INFRASTRUCTURE.

Plain numpy in binary64 over the sequences' tokens in order, for the test
suite only: where a new token's rows lie and what they hold (the rotation of
keys and queries by position), and attention of the newest tokens over the
cached ones, with the readings of the C ABI's header: places outside the pools
hold no token, lengths count the new tokens and are taken between 0 and what
the page table can hold, a query that sees no token gets a zero output.
"""
from __future__ import annotations

import math

import numpy as np


def held(length: int, max_pages: int, page: int) -> int:
    return min(max(int(length), 0), max_pages * page)


def rotate(x: np.ndarray, pos: int, freqs, interleaved: bool) -> np.ndarray:
    """x [heads, d] rotated by position pos: partners j and j + rot / 2, or
    2 j and 2 j + 1, turn by pos * freqs[j]."""
    out = x.astype(np.float64).copy()
    half = len(freqs)
    for j, f in enumerate(freqs):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = math.cos(pos * float(f)), math.sin(pos * float(f))
        out[:, a] = x[:, a] * c - x[:, b] * s
        out[:, b] = x[:, b] * c + x[:, a] * s
    return out


def places(seq_start, lengths, table, n_pages: int, page: int, n_tokens: int):
    """Per new token: (position or -1, page or -1, place)."""
    B, width = table.shape
    out = [(-1, -1, 0)] * n_tokens
    for b in range(B):
        for i in range(int(seq_start[b]), min(int(seq_start[b + 1]), n_tokens)):
            p = int(lengths[b]) - (int(seq_start[b + 1]) - i)
            if 0 <= p < width * page:
                phys = int(table[b, p // page])
                out[i] = (p, phys if 0 <= phys < n_pages else -1, p % page)
    return out


def tokens_of(pool: np.ndarray, pages, n: int):
    """The first n tokens of a sequence with these pages: rows [n, H_kv, d] and
    whether each one's page is there."""
    n_pages, Hkv, page, d = pool.shape
    rows, there = np.zeros((n, Hkv, d)), np.zeros(n, bool)
    for c in range(-(-n // page)):
        lo, hi = c * page, min((c + 1) * page, n)
        phys = int(pages[c])
        if 0 <= phys < n_pages:
            rows[lo:hi] = pool[phys, :, :hi - lo].transpose(1, 0, 2)
            there[lo:hi] = True
    return rows, there


def attention(Q, K, V, table, lengths, routes=None, n_sink=0, n_recent=0, prefix_pages=None, n_prefix=0, scale=None,
              k_scale=None, v_scale=None):
    """Q [B, n_q, H, d], pools K and V [n_pages, H_kv, page, d] -> (O, lse, W,
    S): outputs, logarithms of the sums of exponentials, and for tolerances
    the outputs over |V| and the largest scaled sum of |q_i k_i| of a row."""
    B, nq, H, d = Q.shape
    n_pages, Hkv, page, _ = K.shape
    g = H // Hkv
    scale = 1 / math.sqrt(d) if not scale else scale
    O, W = np.zeros(Q.shape), np.zeros(Q.shape)
    lse, S = np.full((B, nq, H), -np.inf), np.zeros((B, nq, H))
    for b in range(B):
        n = held(lengths[b], table.shape[1], page)
        if n == 0:
            continue
        k, there = tokens_of(K, table[b], n)
        v, _ = tokens_of(V, table[b], n)
        if n_prefix:
            m = min(n, n_prefix)
            k0, t0 = tokens_of(K, prefix_pages, m)
            v0, _ = tokens_of(V, prefix_pages, m)
            k[:m], v[:m], there[:m] = k0, v0, t0
        if k_scale is not None:
            k, v = k * np.asarray(k_scale, np.float64)[:, None], v * np.asarray(v_scale, np.float64)[:, None]
        u = np.arange(n)
        for t in range(nq):
            p = n - nq + t
            for h in range(H):
                seen = there & (u <= p)
                if routes is not None or n_sink or n_recent:
                    ids = set(range(n_sink)) | {p // page - i for i in range(n_recent)}
                    if routes is not None:
                        ids |= set(int(x) for x in routes[(b * H + h) * nq + t])
                    seen &= np.isin(u // page, list(ids))
                if not seen.any():
                    continue
                kk, vv = k[seen, h // g], v[seen, h // g]
                q = Q[b, t, h].astype(np.float64)
                s = kk @ q * scale
                top = s.max()
                w = np.exp(s - top)
                lse[b, t, h] = top + math.log(w.sum())
                w /= w.sum()
                O[b, t, h], W[b, t, h] = w @ vv, w @ np.abs(vv)
                S[b, t, h] = (np.abs(kk) @ np.abs(q)).max() * scale
    return O, lse, W, S
