"""Oracle of the calls around the paged cache -- TEST INFRASTRUCTURE.

Plain Python and numpy in binary64, entry by entry, for the test suite only:
rotation by positions of several axes, page tables that are forked, resized and
compacted, and the verification of drafted tokens, with the readings of the C
ABI's header.
"""
from __future__ import annotations

import math

import numpy as np


def rotate(x, positions, freqs, axis=None, interleaved=False, inverse=False):
    """x [n_tokens, heads, d], positions [n_axes, n_tokens]."""
    out = x.astype(np.float64).copy()
    half = len(freqs)
    for j, f in enumerate(freqs):
        t = 0 if axis is None else int(axis[j])
        if not 0 <= t < len(positions):
            continue
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        angle = np.asarray(positions[t], np.float64) * float(f) * (-1.0 if inverse else 1.0)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        out[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return out


def fork(table, lengths, refs, parent):
    """All in and out as lists of ints; new ones are returned."""
    B, width = len(table), len(table[0])
    refs = list(refs)
    rows = [list(table[p]) if 0 <= p < B else [-1] * width for p in parent]
    for old, by in ((table, -1), (rows, 1)):
        for b, row in enumerate(old):
            if parent[b] == b:
                continue
            for e in row:
                if 0 <= e < len(refs):
                    refs[e] += by
    return rows, [lengths[p] if 0 <= p < B else 0 for p in parent], refs


def resize(table, lengths, refs, new, page):
    """-> (table, refs, missing, copies): copies (from page, to page, places)."""
    table, refs = [list(row) for row in table], list(refs)
    width, n_pages = len(table[0]), len(refs)

    def held(e):
        return 0 <= e < n_pages

    ends = [min(max(n, 0), width * page) for n in lengths]
    for row, n in zip(table, ends):
        for c in range(-(-n // page), width):
            if held(row[c]):
                refs[row[c]] -= 1
                row[c] = -1
    free = [p for p, r in enumerate(refs) if r == 0][::-1]
    missing, copies = [0] * len(table), []
    for b, (row, end) in enumerate(zip(table, ends)):
        begin = max(0, lengths[b] - max(0, new[b]))
        if begin >= end:
            continue
        for c in range(begin // page, -(-end // page)):
            e = row[c]
            if held(e) and refs[e] <= 1:
                continue
            if not free:
                missing[b] += 1
                continue
            p = free.pop()
            if held(e):
                refs[e] -= 1
                if begin > c * page:
                    copies.append((e, p, min(page, begin - c * page)))
            row[c], refs[p] = p, 1
    return table, refs, missing, copies


def compact(table, refs):
    """-> (table, refs, new_ids, n_used)."""
    n = sum(r != 0 for r in refs)
    free = [p for p in range(n) if refs[p] == 0][::-1]
    new_ids = [-1 if r == 0 else p if p < n else free.pop() for p, r in enumerate(refs)]
    out = [0] * len(refs)
    for p, t in enumerate(new_ids):
        if t >= 0:
            out[t] = refs[p]
    return [[new_ids[e] if 0 <= e < len(refs) else e for e in row] for row in table], out, new_ids, n


def verify(P, Q, drafts, uniforms, n_drafts=None):
    """P [B, n + 1, V], Q [B, n, V] or None -> (accepted, tokens, near): near is
    how close any comparison that decided came to its border, relative to the
    sum of what it compared."""
    B, n = drafts.shape
    V = P.shape[2]
    accepted, tokens = np.zeros(B, np.int64), np.full((B, n + 1), -1, np.int64)
    near = math.inf
    for b in range(B):
        count = n if n_drafts is None else min(max(int(n_drafts[b]), 0), n)
        rest, target = P[b, count].astype(np.float64), P[b, count].astype(np.float64)
        for i in range(count):
            x = int(drafts[b, i])
            q = None if Q is None else Q[b, i].astype(np.float64)
            if 0 <= x < V and float(uniforms[b, i]) * (1.0 if q is None else q[x]) < float(P[b, i, x]):
                tokens[b, i] = x
                accepted[b] += 1
                continue
            target = P[b, i].astype(np.float64)
            with np.errstate(invalid="ignore"):
                rest = target.copy() if q is None else target - q
            if q is None and 0 <= x < V:
                rest[x] = 0.0
            break

        def clean(r):
            return np.where((r > 0) & (r < np.inf), r, 0.0)

        rest = clean(rest)
        if not rest.any():
            rest = clean(target)
        v = np.nonzero(rest)[0]
        if len(v) == 0:
            continue
        below = np.array([math.fsum(rest[v[:i + 1]]) for i in range(len(v))]) if len(v) < 64 else np.cumsum(rest[v])
        border = float(uniforms[b, n]) * below[-1]
        over = np.nonzero(below > border)[0]
        tokens[b, accepted[b]] = v[over[0] if len(over) else -1]
        if math.isfinite(border):
            near = min(near, np.abs(below - border).min() / below[-1])
    return accepted, tokens, near
