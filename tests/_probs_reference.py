"""Verification from probabilities in float64, written from its definition (one sequence, one entry at a time where it matters)."""
import numpy as np


def usable(x):
    """Entries that are probabilities: finite and not below zero (-0 is one)."""
    return np.isfinite(x) & (x >= 0)


def verify(target, draft, tokens, u_accept, u_draw, lengths=None, place=None, least=0):
    """target [B, k+1, V] float64; draft [B, k, V] or None (certain drafters).  Returns accepted, token, d_tv [B, k] (NaN behind the
    sequence's length) and the number of near edges: draws whose threshold lies within 1e-11 of the total of an edge."""
    B, kp1, V = target.shape
    k = kp1 - 1
    accepted, token, near = np.zeros(B, np.int64), np.zeros(B, np.int64), 0
    d_tv = np.full((B, k), np.nan)
    for b in range(B):
        n = k if lengths is None else int(min(max(lengths[b], least), k))
        at = b if place is None else int(place[b])
        if draft is not None and n > 0 and not 0 <= at < B:
            accepted[b], token[b], d_tv[b, :n] = 0, -1, 1.0
            continue

        def q_row(j):
            if draft is not None:
                return draft[at, j]
            q = np.zeros(V)
            if 0 <= tokens[b, j] < V:
                q[tokens[b, j]] = 1.0
            return q

        for j in range(n):
            p, q = target[b, j], q_row(j)
            inside = draft is not None or 0 <= tokens[b, j] < V
            fine = usable(p).all() and usable(q).all() and inside
            d_tv[b, j] = 0.5 * np.abs(p - q).sum() if fine else 1.0
        stop = 0
        while stop < n:
            x = tokens[b, stop]
            if not 0 <= x < V:
                break
            p, q = target[b, stop, x], q_row(stop)[x]
            if not (usable(p) and usable(q) and float(u_accept[b, stop]) * q < p):
                break
            stop += 1
        accepted[b] = stop
        p = target[b, stop]
        q = q_row(stop) if stop < n else np.zeros(V)
        if not (usable(p).all() and usable(q).all()):
            token[b] = -1
            continue
        w = np.maximum(p - q, 0.0)
        if not w.any():
            w = p
        if not w.any():
            token[b] = -1
            continue
        reach = np.cumsum(w)
        threshold = float(u_draw[b]) * reach[-1]
        mass = np.flatnonzero(w > 0)
        hit = mass[reach[mass] > threshold]
        token[b] = hit[0] if len(hit) else mass[-1]
        exact = np.all(w * 2.0 ** 40 == np.floor(w * 2.0 ** 40)) and reach[-1] <= 4096     # sums without rounding
        near += not exact and bool(np.min(np.abs(reach - threshold)) < 1e-11 * reach[-1])
    return accepted, token, d_tv, near
