"""A serving step around the paged cache in plain numpy, 64 bits: rotary positions, the token map, page tables, beam search.

Written from the formulas and rules in thk.h, one step at a time on lists; nothing here is shared with the library.
"""
import math

import numpy as np

D = 128
TILE = 64


def speeds(rot, scaling, base, factor=1.0, trained=0, low=0.0, high=0.0):
    """Radians a position of every pair, and the scheme's own gain."""
    half, gain = rot // 2, 1.0
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    w = np.array([base ** (-2.0 * i / rot) for i in range(half)])
    if scaling == "linear":
        w = w / factor
    if scaling == "ramp":
        at = [rot * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (high, low)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        g = np.clip((np.arange(half) - lo) / max(hi - lo, 0.001), 0, 1)
        w, gain = w / factor * g + w * (1 - g), 0.1 * math.log(max(factor, 1.0)) + 1
    if scaling == "bands":
        g = np.clip((trained * w / (2 * math.pi) - low) / (high - low), 0, 1)
        w = w / factor * (1 - g) + w * g
    return w, gain


def rope(x, pos, w, gain, rot, pairs):
    """x [n, heads, D] float64 at positions pos [n]."""
    y = x.copy()
    a = np.asarray(pos, np.float64)[:, None] * w
    c, s = gain * np.cos(a)[:, None], gain * np.sin(a)[:, None]
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def place(buffer, x, seq, row):
    """Rows x [n, heads, D] into buffer [B, heads, rows, D], where the map says."""
    B, _, rows, _ = buffer.shape
    for t in range(len(x)):
        if 0 <= seq[t] < B and 0 <= row[t] < rows:
            buffer[seq[t], :, row[t]] = x[t]


def token_map(n_new, pos0, row0, cap, q_rows, n_tokens):
    records, starts = [], []
    for b, (n, p, r) in enumerate(zip(n_new, pos0, row0)):
        starts.append(min(len(records), n_tokens))
        for i in range(max(n, 0)):
            q = i - (n - q_rows)
            records.append([b, p + i, r + i if 0 <= r + i < cap else -1, q if q >= 0 else -1])
    starts.append(min(len(records), n_tokens))
    records = records[:n_tokens]
    return np.array(records + [[-1, 0, -1, -1]] * (n_tokens - len(records)), np.int64).reshape(-1, 4), starts


def reserve(rows, now, held, table, refs, page_rows):
    """(held, table, refs, room, moves) afterwards, as lists; now may be None."""
    held, table, refs = list(held), [list(t) for t in table], list(refs)
    B, most = len(rows), len(table[0])
    valid = lambda p: 0 <= p < len(refs)  # noqa: E731
    need = [min(-(-max(r, 0) // page_rows), most) for r in rows]
    for b in range(B):
        held[b] = min(max(held[b], 0), most)
        while held[b] > need[b]:
            held[b] -= 1
            if valid(table[b][held[b]]):
                refs[table[b][held[b]]] -= 1
            table[b][held[b]] = -1
    users = {}
    if now is not None:
        for b in range(B):
            e = now[b] // page_rows
            if 0 < now[b] < rows[b] and now[b] % page_rows and e < held[b] and valid(table[b][e]):
                users.setdefault(table[b][e], []).append(b)
    moving = set()
    for p, u in users.items():      # where all users of a page grow, the one with the most rows in it stays, the first of several
        keeper = max(u, key=lambda b: (now[b] % page_rows, -b)) if len(u) >= refs[p] else None
        moving |= {b for b in u if b != keeper}
    free = [p for p, r in enumerate(refs) if r <= 0]
    room, moves = [], []
    for b in range(B):
        move, stuck = [-1, -1, 0, 0], False
        if b in moving:
            stuck = not free
            if free:
                e, to = now[b] // page_rows, free.pop(0)
                move = [table[b][e], to, -(-(now[b] % page_rows) // TILE), 0]
                refs[table[b][e]] -= 1
                refs[to], table[b][e] = 1, to
        while held[b] < need[b] and free:
            to = free.pop(0)
            refs[to], table[b][held[b]] = 1, to
            held[b] += 1
        room.append(now[b] if stuck else held[b] * page_rows)
        moves.append(move)
    return held, table, refs, room, moves


def beam_select(x, scores, done, K, eos):
    """x [B, W, V], scores [B, W] float64, done [B, W]: (parent, token, score, done), a row of K each."""
    B, W, V = x.shape
    out = []
    for b in range(B):
        found = []
        for w in range(W):
            if not np.isfinite(scores[b, w]):
                continue
            if done[b, w]:
                found.append((-scores[b, w], w, 0, eos))
                continue
            row = x[b, w]
            top = row.max()
            if not np.isfinite(top):   # nothing but -inf, or +inf, or NaN
                continue
            with np.errstate(divide="ignore"):
                s = scores[b, w] + ((row - top) - math.log(np.exp(row - top).sum()))
            best = np.argsort(-row, kind="stable")[:K]   # by the logit, then by the token
            found += [(-s[v], w, i, int(v)) for i, v in enumerate(best) if np.isfinite(s[v])]
        found = sorted(found)[:K]
        rows = [(w, v, -s, int(v == eos or done[b, w] != 0)) for s, w, _, v in found]
        out.append(rows + [(-1, -1, -math.inf, 0)] * (K - len(rows)))
    return [np.array([[r[i] for r in rows] for rows in out]) for i in range(4)]


def reorder(parent, W, tails, s_tail, s_pages, held, table, refs, page_rows):
    """tails: arrays [L, B, N_kv, cap, D] (may be empty); the other five lists, or None.  Afterwards, likewise."""
    old = [t.copy() for t in tails]
    copy = lambda v: None if v is None else [list(t) if isinstance(t, (list, tuple)) else t for t in v]  # noqa: E731
    tails, was = [t.copy() for t in tails], (s_tail, s_pages, held, table)
    s_tail, s_pages, held, table, refs = copy(s_tail), copy(s_pages), copy(held), copy(table), copy(refs)
    for p, row in enumerate(parent):
        for j in range(W):
            if not 0 <= row[j] < W or row[j] == j:
                continue
            me, par = p * W + j, p * W + row[j]
            for t, o in zip(tails, old):
                n = min(max(was[0][par], 0), t.shape[3])
                t[:, me, :, :n] = o[:, par, :, :n]
            if s_tail is not None:
                s_tail[me] = was[0][par]
            if s_pages is not None:
                s_pages[me] = was[1][par]
            if held is not None:
                for q in was[3][me][:was[2][me]]:
                    if 0 <= q < len(refs):
                        refs[q] -= 1
                held[me] = min(was[2][par], -(-max(was[1][par], 0) // page_rows))
                for e in range(max(was[2][me], held[me])):
                    table[me][e] = was[3][par][e] if e < held[me] else -1
                for q in table[me][:held[me]]:
                    if 0 <= q < len(refs):
                        refs[q] += 1
    return tails, s_tail, s_pages, held, table, refs
