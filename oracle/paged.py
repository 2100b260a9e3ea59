"""float64 oracle of the paged caches and of the verification of drafted tokens: numpy, one sequence, head and position after the other.

A paged cache is a pair of float arrays [num_pages, h_kv, page_size, width] and a table [b, max_pages] of page numbers; position p of sequence i
is row p % page_size of page table[i, p // page_size], and does not exist where that is no page of the pool.
"""
from __future__ import annotations

import numpy as np


def where(table, i, pos, num_pages, page_size):
    """(page, row in it) of a position, or None."""
    page = int(table[i, pos // page_size])
    return (page, pos % page_size) if 0 <= page < num_pages else None


def append(K, V, table, k_new, v_new, lens, counts=None, rounded=lambda x: x):
    """Writes rows k_new [b,n,h_kv,k] / v_new behind the lens[i] there are, in place.  Returns the new lengths."""
    num_pages, _, page_size, _ = K.shape
    b, n = k_new.shape[:2]
    out = np.array(lens)
    for i in range(b):
        count = n if counts is None else min(max(int(counts[i]), 0), n)
        if lens[i] < 0 or lens[i] + count > table.shape[1] * page_size:
            continue
        out[i] = lens[i] + count
        for r in range(count):
            at = where(table, i, int(lens[i]) + r, num_pages, page_size)
            if at is not None:
                K[at[0], :, at[1]] = rounded(k_new[i, r])
                V[at[0], :, at[1]] = rounded(v_new[i, r])
    return out


def attend(q, K, V, table, lens, scale=1.0, scores=None):
    """q [b,n,h,k] -> o [b,n,h,v], the weights' sums [b,h_kv,positions] on top of scores (None: 0; the newest n positions from 0 on; NaN where
    nothing is written), and a bound on sum_p w |V| per row for tolerances."""
    num_pages, h_kv, page_size, v = V.shape
    b, n, h, _ = q.shape
    group, positions = h // h_kv, table.shape[1] * page_size
    o, size = np.zeros((b, n, h, v)), np.zeros((b, n, h, v))
    total = np.full((b, h_kv, positions), np.nan)
    for i in range(b):
        length = min(max(int(lens[i]), 0), positions)
        at = [where(table, i, p, num_pages, page_size) for p in range(length)]
        for e in range(h_kv):
            total[i, e, :length] = 0
            if scores is not None:
                total[i, e, :max(0, length - n)] = scores[i, e, :max(0, length - n)]
            for j in range(n):
                seen = [p for p in range(length - (n - 1 - j)) if at[p] is not None]
                if not seen:
                    continue
                Ks = np.stack([K[at[p][0], e, at[p][1]] for p in seen])
                Vs = np.stack([V[at[p][0], e, at[p][1]] for p in seen])
                for x in range(e * group, (e + 1) * group):
                    with np.errstate(all="ignore"):
                        z = scale * (Ks @ q[i, j, x])
                        w = np.exp(z - z.max())
                        w = w / w.sum()
                        o[i, j, x], size[i, j, x] = w @ Vs, w @ np.abs(Vs)
                        total[i, e, seen] += w
    return o, total, size


def evict(K, V, table, lens, scores, table_out, budget, recent):
    """Copies what stays to table_out's pages, in place.  Returns (lens_out, kept [b,h_kv,budget], scores_out [b,h_kv,positions out], NaN where nothing is
    written)."""
    num_pages, h_kv, page_size, _ = K.shape
    b, positions = table.shape[0], table.shape[1] * page_size
    kept, lens_out = np.full((b, h_kv, budget), -1, dtype=np.int64), np.zeros(b, dtype=np.int64)
    scores_out = np.full((b, h_kv, table_out.shape[1] * page_size), np.nan)
    K0, V0 = K.copy(), V.copy()
    for i in range(b):
        length = min(max(int(lens[i]), 0), positions)
        at = [where(table, i, p, num_pages, page_size) for p in range(length)]
        old = [p for p in range(max(0, length - recent)) if at[p] is not None]
        newest = [p for p in range(max(0, length - recent), length) if at[p] is not None]
        for e in range(h_kv):
            value = lambda p: -np.inf if np.isnan(scores[i, e, p]) else scores[i, e, p]  # noqa: E731
            best = sorted(old, key=lambda p: (-value(p), p))[:budget - len(newest)]
            stays = sorted(best + newest)
            lens_out[i] = len(stays)
            for slot, p in enumerate(stays):
                kept[i, e, slot], scores_out[i, e, slot] = p, scores[i, e, p]
                to = where(table_out, i, slot, num_pages, page_size)
                if to is not None:
                    K[to[0], e, to[1]] = K0[at[p][0], e, at[p][1]]
                    V[to[0], e, to[1]] = V0[at[p][0], e, at[p][1]]
    return lens_out, kept, scores_out


def probabilities(logits, temperature):
    """softmax(logits / temperature) of one row; zeros where the row is -inf throughout."""
    x = np.where(np.isnan(logits), -np.inf, np.minimum(logits.astype(np.float64), np.finfo(np.float32).max))
    if x.max() == -np.inf:
        return np.zeros_like(x)
    w = np.exp((x - x.max()) / float(np.float32(temperature)))
    return w / w.sum()


def largest(row, temperature):
    """The lowest index of a row's largest logit, 0 if there is none.  With temperature 0 NaN is no logit at all; else NaN counts as -inf, and +inf as the largest number."""
    if temperature == 0:
        there = np.nonzero(~np.isnan(row))[0]
        return int(there[np.argmax(row[there])]) if len(there) else 0
    return int(np.argmax(np.where(np.isnan(row), -np.inf, np.minimum(row, np.finfo(np.float32).max))))


def verify(logits, drafts, u, draft_logits=None, counts=None, temperature=1.0):
    """(tokens [b,n+1], accepted [b])."""
    b, n, vocab = logits.shape[0], logits.shape[1] - 1, logits.shape[2]
    tokens, accepted = np.full((b, n + 1), -1, dtype=np.int64), np.zeros(b, dtype=np.int64)
    for i in range(b):
        count = n if counts is None else min(max(int(counts[i]), 0), n)
        rest = None
        for j in range(count + 1):
            best = largest(logits[i, j], temperature)
            if temperature > 0:
                rest = probabilities(logits[i, j], temperature)
            if j == count:
                break
            t = int(drafts[i, j])
            if temperature == 0:
                if t != best:
                    break
            else:
                p, q = rest, np.zeros(vocab)
                if draft_logits is not None:
                    q = probabilities(draft_logits[i, j], temperature)
                elif 0 <= t < vocab:
                    q[t] = 1
                if not (0 <= t < vocab and float(u[i, j]) * q[t] < p[t]):
                    rest = np.maximum(p - q, 0)
                    break
            tokens[i, j] = t
            accepted[i] += 1
        token = best
        if temperature > 0 and rest.sum() > 0:
            run = np.cumsum(rest)
            above = np.nonzero(run > float(u[i, n]) * run[-1])[0]
            token = int(above[0]) if len(above) else int(np.nonzero(rest > 0)[0][-1])
        tokens[i, accepted[i]] = token
    return tokens, accepted
