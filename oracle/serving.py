"""float64 oracle of paged caches of 8 bits, of who holds which page, and of adjusted logits: numpy, one sequence, block and token after the other.

A cache of 8 bits is a float64 array of the values that its bits have, [num_pages, h_kv, page_size, width], and scales [num_pages, h_kv, page_size / block].
"""
from __future__ import annotations

import math

import numpy as np

from oracle import paged

LARGEST = {"e4m3": 448.0, "int8": 127.0}


def rounded(x, kind):
    """The numbers of 8 bits next to x, of two the even one: e4m3 has three bits behind the first, steps of 2^-9 below 2^-6; int8 the whole numbers to 127."""
    x = np.asarray(x, dtype=np.float64)
    top = LARGEST[kind]
    if kind == "int8":
        return np.where(np.isnan(x), 0.0, np.rint(np.clip(x, -top, top)))
    size = np.minimum(np.abs(x), top)
    exponent = np.frexp(np.where(np.isnan(size), 1.0, size))[1] - 1                    # size in [2^e, 2^(e+1))
    step = 2.0 ** (np.maximum(exponent, -6) - 3.0)
    return np.copysign(np.rint(size / step) * step, x)


def scale_of(largest, kind):
    """The smallest power of two, 2^-126 at least, under which `largest` is no more than the type's largest number."""
    e = -126
    while largest > LARGEST[kind] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def whole(K, scales):
    """The values that a cache of 8 bits holds."""
    return K * np.repeat(scales, K.shape[2] // scales.shape[2], axis=2)[..., None]


def append(K, K_scales, V, V_scales, table, k_new, v_new, lens, counts=None, kind="e4m3"):
    """In place.  Returns the new lengths."""
    num_pages, h_kv, page_size, _ = K.shape
    block = page_size // K_scales.shape[2]
    b, n = k_new.shape[:2]
    out = np.array(lens)
    for i in range(b):
        count = n if counts is None else min(max(int(counts[i]), 0), n)
        if lens[i] < 0 or lens[i] + count > table.shape[1] * page_size:
            continue
        begin, end = int(lens[i]), int(lens[i]) + count
        out[i] = end
        for first in range(begin // block * block, end, block):
            at = paged.where(table, i, first, num_pages, page_size)
            if at is None:
                continue
            page, row = at
            lo, hi = max(first, begin), min(first + block, end)
            for pool, scales, new in ((K, K_scales, k_new), (V, V_scales, v_new)):
                for e in range(h_kv):
                    x = new[i, lo - begin:hi - begin, e].astype(np.float64)
                    size = np.abs(x)[np.isfinite(x)]
                    s = scale_of(size.max() if len(size) else 0.0, kind)
                    had = scales[page, e, row // block]
                    if lo > first:
                        if had > s:
                            s = had
                        elif s != had:
                            old = pool[page, e, row:row + lo - first]
                            pool[page, e, row:row + lo - first] = rounded(old * (had / s), kind)
                    scales[page, e, row // block] = s
                    pool[page, e, row + lo - first:row + hi - first] = rounded(x / s, kind)
    return out


# ------------------------------------------------------------------------------------------ pages
def pages_of(length, page_size):
    return -(-length // page_size)


def fork(table, lens, parents, refs, page_size):
    """(table_out, lens_out); refs in place."""
    out, lens_out = np.full((len(parents), table.shape[1]), -1), np.zeros(len(parents), dtype=np.int64)
    for j, parent in enumerate(parents):
        if not 0 <= parent < len(table):
            continue
        lens_out[j] = min(max(int(lens[parent]), 0), table.shape[1] * page_size)
        for x in range(pages_of(int(lens_out[j]), page_size)):
            if 0 <= table[parent, x] < len(refs):
                out[j, x] = table[parent, x]
                refs[out[j, x]] += 1
    return out, lens_out


def free(table, lens, refs, page_size):
    """In place."""
    for i in range(len(table)):
        for x in range(pages_of(min(max(int(lens[i]), 0), table.shape[1] * page_size), page_size), table.shape[1]):
            if 0 <= table[i, x] < len(refs):
                refs[table[i, x]] -= 1
            table[i, x] = -1


def reserve(table, lens, refs, page_size, n, counts=None):
    """(granted, moves); table and refs in place."""
    b, num_pages = len(table), len(refs)
    wants = {}
    for i in range(b):
        count = n if counts is None else min(max(int(counts[i]), 0), n)
        if count and lens[i] >= 0 and lens[i] + count <= table.shape[1] * page_size:
            wants[i] = (count, range(int(lens[i]) // page_size, pages_of(int(lens[i]) + count, page_size)))
    before = refs.copy()
    is_page = lambda entry: 0 <= entry < num_pages  # noqa: E731
    writers = {}                                                                       # of a shared page that has been begun: who writes to it
    for i, (count, pages) in wants.items():
        entry = table[i, pages[0]]
        if lens[i] % page_size and is_page(entry) and before[entry] > 1:
            writers.setdefault(int(entry), []).append(i)
    free_pages = [page for page in range(num_pages) if before[page] <= 0]
    granted, moves, running = np.zeros(b, dtype=np.int64), np.full((b, 2), -1), 0
    for i, (count, pages) in wants.items():
        takes, keeps = [], False
        for x in pages:
            entry = int(table[i, x])
            if lens[i] % page_size and x == pages[0]:
                if is_page(entry) and before[entry] > 1:
                    keeps = len(writers[entry]) == before[entry] and writers[entry][-1] == i
                    if not keeps:
                        takes.append(x)
            elif not is_page(entry) or before[entry] > 1:
                takes.append(x)
        running += len(takes)
        if running > len(free_pages) and (takes or keeps):
            continue
        granted[i] = count
        for x, page in zip(takes, free_pages[running - len(takes):running]):
            entry = int(table[i, x])
            if is_page(entry):
                refs[entry] -= 1
                if lens[i] % page_size and x == pages[0]:
                    moves[i] = entry, page
            table[i, x] = page
            refs[page] = 1
    return granted, moves


def compact(table, refs):
    """(table_out, refs_out, moves [max(1, num_pages // 2), 2], used)."""
    num_pages = len(refs)
    used = int((refs > 0).sum())
    tails, holes = [x for x in range(used, num_pages) if refs[x] > 0], [x for x in range(used) if refs[x] <= 0]
    moves = np.full((max(1, num_pages // 2), 2), -1)
    place, refs_out = {x: x for x in range(used) if refs[x] > 0}, np.zeros_like(refs)
    for x, (tail, hole) in enumerate(zip(tails, holes)):
        moves[x] = tail, hole
        place[tail] = hole
    for page, to in place.items():
        refs_out[to] = refs[page]
    return np.array([[place.get(int(x), -1) for x in row] for row in table]).reshape(table.shape), refs_out, moves, used


def copy(pool, moves):
    """In place."""
    old = pool.copy()
    for source, to in moves:
        if 0 <= source < len(pool) and 0 <= to < len(pool):
            pool[to] = old[source]


# ------------------------------------------------------------------------------------------ logits
def adjust(logits, history, lens, drafts=None, prompts=None, repetition=None, frequency=None, presence=None, bias_tokens=None, biases=None, allowed=None):
    """logits [b,n+1,vocab]; allowed [b,n+1,vocab] of truth values."""
    out = logits.astype(np.float64)
    b, rows, vocab = out.shape
    for i in range(b):
        length = min(max(int(lens[i]), 0), history.shape[1])
        for j in range(rows):
            count, seen = {}, set()
            for at, t in enumerate([*history[i, :length].tolist(), *(drafts[i, :j].tolist() if drafts is not None else [])]):
                if 0 <= t < vocab:
                    seen.add(t)
                    if at >= length or prompts is None or at >= prompts[i]:
                        count[t] = count.get(t, 0) + 1
            with np.errstate(all="ignore"):
                for t in seen:
                    if repetition is not None:
                        out[i, j, t] = out[i, j, t] / repetition[i] if out[i, j, t] > 0 else out[i, j, t] * float(repetition[i])
                    if t in count:
                        out[i, j, t] -= (0 if frequency is None else float(frequency[i]) * count[t]) + (0 if presence is None else float(presence[i]))
                if biases is not None:
                    for t, y in {t: y for t, y in zip(bias_tokens[i].tolist(), biases[i].tolist()) if 0 <= t < vocab}.items():
                        out[i, j, t] += y
            if allowed is not None:
                out[i, j][~allowed[i, j]] = -math.inf
    return out
