"""CPU oracle of the operators on pages of a cache that requests share or pick from: tables and counts, bounds of keys, selection of pages.

TEST INFRASTRUCTURE ONLY (same rule as the package).  Plain numpy, one function per operator, entry by entry; where a definition names a rounding to 32 bits it stands in its
place.  It imports nothing from the GPU package.
"""
from __future__ import annotations

import numpy as np

PAGE = 64


def _entries(positions, width):
    return min(-(-max(int(positions), 0) // PAGE), width)


def _free(references):
    return [p for p in range(len(references)) if references[p] <= 0]


def take(table, references, positions):
    """(table, references, missing): every entry of a row's first positions that names no page gets the lowest free one."""
    table, references, missing = table.copy(), references.copy(), 0
    free = _free(references)
    for b in range(table.shape[0]):
        for e in range(_entries(positions[b], table.shape[1])):
            if not 0 <= table[b, e] < len(references):
                if free:
                    table[b, e] = free.pop(0)
                    references[table[b, e]] = 1
                else:
                    table[b, e] = -1
                    missing += 1
    return table, references, missing


def fork(source, references, parents, positions, width, pages):
    """(table [len(parents), width], references, pages, missing) of continuations of rows of `source`."""
    references, pages, missing = references.copy(), pages.copy(), 0
    free = _free(references)
    table = np.full((len(parents), width), -1, dtype=np.int32)
    for b, parent in enumerate(parents):
        if not 0 <= parent < source.shape[0]:
            continue
        n = min(max(int(positions[b]), 0), source.shape[1] * PAGE)
        for e in range(min(n // PAGE, width)):
            if 0 <= source[parent, e] < len(references):
                table[b, e] = source[parent, e]
                references[table[b, e]] += 1
        e = n // PAGE
        if n % PAGE and e < width and 0 <= source[parent, e] < len(references):
            if free:
                table[b, e] = free.pop(0)
                references[table[b, e]] = 1
                pages[table[b, e]] = pages[source[parent, e]]
            else:
                missing += 1
    return table, references, pages, missing


def free(table, references, keep=None):
    table, references = table.copy(), references.copy()
    for b in range(table.shape[0]):
        for e in range(_entries(keep[b], table.shape[1]) if keep is not None else 0, table.shape[1]):
            if 0 <= table[b, e] < len(references):
                references[table[b, e]] -= 1
            table[b, e] = -1
    return table, references


def compact(table, references, pages):
    """(table, references, pages, used)"""
    table, references, pages = table.copy(), references.copy(), pages.copy()
    used = int((references > 0).sum())
    far = [p for p in range(used, len(references)) if references[p] > 0]
    near = [p for p in range(used) if references[p] <= 0]
    to = {}
    for a, b in zip(far, near):
        pages[b] = pages[a]
        references[b], references[a] = references[a], 0
        to[a] = b
    for b in range(table.shape[0]):
        for e in range(table.shape[1]):
            table[b, e] = to.get(int(table[b, e]), table[b, e])
    return table, references, pages, used


def bounds(K):
    """(codes int8 [2, d], step) of the keys K [positions, d] of a page (fp64 values of the cache)."""
    k = np.asarray(K).astype(np.float32)
    hi, lo = k.max(0), k.min(0)
    most = np.float32(max(np.abs(hi).max(), np.abs(lo).max()))
    if most == 0:
        return np.zeros((2, k.shape[1]), dtype=np.int8), np.float32(0)
    f = np.float32(127) / most
    codes = np.stack([np.minimum(np.ceil(hi * f), 127), np.maximum(np.floor(lo * f), -127)])
    return codes.astype(np.int8), most / np.float32(127)


def scores(q_f16, codes, steps, there):
    """Scores [pages] of one token and KV head: q [g, d], codes [pages, 2, d], steps [pages], there [pages]: entries that have a page."""
    q = np.asarray(q_f16, dtype=np.float16).astype(np.float32)
    best = np.full(len(steps), -np.inf, dtype=np.float32)
    for row in q:
        most = np.abs(row).max()
        f = np.float32(127) / most if most > 0 else np.float32(0)
        c = np.clip(np.rint(row * f), -127, 127).astype(np.int64)
        n = np.maximum(c, 0) @ codes[:, 0].astype(np.int64).T + np.minimum(c, 0) @ codes[:, 1].astype(np.int64).T
        best = np.maximum(best, n.astype(np.float32) * (most / np.float32(127)))
    return np.where(there, best * steps.astype(np.float32), -np.inf).astype(np.float32)


def select(score, sees, first, last, count):
    """Numbers of pages [count], ascending, -1 behind them."""
    if sees <= count:
        pick = list(range(sees))
    else:
        middle = sorted(range(first, sees - last), key=lambda p: (-score[p], p))[:count - first - last]
        pick = sorted(list(range(first)) + middle + list(range(sees - last, sees)))
    return np.array(pick + [-1] * (count - len(pick)), dtype=np.int32)
