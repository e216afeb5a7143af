"""Definitions of the calls around the attention call in a step of generation - rotary positions, pages shared between
sequences, adjusted logits - in 64 bits, one element or one row after the other.  Nothing is shared with the GPU path."""
from __future__ import annotations

import math

import torch

BLOCK = 16
FULL, BAD_ROW, BAD_LENGTH, BAD_PAGE = 1, 2, 4, 8


def rope_axes(axis_pairs, cyclic: bool):
    """Axis of every pair."""
    n, A = sum(axis_pairs), len(axis_pairs)
    if cyclic:
        return [c % A if c // A < axis_pairs[c % A] else 0 for c in range(n)]
    return [a for a in range(A) for _ in range(axis_pairs[a])]


def rope(x, positions, inv_freq, axis_pairs=None, neighbours=False, cyclic=False, inverse=False, magnitude=1.0):
    """x [T, H, d] turned by positions [A, T] (or [T]) times inv_freq [r/2], in 64 bits, not rounded."""
    x = x.double().clone()
    pos = positions.reshape(-1, x.shape[0])
    n = inv_freq.numel()
    axes = rope_axes([n] if axis_pairs is None else list(axis_pairs), cyclic)
    for c in range(n):
        a = pos[axes[c]].double() * inv_freq[c].double()
        cos, sin = (torch.cos(a) * magnitude)[:, None], (torch.sin(a) * magnitude)[:, None]
        if inverse:
            sin = -sin
        i, j = (2 * c, 2 * c + 1) if neighbours else (c, c + n)
        lo, hi = x[:, :, i].clone(), x[:, :, j].clone()
        x[:, :, i], x[:, :, j] = lo * cos - hi * sin, hi * cos + lo * sin
    return x


def _length(n, mb, status):
    most = mb * BLOCK
    if n < 0 or n > most:
        status[0] |= BAD_LENGTH
    return min(max(n, 0), most)


def _pages(n):
    return -(-n // BLOCK)


def fork(src_rows, table, lens, refs, src_lens=None, num_blocks=None):
    """(rows as lists of pages, lengths, counts, status) of hook_pages_fork; lists in, lists out."""
    status = [0]
    mb, nb, S = len(table[0]) if table else 0, len(refs), len(table)
    refs = list(refs)
    rows, new = [], []
    L = [_length(n, mb, status) for n in lens]
    for j, p in enumerate(src_rows):
        if p < -1 or p >= S:
            status[0] |= BAD_ROW
        n = L[p] if 0 <= p < S else 0
        if src_lens is not None:
            n = min(n, max(src_lens[j], 0))
        new.append(n)
        rows.append(list(table[p][:_pages(n)]) if n else [])
    for i in range(S):
        for page in table[i][:_pages(L[i])]:
            if 0 <= page < nb:
                refs[page] -= 1
            else:
                status[0] |= BAD_PAGE
    for r in rows:
        for page in r:
            if 0 <= page < nb:
                refs[page] += 1
    return rows, new, refs, status[0]


def append(cu, table, lens, refs):
    """(rows, lengths, counts, copies [(from page, to page, token rows)], status) of hook_pages_append."""
    status = [0]
    mb, nb, S = len(table[0]) if table else 0, len(refs), len(table)
    L = [_length(n, mb, status) for n in lens]
    rows = [list(table[i][:_pages(L[i])]) for i in range(S)]
    before = [list(r) for r in rows], list(L), list(refs)
    refs, free = list(refs), [p for p in range(nb) if refs[p] <= 0]
    holders, copies, new = list(refs), [], list(L)
    fits = True
    for i in range(S):
        n = cu[i + 1] - cu[i]
        if n < 0:
            status[0] |= BAD_LENGTH
            n = 0
        if n == 0:
            continue
        if L[i] % BLOCK:
            page = rows[i][-1]
            if not 0 <= page < nb:
                status[0] |= BAD_PAGE
            else:
                if holders[page] > 1:
                    holders[page] -= 1
                    to = free.pop(0) if free else None
                    fits = fits and to is not None
                    copies.append((page, to, L[i] % BLOCK))
                    rows[i][-1] = to
                else:
                    holders[page] -= 1      # later rows with this page see one holder less, as if this one had left
        if L[i] + n > mb * BLOCK:
            fits = False
            continue
        for _ in range(_pages(L[i] + n) - _pages(L[i])):
            to = free.pop(0) if free else None
            fits = fits and to is not None
            rows[i].append(to)
        new[i] = L[i] + n
    if not fits:
        status[0] |= FULL
        return before[0], before[1], before[2], [], status[0]
    for page, to, _ in copies:
        refs[page] -= 1
    old = {i: _pages(L[i]) for i in range(S)}
    for i in range(S):
        for e in range(old[i], len(rows[i])):
            refs[rows[i][e]] = 1
    for _, to, _ in copies:
        refs[to] = 1
    return rows, new, refs, copies, status[0]


def compact(table, lens, refs):
    """(rows, counts, map, live, moves [(from, to)], status) of hook_pages_compact."""
    status = [0]
    mb, nb = len(table[0]) if table else 0, len(refs)
    live = sum(n > 0 for n in refs)
    moves = list(zip([p for p in range(live, nb) if refs[p] > 0], [p for p in range(live) if refs[p] <= 0]))
    page_map = [p if refs[p] > 0 else -1 for p in range(nb)]
    out = list(refs)
    for a, b in moves:
        page_map[a], out[b], out[a] = b, refs[a], 0
    rows = []
    for i, r in enumerate(table):
        row = []
        for page in r[:_pages(_length(lens[i], mb, status))]:
            if not 0 <= page < nb or page_map[page] < 0:
                status[0] |= BAD_PAGE
                row.append(page)
            else:
                row.append(page_map[page])
        rows.append(row)
    return rows, out, page_map, live, moves, status[0]


def steer_logits(logits, history=None, prompt_lens=None, repetition=None, frequency=None, presence=None, bias=None, mask=None,
                 mask_rows=None):
    """logits [R, V] adjusted, in 64 bits.  history: R lists of tokens; bias: R lists of (token, value); mask: [M, words] int32 words."""
    y = logits.double().clone()
    R, V = y.shape
    for i in range(R):
        rep = 1.0 if repetition is None else float(repetition[i])
        freq = 0.0 if frequency is None else float(frequency[i])
        pres = 0.0 if presence is None else float(presence[i])
        count, seen = {}, set()
        for j, t in enumerate(history[i] if history is not None else []):
            if 0 <= t < V:
                seen.add(t)
                if j >= (0 if prompt_lens is None else int(prompt_lens[i])):
                    count[t] = count.get(t, 0) + 1
        for t in seen:
            x = float(y[i, t])
            x = x / rep if x > 0 else x * rep
            if t in count:
                x = x - count[t] * freq - pres
            y[i, t] = x
        for t, v in dict(bias[i] if bias is not None else []).items():
            if 0 <= t < V:
                y[i, t] += float(v)
        if mask is not None:
            m = i if mask_rows is None else int(mask_rows[i])
            if 0 <= m < mask.shape[0]:
                words = mask[m].tolist()
                for t in range(V):
                    if not (words[t // 32] >> (t % 32)) & 1:
                        y[i, t] = -math.inf
    return y
