"""Oracle of the operators that take prompts and drafts into a decoding loop, in numpy and 64 bits (angles in extended
precision), from their definitions: rotary positions, appending with them, attention of a chunk of new tokens over a paged
cache, and what a sampler lays over logits.

Everything is written token by token and row by row; nothing is shared with the CUDA side.
"""
from __future__ import annotations

import numpy as np

NEG = -np.inf


# --- rotary positions -----------------------------------------------------------------------------------------------

def rotary(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False):
    """x (tokens, heads, dim), positions (tokens,): (turned, magnitude * (|x_1| + |x_2|) of each element's pair, |angle|)."""
    x = np.asarray(x, dtype=np.float64)
    f = np.asarray(frequencies, dtype=np.longdouble)
    half = f.size
    a = np.asarray(positions, dtype=np.int64).astype(np.longdouble)[:, None] * f
    cos, sin = (np.asarray(g(a), dtype=np.float64)[:, None] * magnitude for g in (np.cos, np.sin))
    if inverse:
        sin = -sin
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    out, size, angle = x.copy(), np.zeros(x.shape), np.zeros(x.shape)
    out[..., first] = x[..., first] * cos - x[..., second] * sin
    out[..., second] = x[..., second] * cos + x[..., first] * sin
    for s in (first, second):
        size[..., s] = (np.abs(x[..., first]) + np.abs(x[..., second])) * abs(magnitude)
        angle[..., s] = np.abs(np.asarray(a, dtype=np.float64))[:, None]
    return out, size, angle


def sequences(seqs, rows, starts=None):
    """The rows of every sequence, as ranges."""
    if starts is None:
        return [range(s * (rows // seqs), (s + 1) * (rows // seqs)) for s in range(seqs)]
    return [range(int(starts[s]), int(starts[s + 1])) for s in range(seqs)]


def places(lengths, rows, starts=None):
    """(sequence, place) of every row; sequence -1: none holds it."""
    seq, place = np.full(rows, -1), np.zeros(rows, dtype=np.int64)
    for s, held in enumerate(sequences(len(lengths), rows, starts)):
        for i, r in enumerate(held):
            seq[r], place[r] = s, int(lengths[s]) - len(held) + i
    return seq, place


def append(pages, values, tables, lengths, starts=None):
    """Writes rows (rows, kv_heads, dim) to their places in `pages` (pages, kv_heads, page_size, dim), in place."""
    page, width = pages.shape[2], tables.shape[1]
    seq, place = places(lengths, len(values), starts)
    for r in range(len(values)):
        if seq[r] < 0 or not 0 <= place[r] < width * page:
            continue
        p = int(tables[seq[r]][place[r] // page])
        if 0 <= p < len(pages):
            pages[p, :, place[r] % page] = values[r]


# --- attention of a chunk over a paged cache ------------------------------------------------------------------------

def paged_attention_chunk(q, k_pages, v_pages, tables, lengths, scale, starts=None):
    """q (rows, heads, dim), pages (pages, kv_heads, page_size, dim): (out, lse, sum p |v|, largest scale * sum |q k|)."""
    q, k_pages, v_pages = (np.asarray(a, dtype=np.float64) for a in (q, k_pages, v_pages))
    rows, heads, dim = q.shape
    pages, kv_heads, page, _ = k_pages.shape
    group = heads // kv_heads
    out, lse, size, reach = np.zeros(q.shape), np.full((rows, heads), NEG), np.zeros(q.shape), np.zeros((rows, heads))
    for s, held in enumerate(sequences(len(lengths), rows, starts)):
        if not len(held):
            continue
        room = len(tables[s]) * page
        n = min(max(int(lengths[s]), 0), room)
        at = np.array([t for t in range(n) if 0 <= int(tables[s][t // page]) < pages], dtype=np.int64)
        first = int(lengths[s]) - len(held)
        if not len(at):
            continue
        ids = np.asarray(tables[s])[at // page].astype(np.int64)
        late = at[None, :] > (first + np.arange(len(held)))[:, None]
        for h in range(heads):
            k, v = k_pages[ids, h // group, at % page], v_pages[ids, h // group, at % page]
            rows_q = q[held.start:held.stop, h]
            with np.errstate(invalid="ignore"):
                z = np.where(late, NEG, rows_q @ k.T * scale)
                some = ~late.all(1)
                m = np.where(some, z.max(1, initial=NEG), 0.0)
                e = np.where(late, 0.0, np.exp(z - m[:, None]))
                total = np.where(some, e.sum(1), 1.0)
                w = e / total[:, None]
                o = np.where(some[:, None], _weighted(w, v, late), 0.0)
                out[held.start:held.stop, h] = o
                size[held.start:held.stop, h] = _weighted(w, np.abs(v), late)
                lse[held.start:held.stop, h] = np.where(some, m + np.log(total), NEG)
                reach[held.start:held.stop, h] = np.where(late, 0.0, np.abs(rows_q) @ np.abs(k).T).max(1, initial=0.0) * scale
    return out, lse, size, reach


def _weighted(w, v, late):
    """w @ v where a token that a row does not see takes no part, whatever its values are."""
    if np.isfinite(v).all():
        return w @ v
    return np.stack([w[i][~late[i]] @ v[~late[i]] if (~late[i]).any() else np.zeros(v.shape[1]) for i in range(len(w))])


# --- penalties, biases and masks ------------------------------------------------------------------------------------

def adjust_row(x, tokens=(), prompt=0, repetition=1.0, frequency=0.0, presence=0.0, bias_tokens=(), bias_values=(), mask=None):
    """One row of logits: (adjusted, sum of the magnitudes that its rounding errors go by, whether anything applied)."""
    y = np.asarray(x, dtype=np.float64).copy()
    size, changed = np.zeros(y.shape), np.zeros(y.shape, dtype=bool)
    seen, count = set(), {}
    for i, t in enumerate(int(t) for t in tokens):
        if 0 <= t < y.size:
            seen.add(t)
            if i >= prompt:
                count[t] = count.get(t, 0) + 1
    for t in seen:
        y[t] = y[t] / repetition if y[t] > 0 else y[t] * repetition
        size[t] += abs(y[t])
        changed[t] = True
    for t, c in count.items():
        y[t] -= frequency * c + presence
        size[t] += 2 * (abs(frequency) * c + abs(presence))
    total = {}
    for t, b in zip(bias_tokens, bias_values):
        if 0 <= int(t) < y.size:
            total.setdefault(int(t), []).append(float(b))
    for t, b in total.items():
        y[t] += sum(b)
        size[t] += abs(y[t]) + len(b) * sum(abs(e) for e in b)
        changed[t] = True
    if mask is not None:
        v = np.arange(y.size)
        off = (np.asarray(mask).astype(np.int64)[v // 32] >> (v % 32) & 1) == 0
        y[off] = NEG
        changed |= off
    return y, size, changed
