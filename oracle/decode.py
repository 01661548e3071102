"""Oracle of the decoding operators, in numpy and 64 bits, from their definitions: log probabilities with entropy and top
alternatives, their gradient, attention over a paged cache, and the forking and compaction of its pages.

Everything is written row by row and page by page; nothing is shared with the CUDA side.
"""
from __future__ import annotations

import numpy as np

NEG = -np.inf


# --- log probabilities ----------------------------------------------------------------------------------------------

def logprobs_row(x, token=None, k: int = 0, temperature: float = 1.0) -> dict:
    """One row of logits (any float type, taken exactly)."""
    x = np.asarray(x, dtype=np.float64)
    z = x / temperature
    bad = bool(np.isnan(z).any() or (z == np.inf).any())
    if bad:
        lse, logp, entropy = np.nan, np.full(z.shape, np.nan), np.nan
    elif (z == NEG).all():
        lse, logp, entropy = NEG, np.full(z.shape, NEG), 0.0
    else:
        m = z.max()
        s = np.exp(z - m).sum()
        lse = m + np.log(s)
        logp = (z - m) - np.log(s)
        p = np.exp(logp)
        entropy = -float(np.sum(p[p > 0] * logp[p > 0]))
    out = {"lse": lse, "entropy": entropy, "logp": logp}
    if token is not None:
        out["logprob"] = 0.0 if token < 0 else (np.nan if token >= x.size else logp[token])
    if k:
        # value descending in the order of the bit patterns (-0 below +0), index ascending; NaN is never among them
        order = sorted((i for i in range(x.size) if not np.isnan(x[i])), key=lambda i: (-x[i], np.signbit(x[i]) if x[i] == 0 else False, i))[:k]
        out["top_tokens"] = np.array(order + [-1] * (k - len(order)), dtype=np.int64)
        out["top_logprobs"] = np.array([logp[i] if i >= 0 else np.nan for i in out["top_tokens"]])
    return out


def logprobs_loss(x, temperature, token, g_lp, g_h, g_lse, top, g_top) -> float:
    """The scalar whose gradient the backward call takes, of one row."""
    r = logprobs_row(x, temperature=temperature)
    total = g_h * r["entropy"] + g_lse * r["lse"]
    if token is not None and 0 <= token < len(x):
        total += g_lp * r["logp"][token]
    for i, g in zip(top, g_top):
        if 0 <= i < len(x):
            total += g * r["logp"][i]
    return float(total)


def logprobs_gradient_row(x, temperature, token, g_lp, g_h, g_lse, top, g_top):
    """(gradient, magnitude): the magnitude bounds what roundings of the probabilities can do to each entry."""
    r = logprobs_row(x, temperature=temperature)
    x = np.asarray(x, dtype=np.float64)
    if r["lse"] == NEG:
        return np.zeros(x.size), np.zeros(x.size)
    given = token is not None and 0 <= token < x.size
    g_top = np.array([g if 0 <= i < x.size else 0.0 for i, g in zip(top, g_top)])     # a place without a token has no gradient
    g = (g_lp if given else 0.0) + float(np.sum(g_top)) - g_lse
    a = r["logp"]
    p = np.exp(a)
    safe = np.where(p > 0, a, 0.0)
    grad = -p * (g + g_h * (safe + r["entropy"]))
    # one rounding of p is at most 2^-22 (exponential) + 2^-23 |log2 p| (its argument), of the factor 2^-22 of its parts
    rel = 2.0 ** -21 + 2.0 ** -22 * np.abs(safe) * 1.4427
    size = p * (abs(g) + np.sum(np.abs(g_top)) + abs(g_lse) + abs(g_lp) + abs(g_h) * (np.abs(safe) + abs(r["entropy"]))) * rel
    if given:
        grad[token] += g_lp
        size[token] += abs(g_lp) * 2.0 ** -23
    for i, gt in zip(top, g_top):
        if 0 <= i < x.size:
            grad[i] += gt
            size[i] += abs(gt) * 2.0 ** -22
    return grad / temperature, size / temperature


# --- attention of one token over a paged cache ----------------------------------------------------------------------

def paged_attention(q, k_pages, v_pages, tables, lengths, scale):
    """q (seqs, heads, dim), pages (pages, kv_heads, page_size, dim): (out, lse) in 64 bits."""
    q, k_pages, v_pages = (np.asarray(a, dtype=np.float64) for a in (q, k_pages, v_pages))
    seqs, heads, dim = q.shape
    pages, kv_heads, page, _ = k_pages.shape
    group = heads // kv_heads
    out, lse = np.zeros(q.shape), np.full((seqs, heads), NEG)
    for s in range(seqs):
        n = min(max(int(lengths[s]), 0), len(tables[s]) * page)
        at = [(int(tables[s][t // page]), t % page) for t in range(n)]
        at = [(p, o) for p, o in at if 0 <= p < pages]              # tokens of pages that do not exist take no part
        if not at:
            continue
        ids, off = np.array(at).T
        for h in range(heads):
            k, v = k_pages[ids, h // group, off], v_pages[ids, h // group, off]
            z = k @ q[s, h] * scale
            m = z.max()
            e = np.exp(z - m)
            out[s, h] = e @ v / e.sum()
            lse[s, h] = m + np.log(e.sum())
    return out, lse


# --- pages ----------------------------------------------------------------------------------------------------------

def fork(pool, tables, lengths, refs, parents, grow, past_room=False):
    """pool (layers, 2, pages, kv_heads, page_size, dim) is changed in place; returns (tables, lengths, refs, missing).  With
    `past_room` lengths count what was wanted, not what the table holds."""
    n_old, width = tables.shape
    pages, page = pool.shape[2], pool.shape[4]
    held = [min(max(int(n), 0), width * page) for n in lengths]
    valid = lambda p: 0 <= p < pages  # noqa: E731
    free = [p for p in range(pages) if refs[p] <= 0]
    new_refs = refs.astype(np.int64).copy()
    new_tables, new_lengths = np.full((len(parents), width), -1, dtype=np.int32), np.zeros(len(parents), dtype=np.int32)
    missing, kept, before = 0, set(), pool.copy()
    for s in range(n_old):
        for c in range(-(-held[s] // page)):
            if valid(tables[s][c]):
                new_refs[tables[s][c]] -= 1
    for i, parent in enumerate(int(p) for p in parents):
        known = 0 <= parent < n_old
        old = held[parent] if known else 0
        wanted = old + grow
        length = min(wanted, width * page)
        new_lengths[i] = wanted if past_room else length
        have, fill = -(-old // page), old % page
        copy = known and fill > 0 and parent in kept
        if known:
            kept.add(parent)
        for c in range(-(-length // page)):
            if c < have and not (copy and c == have - 1):
                new_tables[i, c] = tables[parent][c] if valid(tables[parent][c]) else -1
                if valid(tables[parent][c]):
                    new_refs[tables[parent][c]] += 1
                continue
            if not free:
                missing += 1
                continue
            p = free.pop(0)
            new_tables[i, c] = p
            new_refs[p] += 1
            if c == have - 1 and valid(tables[parent][c]):
                pool[:, :, p, :, :fill] = before[:, :, tables[parent][c], :, :fill]
        missing += -(-wanted // page) - -(-length // page)
    return new_tables, new_lengths, new_refs.astype(np.int32), missing


def compact(pool, tables, refs):
    """pool is changed in place; returns (tables, refs, page_map, live)."""
    pages = len(refs)
    live = int((refs > 0).sum())
    page_map = np.where(refs > 0, np.arange(pages), -1).astype(np.int32)
    movers = [p for p in range(live, pages) if refs[p] > 0]
    holes = [p for p in range(live) if refs[p] <= 0]
    new_refs = refs.copy()
    for src, dst in zip(movers, holes):
        pool[:, :, dst] = pool[:, :, src]
        page_map[src] = dst
        new_refs[dst], new_refs[src] = refs[src], 0
    new_refs[live:] = 0
    new_refs = np.where(new_refs > 0, new_refs, 0).astype(np.int32)
    new = np.array([[page_map[t] if 0 <= t < pages else -1 for t in row] for row in tables], dtype=np.int32).reshape(tables.shape)
    return new, new_refs, page_map, live
