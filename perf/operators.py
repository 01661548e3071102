"""The operators of one decoding step, as they are timed and compared: log probabilities (and their gradient), attention
of one new token over a paged cache, and the forking and compaction of that cache's pages.

`run` computes a case either in its plain form (elementary torch operations in 32 bits) or, where `own` is true, through
the library's public functions.  `exact` computes it from the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------------------------------------------------
# cases

def _logprobs(name, rows, vocab, dtype, k, temperature=1.0, masked=False, entropy=True):
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "k": k,
            "temperature": temperature, "masked": masked, "entropy": entropy}


def _gradient(name, rows, vocab, dtype, k, temperature=1.0, masked=False):
    return {"name": name, "op": "gradient", "rows": rows, "vocab": vocab, "dtype": dtype, "k": k,
            "temperature": temperature, "masked": masked}


def _attention(name, seqs, least, most, heads, kv_heads, dim, page, dtype, tokens_first=False):
    return {"name": name, "op": "attention", "seqs": seqs, "least": least, "most": most, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "tokens_first": tokens_first}


def _fork(name, groups, beams, least, most, grow, layers, kv_heads, dim, page, tokens_first=False):
    return {"name": name, "op": "fork", "groups": groups, "beams": beams, "least": least, "most": most, "grow": grow,
            "layers": layers, "kv_heads": kv_heads, "dim": dim, "page": page, "tokens_first": tokens_first}


def _compact(name, pages, live, seqs, layers, kv_heads, dim, page):
    return {"name": name, "op": "compact", "pages": pages, "live": live, "seqs": seqs, "layers": layers,
            "kv_heads": kv_heads, "dim": dim, "page": page}


def listed():
    return [
        # one step of a beam search with four beams: the scores that the next selection is made from; latency counts
        _logprobs("logprobs 4 beams", 4, 32768, "f32", 8, entropy=False),
        # a serving batch that answers with the twenty best alternatives, most rows under a grammar that forbids most
        # tokens, one of them all; an odd vocabulary, so that rows start at any alignment
        _logprobs("logprobs batch masked", 61, 131071, "bf16", 20, temperature=0.7, masked=True),
        # scoring a batch of 4096 tokens, as for distillation: log probability, entropy and the five best
        _logprobs("logprobs scoring", 4096, 131072, "bf16", 5),
        # the gradient of a policy loss over a small batch in 32 bits
        _gradient("gradient small", 100, 50001, "f32", 4, temperature=0.7, masked=True),
        # the gradient of a training step over 4096 tokens
        _gradient("gradient step", 4096, 131072, "bf16", 0),
        # one conversation: the latency of a single short sequence
        _attention("attention one", 1, 1000, 1000, 32, 8, 128, 16, "bf16"),
        # a serving batch of ragged lengths with shared key-value heads
        _attention("attention ragged", 32, 1, 8192, 64, 8, 128, 16, "bf16"),
        # many short sequences, each head with keys of its own, a cache laid out tokens first
        _attention("attention many short", 200, 17, 700, 16, 16, 64, 32, "f16", tokens_first=True),
        # few very long contexts
        _attention("attention long", 4, 100000, 131072, 32, 8, 128, 64, "bf16"),
        # the fork of one small beam search: latency
        _fork("fork one search", 1, 8, 200, 200, 1, 4, 8, 128, 16),
        # the fork of 32 searches of eight beams on a deep model's cache
        _fork("fork many", 32, 8, 64, 1000, 1, 16, 8, 128, 16),
        # moving a half-empty pool's live pages to its front
        _compact("compact half", 2000, 1000, 64, 16, 8, 128, 16),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprobs", "gradient", "attention", "attention", "fork", "compact"])
    if kind in ("logprobs", "gradient"):
        rows, vocab = _spread(rng, 1, 4096), _spread(rng, 1000, 200000)
        dtype = rng.choice(["f32", "bf16", "f16"])
        while rows * vocab * BYTES[dtype] > 4096 * 131072 * 2:
            rows = rows // 2
        temperature, masked = rng.choice([1.0, 0.7, 1.3]), rng.random() < 0.4
        if kind == "logprobs":
            c = _logprobs("", rows, vocab, dtype, rng.choice([0, 1, 5, 8, 20, 64, 100]), temperature, masked, rng.random() < 0.6)
        else:
            c = _gradient("", rows, vocab, dtype, rng.choice([0, 0, 4, 20]), temperature, masked)
    elif kind == "attention":
        dim, kv_heads, group = rng.choice([64, 128, 128, 96, 256]), rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 5, 7, 8, 16])
        seqs, most = _spread(rng, 1, 256), _spread(rng, 16, 131072)
        while seqs * most * kv_heads * dim > 4 * 131072 * 8 * 128 // 2:
            seqs, most = max(1, seqs // 2), max(16, most // 2)
        least = rng.choice([1, max(1, most // 4), most])
        c = _attention("", seqs, least, most, kv_heads * group, kv_heads, dim, rng.choice([8, 16, 24, 32, 64]),
                       rng.choice(["bf16", "f16"]), rng.random() < 0.4)
    elif kind == "fork":
        groups, beams = _spread(rng, 1, 48), rng.choice([1, 2, 4, 5, 8, 16])
        layers, kv_heads, dim, page = _spread(rng, 1, 24), rng.choice([1, 2, 4, 8]), rng.choice([64, 96, 128]), rng.choice([8, 16, 24, 32, 64])
        most = _spread(rng, 16, 2000)
        least = rng.choice([1, max(1, most // 4), most])
        c = _fork("", groups, beams, least, most, rng.choice([0, 1, 1, 4]), layers, kv_heads, dim, page, rng.random() < 0.4)
        while _fork_pages(c) * _page_bytes(c) > 2 << 30 or groups * beams > 400:
            groups, most, layers = max(1, groups // 2), max(16, most // 2), max(1, layers // 2)
            c.update(groups=groups, most=most, least=min(c["least"], most), layers=layers)
    else:
        layers, kv_heads, dim, page = _spread(rng, 1, 24), rng.choice([1, 2, 4, 8]), rng.choice([64, 96, 128]), rng.choice([8, 16, 24, 32, 64])
        pages = _spread(rng, 50, 20000)
        c = _compact("", pages, 1, _spread(rng, 1, 64), layers, kv_heads, dim, page)
        while c["pages"] * _page_bytes(c) > 2 << 30:
            c["pages"] //= 2
        c["live"] = max(1, int(c["pages"] * rng.uniform(0.1, 0.95)))
        c["seqs"] = min(c["seqs"], c["live"])
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------------
# what a user's program has in hand

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _lengths(least, most, n, g):
    """n lengths spread evenly over [least, most], in an order that the seed gives; int32."""
    x = torch.tensor(_length_list(least, most, n), dtype=torch.int32, device="cuda")
    return x[torch.randperm(n, generator=g, device="cuda")]


def _length_list(least, most, n):
    return [most] if n == 1 else [round(least + (most - least) * i / (n - 1)) for i in range(n)]


def _logits(case, g):
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3.0
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    if case["masked"]:
        # a grammar's mask: about one token in a hundred is allowed in two rows of three, the given token among them
        allowed = torch.rand(rows, vocab, generator=g, device="cuda") < 0.01
        allowed.scatter_(1, tokens[:, None], True)
        allowed |= (torch.arange(rows, device="cuda") % 3 == 0)[:, None]
        x.masked_fill_(~allowed, -math.inf)
        if rows > 3:
            x[rows // 2] = -math.inf             # nothing is allowed here
            tokens[rows // 3] = -100             # no token is given here
    return x.to(DTYPES[case["dtype"]]), tokens


def _prepare_gradient(case, g):
    x, tokens = _logits(case, g)
    rows, k, t = case["rows"], case["k"], case["temperature"]
    z = x.float() * (1.0 / t)
    lse = torch.logsumexp(z, -1)
    shifted = z - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None]
    p = torch.exp(shifted)
    entropy = -torch.where(p > 0, p * shifted, torch.zeros_like(p)).sum(-1)
    del z, shifted, p
    top = torch.topk(x, k, dim=-1).indices if k else None
    return {"logits": x, "tokens": tokens, "lse": lse, "entropy": entropy, "top": top,
            "g_logprob": torch.randn(rows, generator=g, device="cuda"),
            "g_entropy": torch.randn(rows, generator=g, device="cuda") * 0.1,
            "g_top": torch.randn(rows, k, generator=g, device="cuda") if k else None}


def _prepare_attention(case, g):
    seqs, page, kvh, dim = case["seqs"], case["page"], case["kv_heads"], case["dim"]
    lengths = _lengths(case["least"], case["most"], seqs, g)
    width = -(-case["most"] // page)
    need = (lengths + page - 1) // page
    total = sum(-(-n // page) for n in _length_list(case["least"], case["most"], seqs)) + 8
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(width, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    tables = torch.where(col < need[:, None], order[at.clamp(max=total - 1)], torch.full_like(at, -1, dtype=torch.int32))
    shape = (total, page, kvh, dim) if case["tokens_first"] else (total, kvh, page, dim)
    k, v = (torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]]) for _ in range(2))
    if case["tokens_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    q = (torch.randn(seqs, case["heads"], dim, generator=g, device="cuda") * 1.5).to(DTYPES[case["dtype"]])
    return {"q": q, "k": k, "v": v, "tables": tables.to(torch.int32), "lengths": lengths, "scale": dim ** -0.5}


def _page_bytes(case):
    return case["layers"] * 2 * case["kv_heads"] * case["page"] * case["dim"] * 2


def _shared_pages(case):
    return case["least"] // case["page"] // 2          # of each search's prompt


def _fork_pages(case):
    seqs = case["groups"] * case["beams"]
    own_pages = sum(-(-n // case["page"]) for n in _length_list(case["least"], case["most"], seqs)) - seqs * _shared_pages(case)
    return case["groups"] * _shared_pages(case) + own_pages + seqs * (1 + -(-case["grow"] // case["page"]))


def _pool(case, pages, g):
    """A cache of random bits, (layers, 2, pages, kv_heads, page, dim) in bf16."""
    shape = (case["layers"], 2, pages, case["kv_heads"], case["page"], case["dim"])
    if case.get("tokens_first"):
        shape = shape[:3] + (shape[4], shape[3], shape[5])
    pool = torch.randint(-32768, 32768, shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
    return pool.transpose(3, 4) if case.get("tokens_first") else pool


def _prepare_fork(case, g):
    page, beams, groups = case["page"], case["beams"], case["groups"]
    seqs, shared, pages = groups * beams, _shared_pages(case), _fork_pages(case)
    lengths = _lengths(case["least"], case["most"], seqs, g)
    need = (lengths + page - 1) // page - shared
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = -(-(case["most"] + case["grow"]) // page)
    col = torch.arange(width, device="cuda")
    group = (torch.arange(seqs, device="cuda") // beams)[:, None]
    at = torch.where(col < shared, group * shared + col, groups * shared + (torch.cumsum(need, 0) - need)[:, None] + col - shared)
    held = col < (need + shared)[:, None]
    tables = torch.where(held, order[at.clamp(max=pages - 1)], torch.full_like(at, -1, dtype=torch.int32)).to(torch.int32)
    refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    refs.scatter_add_(0, torch.where(held, tables, torch.full_like(tables, pages)).flatten().long(), torch.ones(seqs * width, dtype=torch.int32, device="cuda"))
    parents = torch.randint(0, beams, (seqs,), generator=g, device="cuda") + group[:, 0] * beams
    return {"pool": _pool(case, pages, g), "tables": tables, "lengths": lengths, "refs": refs[:pages].contiguous(),
            "parents": parents.to(torch.int32), "grow": case["grow"]}


def _prepare_compact(case, g):
    pages, live, seqs = case["pages"], case["live"], case["seqs"]
    order = torch.randperm(pages, generator=g, device="cuda")[:live].to(torch.int32)
    width = -(-live // seqs) + 1
    at = torch.arange(seqs, device="cuda")[:, None] * (width - 1) + torch.arange(width, device="cuda") - 1
    at[:, 0] = 0                                       # every sequence begins with the same page
    tables = torch.where(at < live, order[at.clamp(max=live - 1)], torch.full_like(at, -1, dtype=torch.int32)).to(torch.int32)
    refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    refs.scatter_add_(0, torch.where(tables >= 0, tables, torch.full_like(tables, pages)).flatten().long(), torch.ones(seqs * width, dtype=torch.int32, device="cuda"))
    return {"pool": _pool(case, pages, g), "tables": tables, "refs": refs[:pages].contiguous()}


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "logprobs":
        x, tokens = _logits(case, g)
        state = {"logits": x, "tokens": tokens}
    else:
        state = {"gradient": _prepare_gradient, "attention": _prepare_attention, "fork": _prepare_fork, "compact": _prepare_compact}[op](case, g)
    state["case"] = dict(case)
    return state


# ---------------------------------------------------------------------------------------------------------------------
# plain forms

def _plain_logprobs(s):
    case, x, tokens = s["case"], s["logits"], s["tokens"]
    vocab, k = case["vocab"], case["k"]
    z = x.float() * (1.0 / case["temperature"])
    m = z.amax(-1)
    empty = m == -math.inf
    m = torch.where(empty, torch.zeros_like(m), m)
    d = z - m[:, None]
    e = torch.exp(d)
    total = e.sum(-1)
    log_total = torch.log(total)
    lse = m + log_total
    given = (tokens >= 0)
    at = torch.where(given, tokens, torch.zeros_like(tokens))[:, None]
    minus = torch.full_like(lse, -math.inf)
    nought = torch.zeros_like(lse)
    logprob = torch.where(empty, minus, d.gather(1, at)[:, 0] - log_total)
    out = {"logprob": torch.where(given, logprob, nought), "lse": lse}
    if case["entropy"]:
        out["entropy"] = torch.where(empty, nought, log_total - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(-1) / total)
    if k:
        # the largest logits, of equal ones the lowest index: one whole number holds both
        bits = x.float().view(torch.int32).long()
        order = torch.where(bits < 0, -2147483648 - bits, bits)
        key = (order << 32) + (vocab - torch.arange(vocab, device=x.device))
        best = vocab - (torch.topk(key, k, dim=-1).values & 0xFFFFFFFF)
        out["top_tokens"] = best
        out["top_logprobs"] = torch.where(empty[:, None], minus[:, None], d.gather(1, best) - log_total[:, None])
    return out


def _plain_gradient(s):
    case, x, tokens, lse = s["case"], s["logits"], s["tokens"], s["lse"]
    inv = 1.0 / case["temperature"]
    empty = lse == -math.inf
    given = (tokens >= 0)
    g_logprob = torch.where(given, s["g_logprob"], torch.zeros_like(lse))
    whole = g_logprob + (s["g_top"].sum(-1) if case["k"] else 0.0)
    logp = x.float() * inv - torch.where(empty, torch.zeros_like(lse), lse)[:, None]
    p = torch.exp(logp)
    inner = whole[:, None] + s["g_entropy"][:, None] * (logp + s["entropy"][:, None])
    dz = torch.where(p > 0, -p * inner, torch.zeros_like(p))
    dz.scatter_add_(1, torch.where(given, tokens, torch.zeros_like(tokens))[:, None], g_logprob[:, None])
    if case["k"]:
        dz.scatter_add_(1, s["top"], s["g_top"])
    return {"grad": torch.where(empty[:, None], torch.zeros_like(dz), dz * inv).to(x.dtype)}


def _plain_attention(s):
    case, q, tables, lengths = s["case"], s["q"], s["tables"], s["lengths"]
    seqs, kvh, dim = case["seqs"], case["kv_heads"], case["dim"]
    at = tables.clamp(min=0).long()
    k, v = (c[at].transpose(1, 2).reshape(seqs, kvh, -1, dim).float() for c in (s["k"], s["v"]))
    scores = torch.matmul(q.float().view(seqs, kvh, -1, dim), k.transpose(2, 3)) * s["scale"]
    held = torch.arange(k.shape[2], device=q.device) < lengths[:, None]
    scores = scores.masked_fill(~held[:, None, None, :], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - m)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total
    return {"out": out.view(q.shape).to(q.dtype), "lse": (m + torch.log(total)).view(seqs, -1)}


def _bits(pool):
    return pool.view(torch.int16)


def _plain_fork(s):
    pool, tables, lengths, refs, grow = s["pool"], s["tables"], s["lengths"].long(), s["refs"], s["grow"]
    parents = s["parents"].long()
    n_old, width = tables.shape
    n, pages, page = parents.shape[0], refs.shape[0], pool.shape[-2]
    dev = tables.device
    i, col = torch.arange(n, device=dev), torch.arange(width, device=dev)
    old = lengths[parents]
    length = (old + grow).clamp(max=width * page)
    have, want, fill = (old + page - 1) // page, (length + page - 1) // page, old % page
    first = torch.full((n_old,), n, device=dev).scatter_reduce(0, parents, i, "amin")
    copied = (fill > 0) & (first[parents] != i)
    inherited = (col < have[:, None]) & ~(copied[:, None] & (col == have[:, None] - 1))
    fresh = (col < want[:, None]) & ~inherited
    # the lowest-numbered free pages, in the order of need
    free = refs <= 0
    lowest = torch.full((pages + 1,), -1, device=dev)
    lowest.scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, torch.full((pages,), pages, device=dev)), torch.arange(pages, device=dev))
    number = torch.cumsum(fresh.flatten(), 0).view(n, width) - 1
    got = torch.where(number < free.sum(), lowest[number.clamp(0, pages - 1)], torch.full_like(number, -1))
    new = torch.where(inherited, tables[parents].long(), torch.where(fresh, got, torch.full_like(got, -1)))
    missing = (fresh & (new < 0)).sum()
    one = torch.ones(1, dtype=torch.int32, device=dev)
    counts = torch.cat([refs, torch.zeros_like(refs[:1])])
    before = torch.where(col < ((lengths + page - 1) // page)[:, None], tables.long(), torch.full_like(tables, pages, dtype=torch.int64))
    counts.scatter_add_(0, before.flatten(), -one.expand(before.numel()))
    after = torch.where(new >= 0, new, torch.full_like(new, pages))
    counts.scatter_add_(0, after.flatten(), one.expand(after.numel()))
    # the tokens of the copied pages
    who = copied.nonzero()[:, 0]
    where = have[who] - 1
    src, dst = tables[parents[who], where].long(), new[who, where]
    tokens = torch.arange(page, device=dev) < fill[who][:, None]
    bits = _bits(pool)
    bits[:, :, dst] = torch.where(tokens[:, None, :, None], bits[:, :, src], bits[:, :, dst])
    return {"pool": bits, "tables": new.to(torch.int32), "lengths": length.to(torch.int32), "refs": counts[:pages], "missing": missing.to(torch.int32)}


def _plain_compact(s):
    pool, tables, refs = s["pool"], s["tables"], s["refs"]
    pages = refs.shape[0]
    ids = torch.arange(pages, device=refs.device)
    held = refs > 0
    live = held.sum()
    src, dst = (held & (ids >= live)).nonzero()[:, 0], (~held & (ids < live)).nonzero()[:, 0]
    page_map = torch.where(held, ids, torch.full_like(ids, -1))
    page_map[src] = dst
    bits = _bits(pool)
    bits[:, :, dst] = bits[:, :, src]
    new_refs = torch.where(held & (ids < live), refs, torch.zeros_like(refs))
    new_refs[dst] = refs[src]
    new = torch.where(tables >= 0, page_map[tables.clamp(min=0).long()].to(torch.int32), torch.full_like(tables, -1))
    return {"pool": bits, "tables": new, "refs": new_refs, "page_map": page_map.to(torch.int32), "live": live.to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------------
# the library's calls

def _own(s):
    import paper_2608_12573_b200 as profk

    case = s["case"]
    op = case["op"]
    if op == "logprobs":
        r = profk.logprobs(s["logits"], s["tokens"], k=case["k"], temperature=case["temperature"], entropy=case["entropy"])
        out = {"logprob": r.logprob, "lse": r.lse}
        if case["entropy"]:
            out["entropy"] = r.entropy
        if case["k"]:
            out["top_tokens"], out["top_logprobs"] = r.top_tokens, r.top_logprobs
        return out
    if op == "gradient":
        return {"grad": profk.logprobs_backward(s["logits"], s["lse"], s["tokens"], s["g_logprob"], entropy=s["entropy"],
                                                grad_entropy=s["g_entropy"], top_tokens=s["top"], grad_top=s["g_top"],
                                                temperature=case["temperature"])}
    if op == "attention":
        out, lse = profk.paged_attention(s["q"], s["k"], s["v"], s["tables"], s["lengths"], scale=s["scale"])
        return {"out": out, "lse": lse}
    if op == "fork":
        r = profk.pages_fork(s["pool"], s["tables"], s["lengths"], s["refs"], s["parents"], grow=s["grow"])
        return {"pool": _bits(s["pool"]), "tables": r.tables, "lengths": r.lengths, "refs": r.refs, "missing": r.missing}
    r = profk.pages_compact(s["pool"], s["tables"], s["refs"])
    return {"pool": _bits(s["pool"]), "tables": r.tables, "refs": r.refs, "page_map": r.page_map, "live": r.live}


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "gradient": _plain_gradient, "attention": _plain_attention,
            "fork": _plain_fork, "compact": _plain_compact}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    op = case["op"]
    if op in ("logprobs", "gradient"):
        n, b = case["rows"] * case["vocab"], BYTES[case["dtype"]]
        per_row = 16 + 12 * case["k"]
        if op == "logprobs":
            return {"bytes": n * b + case["rows"] * per_row, "flops": n * (6 if case["entropy"] else 4)}
        return {"bytes": 2 * n * b + case["rows"] * (per_row + 16), "flops": n * 7}
    if op == "attention":
        tokens = sum(_length_list(case["least"], case["most"], case["seqs"]))
        rows = case["seqs"] * case["heads"]
        return {"bytes": tokens * case["kv_heads"] * case["dim"] * 4 + rows * case["dim"] * 4 + rows * 4, "flops": 4 * tokens * case["heads"] * case["dim"]}
    if op == "fork":
        beams, page = case["beams"], case["page"]
        seqs = case["groups"] * beams
        copies = case["groups"] * beams * (1 - 1 / beams) ** beams     # expected children that are not a parent's first
        fills = [n % page for n in _length_list(case["least"], case["most"], seqs)]
        moved = copies * sum(fills) / len(fills) / page * _page_bytes(case)
        width = -(-(case["most"] + case["grow"]) // page)
        return {"bytes": 2 * moved + 8 * seqs * width + 8 * _fork_pages(case), "flops": 0}
    moved = case["live"] * (1 - case["live"] / case["pages"]) * _page_bytes(case)
    return {"bytes": 2 * moved + 12 * case["pages"] + 8 * (case["live"] + 2 * case["seqs"]), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits

def _exact_logprobs(s):
    case, tokens = s["case"], s["tokens"].tolist()
    inv = 1.0 / case["temperature"]
    logprob, entropy, lse, top = [], [], [], []
    for r0 in range(0, case["rows"], 256):
        z = s["logits"][r0:r0 + 256].double() * inv
        full = torch.logsumexp(z, 1)
        lse.append(full)
        t = torch.tensor(tokens[r0:r0 + 256], device=z.device)
        own_token = z[torch.arange(z.shape[0], device=z.device), t.clamp(min=0)]
        lp = torch.where(torch.isinf(full), full, own_token - full)
        logprob.append(torch.where(t < 0, torch.zeros_like(lp), lp))
        log_p = z - torch.where(torch.isinf(full), torch.zeros_like(full), full)[:, None]
        entropy.append(torch.special.entr(torch.exp(log_p)).sum(1))
        if case["k"]:
            best = torch.sort(z, dim=1, descending=True).values[:, :case["k"]]
            top.append(torch.where(torch.isinf(full)[:, None], best, best - full[:, None]))
    out = {"logprob": torch.cat(logprob), "lse": torch.cat(lse)}
    if case["entropy"]:
        out["entropy"] = torch.cat(entropy)
    if case["k"]:
        out["top_tokens"], out["top_logprobs"] = None, torch.cat(top)
    return out


def _exact_gradient(s):
    """Of L = sum over rows of g_logprob * logprob + g_entropy * entropy + g_top . top_logprobs, row by row in blocks, with
    the log probabilities and the entropy taken from the logits themselves."""
    case = s["case"]
    parts = []
    for r0 in range(0, case["rows"], 256):
        sl = slice(r0, r0 + 256)
        z = s["logits"][sl].double() / case["temperature"]
        t = s["tokens"][sl]
        full = torch.logsumexp(z, 1)
        nothing = torch.isinf(full)
        log_p = z - torch.where(nothing, torch.zeros_like(full), full)[:, None]
        p = torch.exp(log_p)
        entropy = torch.special.entr(p).sum(1, keepdim=True)
        upstream = torch.zeros_like(z)                                 # dL / d log_p through the picked entries
        upstream[torch.arange(z.shape[0], device=z.device), t.clamp(min=0)] += torch.where(t < 0, 0.0, s["g_logprob"][sl].double())
        if case["k"]:
            upstream.scatter_add_(1, s["top"][sl], s["g_top"][sl].double())
        grad = upstream - p * upstream.sum(1, keepdim=True)
        grad += s["g_entropy"][sl].double()[:, None] * (torch.special.entr(p) - p * entropy)
        grad[nothing] = 0.0
        parts.append((grad / case["temperature"]).float() if case["dtype"] != "f32" else grad / case["temperature"])
    return {"grad": torch.cat(parts)}


def _exact_attention(s):
    case = s["case"]
    out, lse = [], []
    tables, lengths = s["tables"].tolist(), s["lengths"].tolist()
    for b in range(case["seqs"]):
        n = lengths[b]
        ids = torch.tensor(tables[b][:-(-n // case["page"])], device="cuda")
        k, v = (torch.cat([x for x in c[ids].double().permute(1, 0, 2, 3).flatten(1, 2)[None]])[:, :n] for c in (s["k"], s["v"]))
        q = s["q"][b].double().unflatten(0, (case["kv_heads"], -1))
        scores = torch.einsum("hgd,htd->hgt", q, k) * s["scale"]
        total = torch.logsumexp(scores, -1)
        out.append(torch.einsum("hgt,htd->hgd", torch.exp(scores - total[..., None]), v).flatten(0, 1))
        lse.append(total.flatten())
    return {"out": torch.stack(out), "lse": torch.stack(lse)}


def exact(case, seed):
    how = {"logprobs": _exact_logprobs, "gradient": _exact_gradient, "attention": _exact_attention}.get(case["op"])
    return how(prepare(case, seed)) if how else None     # pages are moved, not computed: whole numbers, compared bit for bit
