"""The operators that take prompts and drafts into a decoding loop, as they are timed and compared: rotary positions (and
their gradient), the appending of rotated keys and values to a paged cache, attention of a chunk of new tokens over that
cache, and the penalties, biases and masks that are laid over logits before a selection.

`run` computes a case either in its plain form (elementary torch operations in 32 bits, angles in 64) or, where `own` is
true, through the library's public functions.  `exact` computes it from the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------------------------------------------------
# cases

def _rotary(name, tokens, heads, dim, turned, dtype, interleaved=False, far=0, stretch=1.0, magnitude=1.0, gradient=False):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "dim": dim, "turned": turned, "dtype": dtype,
            "interleaved": interleaved, "far": far, "stretch": stretch, "magnitude": magnitude, "gradient": gradient}


def _append(name, seqs, new_least, new_most, held, heads, kv_heads, dim, turned, page, dtype, interleaved=False, tokens_first=False):
    return {"name": name, "op": "append", "seqs": seqs, "new_least": new_least, "new_most": new_most, "held": held, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "turned": turned, "page": page, "dtype": dtype, "interleaved": interleaved,
            "tokens_first": tokens_first}


def _chunk(name, seqs, new_least, new_most, least, most, heads, kv_heads, dim, page, dtype, tokens_first=False):
    """Between `new_least` and `new_most` new tokens to a sequence, behind between `least` and `most` that are there already."""
    return {"name": name, "op": "chunk", "seqs": seqs, "new_least": new_least, "new_most": new_most, "least": least, "most": most,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "tokens_first": tokens_first}


def _adjust(name, rows, vocab, dtype, history, biases, masked):
    return {"name": name, "op": "adjust", "rows": rows, "vocab": vocab, "dtype": dtype, "history": history, "biases": biases,
            "masked": masked}


def listed():
    return [
        # positions of a small odd batch in 32 bits, part of each head turned, far positions, frequencies stretched for them
        _rotary("rotary small", 333, 5, 80, 40, "f32", far=1000000, stretch=8.0, magnitude=1.2),
        # the queries of a training batch of 16384 tokens, forward and backward
        _rotary("rotary training", 16384, 32, 128, 128, "bf16", gradient=True),
        # one step of 64 conversations: the new token's query turned, its key and value put into the cache; latency counts
        _append("append step", 64, 1, 1, 4000, 32, 8, 128, 128, 16, "bf16"),
        # sixteen ragged prompts into a cache laid out tokens first, neighbouring elements turned, half of each head
        _append("append prompts", 16, 1, 2047, 0, 64, 8, 128, 64, 24, "f16", interleaved=True, tokens_first=True),
        # one prompt: latency
        _chunk("chunk one prompt", 1, 301, 301, 0, 0, 32, 8, 128, 16, "bf16"),
        # four drafted tokens of each of 32 ragged sequences are checked
        _chunk("chunk drafts", 32, 4, 4, 1, 8192, 64, 8, 128, 16, "bf16"),
        # ragged prompts behind a shared beginning, each head with keys of its own, a cache laid out tokens first
        _chunk("chunk ragged prompts", 24, 1, 2500, 200, 200, 16, 16, 64, 32, "f16", tokens_first=True),
        # the last part of two very long prompts
        _chunk("chunk long", 2, 2048, 2048, 65536, 129024, 32, 8, 128, 64, "bf16"),
        # one step of a beam search with four beams: latency
        _adjust("adjust 4 beams", 4, 32768, "f32", 200, 0, False),
        # a serving batch under a grammar, with biases; an odd vocabulary, so that rows start at any alignment
        _adjust("adjust batch", 256, 131071, "bf16", 4096, 30, True),
        # long conversations
        _adjust("adjust long histories", 64, 131072, "f32", 100000, 0, False),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "chunk", "chunk", "adjust"])
    dtype = rng.choice(["bf16", "f16"])
    if kind == "rotary":
        dim = rng.choice([16, 64, 80, 96, 128, 256])
        turned = rng.choice([dim, dim, dim // 2, dim // 4])
        heads = rng.choice([1, 5, 8, 16, 32, 64])
        tokens = _spread(rng, 1, 65536)
        while tokens * heads * dim > 16384 * 32 * 128:
            tokens //= 2
        c = _rotary("", max(1, tokens), heads, dim, turned, rng.choice(["f32", "bf16", "f16"]), rng.random() < 0.5,
                    rng.choice([0, 5000, 1000000]), rng.choice([1.0, 1.0, 4.0, 32.0]), rng.choice([1.0, 1.1]), rng.random() < 0.5)
    elif kind in ("append", "chunk"):
        dim, kv_heads, group = rng.choice([64, 128, 128, 96, 256]), rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 5, 7, 8, 16])
        page, tokens_first = rng.choice([8, 16, 24, 32, 64]), rng.random() < 0.4
        seqs = _spread(rng, 1, 256)
        new_most = rng.choice([1, 2, 4, 7, 16, _spread(rng, 17, 4096), _spread(rng, 17, 4096)])
        if kind == "append":
            while seqs * new_most * kv_heads * (group + 2) * dim > 16384 * 80 * 128:
                seqs, new_most = max(1, seqs // 2), max(1, new_most // 2)
            c = _append("", seqs, rng.choice([1, new_most]), new_most, rng.choice([0, 33, 4000]), kv_heads * group, kv_heads, dim,
                        rng.choice([dim, dim, dim // 2]), page, dtype, rng.random() < 0.5, tokens_first)
        else:
            most = rng.choice([0, _spread(rng, 16, 131072), _spread(rng, 16, 131072)])
            while seqs * (most + new_most) * kv_heads * dim > 2 * 131072 * 8 * 128 or \
                    seqs * new_most * (most + new_most) * kv_heads * group * dim > 2 * 2048 * 98304 * 32 * 128:
                seqs, most, new_most = max(1, seqs // 2), most // 2, max(1, new_most * 3 // 4)
            c = _chunk("", seqs, rng.choice([1, new_most]), new_most, rng.choice([most // 4, most]), most, kv_heads * group, kv_heads, dim,
                       page, dtype, tokens_first)
    else:
        rows, vocab = _spread(rng, 1, 1024), _spread(rng, 1000, 200000)
        dtype = rng.choice(["f32", "bf16", "f16"])
        while rows * vocab * BYTES[dtype] > 256 * 131072 * 2:
            rows //= 2
        c = _adjust("", rows, vocab, dtype, rng.choice([0, _spread(rng, 1, 100000), _spread(rng, 1, 8192)]), rng.choice([0, 0, 1, 30, 300]), rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------------
# what a user's program has in hand

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _even(least, most, n):
    """n whole numbers spread evenly over [least, most]."""
    return [most] if n == 1 else [round(least + (most - least) * i / (n - 1)) for i in range(n)]


def _shuffled(values, g):
    x = torch.tensor(values, dtype=torch.int32, device="cuda")
    return x[torch.randperm(len(values), generator=g, device="cuda")]


def _frequencies(turned, stretch=1.0):
    """Angle per position of every pair, in 64 bits; stretched: the slow pairs (long wavelengths) are slowed down further."""
    i = torch.arange(turned // 2, dtype=torch.float64, device="cuda")
    f = 10000.0 ** (-2.0 * i / turned)
    share = (i / max(1, turned // 2 - 1)).clamp(0, 1)
    return f * (1 - share) + f / stretch * share


def _randn(shape, g, dtype, factor=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * factor).to(DTYPES[dtype])


def _prepare_rotary(case, g):
    tokens, shape = case["tokens"], (case["tokens"], case["heads"], case["dim"])
    positions = torch.arange(tokens, device="cuda")
    if case["far"]:
        positions = torch.randint(0, case["far"], (tokens,), generator=g, device="cuda")
    s = {"x": _randn(shape, g, case["dtype"]), "positions": positions, "frequencies": _frequencies(case["turned"], case["stretch"])}
    if case["gradient"]:
        s["x"].requires_grad_(True)
        s["upstream"] = _randn(shape, g, case["dtype"])
    return s


def _cache(case, lengths, most, g):
    """Room for `most` tokens of every sequence, in pages in a random order: (k_pages, v_pages, tables)."""
    page, kvh, dim = case["page"], case["kv_heads"], case["dim"]
    need, width = (lengths + page - 1) // page, -(-most // page)
    total = case["seqs"] * width + 8
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(width, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    tables = torch.where(col < need[:, None], order[at.clamp(max=total - 1)], torch.full_like(at, -1, dtype=torch.int32))
    shape = (total, page, kvh, dim) if case["tokens_first"] else (total, kvh, page, dim)
    k, v = (torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]]) for _ in range(2))
    if case["tokens_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return k, v, tables.to(torch.int32)


def _prepare_append(case, g):
    new = _shuffled(_even(case["new_least"], case["new_most"], case["seqs"]), g)
    held = torch.randint(case["held"] // 2, case["held"] + 1, (case["seqs"],), generator=g, device="cuda").to(torch.int32)
    lengths = held + new
    k_pages, v_pages, tables = _cache(case, lengths, case["held"] + case["new_most"], g)
    rows = sum(_even(case["new_least"], case["new_most"], case["seqs"]))
    starts = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0, dtype=torch.int32)])
    # as they come from one projection: queries, keys and values side by side
    joint = _randn((rows, case["heads"] + 2 * case["kv_heads"], case["dim"]), g, case["dtype"])
    q, k, v = joint.split([case["heads"], case["kv_heads"], case["kv_heads"]], 1)
    return {"q": q, "k": k, "v": v, "k_pages": k_pages, "v_pages": v_pages, "tables": tables, "lengths": lengths, "starts": starts,
            "frequencies": _frequencies(case["turned"])}


def _prepare_chunk(case, g):
    news = _even(case["new_least"], case["new_most"], case["seqs"])
    new = _shuffled(news, g)
    lengths = _shuffled(_even(case["least"], case["most"], case["seqs"]), g) + new
    k, v, tables = _cache(case, lengths, case["most"] + case["new_most"], g)
    starts = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0, dtype=torch.int32)])
    q = _randn((sum(news), case["heads"], case["dim"]), g, case["dtype"], 1.5)
    return {"q": q, "k": k, "v": v, "tables": tables, "lengths": lengths, "starts": starts, "scale": case["dim"] ** -0.5}


def _prepare_adjust(case, g):
    rows, vocab, most = case["rows"], case["vocab"], case["history"]
    s = {"logits": _randn((rows, vocab), g, case["dtype"], 3.0)}
    if most:
        # few tokens come again and again: squares of even draws
        s["tokens"] = (torch.rand(rows, most, generator=g, device="cuda") ** 2 * vocab).long().clamp(max=vocab - 1)
        s["lengths"] = _shuffled(_even(most // 2, most, rows), g)
        s["prompts"] = s["lengths"] // 2
        s["repetition"] = 1.0 + torch.rand(rows, generator=g, device="cuda") * 0.3
        s["frequency"] = torch.rand(rows, generator=g, device="cuda") * 0.2
        s["presence"] = torch.rand(rows, generator=g, device="cuda") * 0.5
    if case["biases"]:
        s["bias_tokens"] = torch.randint(0, vocab, (rows, case["biases"]), generator=g, device="cuda")
        s["bias_values"] = torch.randn(rows, case["biases"], generator=g, device="cuda") * 5.0
    if case["masked"]:
        # a grammar's mask: about one token in a hundred is allowed in two rows of three
        words = -(-vocab // 32)
        mask = torch.zeros(rows, words, dtype=torch.int32, device="cuda")
        for bit in range(32):
            on = torch.rand(rows, words, generator=g, device="cuda") < 0.01
            mask |= on.to(torch.int32) << bit
        s["mask"] = torch.where((torch.arange(rows, device="cuda") % 3 == 0)[:, None], torch.full_like(mask, -1), mask)
    return s


def prepare(case, seed):
    g = _generator(seed)
    state = {"rotary": _prepare_rotary, "append": _prepare_append, "chunk": _prepare_chunk, "adjust": _prepare_adjust}[case["op"]](case, g)
    state["case"] = dict(case)
    return state


# ---------------------------------------------------------------------------------------------------------------------
# plain forms

def _turn(x, positions, frequencies, interleaved, magnitude=1.0):
    """x (tokens, heads, dim) in 32 bits, the first 2 * len(frequencies) elements of every head turned."""
    angle = positions.double()[:, None] * frequencies
    cos, sin = (torch.cos(angle) * magnitude).float()[:, None], (torch.sin(angle) * magnitude).float()[:, None]
    half = frequencies.shape[0]
    y = x.float().clone()
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    a, b = a.float(), b.float()
    first, second = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = first, second
    else:
        y[..., :half], y[..., half:2 * half] = first, second
    return y


def _plain_rotary(s):
    case, x = s["case"], s["x"]
    with torch.no_grad():
        out = {"y": _turn(x, s["positions"], s["frequencies"], case["interleaved"], case["magnitude"]).to(x.dtype)}
        if case["gradient"]:
            out["grad"] = _turn(s["upstream"], s["positions"], -s["frequencies"], case["interleaved"], case["magnitude"]).to(x.dtype)
    return out


def _places(s):
    """(sequence, place in it) of every row."""
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].contiguous(), row.to(torch.int32), right=True)
    return seq, s["lengths"].long()[seq] - new[seq] + row - s["starts"].long()[seq]


def _plain_append(s):
    case = s["case"]
    seq, place = _places(s)
    page = s["tables"][seq, place // case["page"]].long()
    slot = place % case["page"]
    s["k_pages"][page, :, slot] = _turn(s["k"], place, s["frequencies"], case["interleaved"]).to(s["k"].dtype)
    s["v_pages"][page, :, slot] = s["v"]
    return {"q": _turn(s["q"], place, s["frequencies"], case["interleaved"]).to(s["q"].dtype), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_chunk(s):
    case, q = s["case"], s["q"]
    kvh, dim, page = case["kv_heads"], case["dim"], case["page"]
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=q.device)
    for b in range(case["seqs"]):
        n = lengths[b]
        at = s["tables"][b, :-(-n // page)].long()
        k, v = (c[at].transpose(0, 1).reshape(kvh, -1, dim)[:, :n].float() for c in (s["k"], s["v"]))
        first = n - (starts[b + 1] - starts[b])
        step = max(1, (1 << 31) // (n * case["heads"]))          # rows whose scores are held at a time
        for r0 in range(starts[b], starts[b + 1], step):
            r1 = min(starts[b + 1], r0 + step)
            place = first + torch.arange(r0 - starts[b], r1 - starts[b], device=q.device)
            rows = q[r0:r1].float().view(r1 - r0, kvh, -1, dim).permute(1, 2, 0, 3).reshape(kvh, -1, dim)
            scores = (torch.matmul(rows, k.transpose(1, 2)) * s["scale"]).view(kvh, -1, r1 - r0, n)
            scores = scores.masked_fill(torch.arange(n, device=q.device) > place[:, None], -math.inf)
            m = scores.amax(-1, keepdim=True)
            p = torch.exp(scores - m)
            del scores
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(kvh, -1, n), v).view(kvh, -1, r1 - r0, dim) / total
            del p
            out[r0:r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, -1, dim).to(q.dtype)
            lse[r0:r1] = (m + torch.log(total))[..., 0].permute(2, 0, 1).reshape(r1 - r0, -1)
    return {"out": out, "lse": lse}


def _plain_adjust(s):
    case, x = s["case"], s["logits"]
    rows, vocab = case["rows"], case["vocab"]
    y = x.float()
    if case["history"]:
        col = torch.arange(case["history"], device=x.device)
        held = col < s["lengths"][:, None]
        answer = held & (col >= s["prompts"][:, None])
        one = torch.zeros(rows, vocab, dtype=torch.int32, device=x.device)
        seen = one.scatter_add(1, s["tokens"], held.to(torch.int32)) > 0
        count = one.scatter_add(1, s["tokens"], answer.to(torch.int32))
        rho = s["repetition"][:, None]
        y = torch.where(seen, torch.where(y > 0, y / rho, y * rho), y)
        y = y - (s["frequency"][:, None] * count + s["presence"][:, None] * (count > 0))
    if case["biases"]:
        y = y + torch.zeros_like(y).scatter_add_(1, s["bias_tokens"], s["bias_values"])
    if case["masked"]:
        v = torch.arange(vocab, device=x.device)
        y = y.masked_fill((s["mask"][:, v // 32] >> (v % 32)) & 1 == 0, -math.inf)
    return {"logits": y.to(x.dtype)}


# ---------------------------------------------------------------------------------------------------------------------
# the library's calls

def _own(s):
    import paper_2608_12573_b200 as profk

    case = s["case"]
    op = case["op"]
    if op == "rotary":
        y = profk.rotary(s["x"], s["positions"], s["frequencies"], interleaved=case["interleaved"], magnitude=case["magnitude"])
        if not case["gradient"]:
            return {"y": y}
        return {"y": y.detach(), "grad": torch.autograd.grad(y, s["x"], s["upstream"])[0]}
    if op == "append":
        q = profk.pages_append_rotary(s["k_pages"], s["v_pages"], s["tables"], s["lengths"], s["q"], s["k"], s["v"], s["frequencies"],
                                      starts=s["starts"], interleaved=case["interleaved"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if op == "chunk":
        out, lse = profk.paged_attention_chunk(s["q"], s["k"], s["v"], s["tables"], s["lengths"], starts=s["starts"], scale=s["scale"])
        return {"out": out, "lse": lse}
    given = {name: s[name] for name in ("tokens", "lengths", "prompts", "repetition", "frequency", "presence", "bias_tokens", "bias_values", "mask") if name in s}
    return {"logits": profk.adjust_logits(s["logits"], **given)}


def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "append": _plain_append, "chunk": _plain_chunk, "adjust": _plain_adjust}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    op = case["op"]
    b = BYTES[case["dtype"]]
    if op == "rotary":
        n = case["tokens"] * case["heads"] * case["dim"]
        passes = 2 if case["gradient"] else 1
        return {"bytes": passes * 2 * n * b + 8 * case["tokens"], "flops": passes * 3 * n * case["turned"] // case["dim"]}
    if op == "append":
        rows = sum(_even(case["new_least"], case["new_most"], case["seqs"]))
        n = rows * (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * n * b, "flops": 3 * rows * (case["heads"] + case["kv_heads"]) * case["turned"]}
    if op == "chunk":
        news, befores = _even(case["new_least"], case["new_most"], case["seqs"]), _even(case["least"], case["most"], case["seqs"])
        rows, seqs = sum(news), case["seqs"]
        # (which sequence has how many of either is the seed's)
        seen = sum(n * (n + 1) // 2 for n in news) + rows * (sum(befores) / seqs)
        held = rows + sum(befores)
        return {"bytes": held * case["kv_heads"] * case["dim"] * 2 * b + rows * case["heads"] * (case["dim"] * 2 * b + 4),
                "flops": int(4 * seen * case["heads"] * case["dim"])}
    rows, n = case["rows"], case["rows"] * case["vocab"]
    held = sum(_even(case["history"] // 2, case["history"], rows)) if case["history"] else 0
    return {"bytes": 2 * n * b + 8 * held + 12 * rows * case["biases"] + (n // 8 if case["masked"] else 0), "flops": 2 * held + n}


# ---------------------------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits

def _exact_turn(x, positions, frequencies, interleaved, magnitude=1.0):
    """Each pair as a complex number, times magnitude * e^(i position frequency)."""
    half = frequencies.shape[0]
    z = x.double()
    turned, rest = z[..., :2 * half], z[..., 2 * half:]
    pairs = turned.unflatten(-1, (half, 2)) if interleaved else turned.unflatten(-1, (2, half)).transpose(-1, -2)
    turn = torch.polar(torch.full((1,), float(magnitude), dtype=torch.float64, device=x.device), torch.outer(positions.double(), frequencies))
    w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
    w = w if interleaved else w.transpose(-1, -2)
    return torch.cat([w.flatten(-2), rest], -1)


def _exact_rotary(s):
    case = s["case"]
    with torch.no_grad():
        out = {"y": _exact_turn(s["x"], s["positions"], s["frequencies"], case["interleaved"], case["magnitude"])}
        if case["gradient"]:
            # the transpose of a turn is the turn back
            out["grad"] = _exact_turn(s["upstream"], -s["positions"], s["frequencies"], case["interleaved"], case["magnitude"])
    return out


def _exact_append(s):
    case = s["case"]
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    queries = []
    for b in range(case["seqs"]):
        rows = slice(starts[b], starts[b + 1])
        place = torch.arange(lengths[b] - (starts[b + 1] - starts[b]), lengths[b], device="cuda")
        k = _exact_turn(s["k"][rows], place, s["frequencies"], case["interleaved"])
        queries.append(_exact_turn(s["q"][rows], place, s["frequencies"], case["interleaved"]))
        where = (s["tables"][b][place // case["page"]].long(), slice(None), place % case["page"])
        k_pages[where], v_pages[where] = k, s["v"][rows].double()
    return {"q": torch.cat(queries), "k_pages": k_pages, "v_pages": v_pages}


def _exact_chunk(s):
    """Head by head, by the log-sum-exp of each row."""
    case = s["case"]
    starts, lengths, page, group = s["starts"].tolist(), s["lengths"].tolist(), case["page"], case["heads"] // case["kv_heads"]
    outs, lses = [], []
    for b in range(case["seqs"]):
        n, new = lengths[b], starts[b + 1] - starts[b]
        ids = s["tables"][b][:-(-n // page)].long()
        late = torch.ones(new, n, dtype=torch.bool, device="cuda").triu(n - new + 1)
        o, l = [], []
        for h in range(case["heads"]):
            if h % group == 0:
                k, v = (c[ids, h // group].double().flatten(0, 1)[:n] for c in (s["k"], s["v"]))
            scores = (s["q"][starts[b]:starts[b + 1], h].double() @ k.mT).mul_(s["scale"]).masked_fill_(late, -math.inf)
            total = torch.logsumexp(scores, 1)
            o.append(scores.sub_(total[:, None]).exp_() @ v)
            l.append(total)
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_adjust(s):
    case = s["case"]
    vocab, out = case["vocab"], []
    for r in range(case["rows"]):
        y = s["logits"][r].double()
        if case["history"]:
            n, first = int(s["lengths"][r]), int(s["prompts"][r])
            rho = s["repetition"][r].double()
            seen = torch.bincount(s["tokens"][r, :n], minlength=vocab) > 0
            count = torch.bincount(s["tokens"][r, first:n], minlength=vocab).double()
            y = torch.where(seen, y * rho ** (-torch.sign(y)), y)
            y = y - s["frequency"][r].double() * count - s["presence"][r].double() * count.clamp(max=1)
        if case["biases"]:
            y = y.index_add(0, s["bias_tokens"][r], s["bias_values"][r].double())
        if case["masked"]:
            bits = (s["mask"][r][:, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
            y = y + torch.log(bits.flatten()[:vocab].double())
        out.append(y if case["dtype"] == "f32" else y.float())
    return {"logits": torch.stack(out)}


def exact(case, seed):
    return {"rotary": _exact_rotary, "append": _exact_append, "chunk": _exact_chunk, "adjust": _exact_adjust}[case["op"]](prepare(case, seed))
