"""Operators on a paged K/V cache and on positions: cases, inputs, plain forms and the framework's calls.

A *paged cache* holds K and V rows in pages of one pool, [pages, page rows, heads, dim], float32 or bfloat16; a table gives each
sequence's pages in order, so a sequence grows without being moved.  Operators:

  rotate   rotary positions of one or several axes (time, height, width) applied to heads, or taken back (the gradient)
  append   new tokens' K and V written into their sequences' pages, K and the queries rotated on the way
  attend   attention of each sequence's new tokens (one, or a prompt) to its rows in the pages, causal; with a window W
           and S sinks a query at row p sees the rows x <= p with x < S or x > p - W

`run` computes an operator in elementary torch operations, or, where `own` is true, with the framework's calls.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _rotate(name, dtype, tokens, heads, dim, rotary, sections, pairs, reach, inverse=False):
    return {"name": name, "op": "rotate", "dtype": dtype, "tokens": tokens, "heads": heads, "dim": dim, "rotary": rotary,
            "axes": len(sections), "sections": "/".join(map(str, sections)), "pairs": pairs, "reach": reach, "inverse": inverse}


def _append(name, dtype, batch, heads, group, dim, page, new, held, rotary, sections, pairs, explicit):
    return {"name": name, "op": "append", "dtype": dtype, "batch": batch, "heads": heads, "group": group, "dim": dim, "page": page,
            "new": new, "held": held, "rotary": rotary, "axes": len(sections), "sections": "/".join(map(str, sections)), "pairs": pairs,
            "explicit": explicit}


def _attend(name, dtype, batch, heads, group, dim, page, new, length, window=0, sinks=0):
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "heads": heads, "group": group, "dim": dim, "page": page,
            "new": new, "length": length, "window": window, "sinks": sinks}


def listed():
    return [
        # queries of a video's 9001 patches, positions of three axes
        _rotate("rotate video", "bf16", 9001, 32, 128, 128, (16, 24, 24), "halves", 700),
        # the gradient of an image's 577 patches, two axes, float32
        _rotate("rotate image gradient", "f32", 577, 16, 64, 64, (16, 16), "neighbours", 24, inverse=True),
        # the new token of each of 64 sequences, four query heads to a K/V head: one such call for each layer and token
        _append("append step", "bf16", 64, 8, 4, 128, 16, 1, 2048, 128, (64,), "halves", False),
        # 16 ragged prompts of up to 1500 tokens enter an empty cache at once, with images among the text
        _append("append prompts", "bf16", 16, 32, 1, 128, 64, 1500, 0, 128, (16, 24, 24), "halves", True),
        # a small float32 model that turns a quarter of its channels, far into a stream
        _append("append float32", "f32", 3, 4, 1, 64, 24, 77, 1000, 16, (8,), "neighbours", True),
        # one token of each of 64 sequences of up to 4096: every layer, every token
        _attend("step", "bf16", 64, 32, 1, 128, 16, 1, 4096),
        # the same with grouped heads and long sequences
        _attend("step grouped", "bf16", 24, 8, 4, 128, 64, 1, 16384),
        # a handful of short sequences: latency is all
        _attend("step small", "bf16", 3, 8, 1, 64, 16, 1, 300),
        # float32 steps, pages of an odd size
        _attend("step float32", "f32", 16, 16, 1, 128, 24, 1, 1500),
        # streams of up to 8192 tokens of which the first four and the last 1020 are seen, the others' pages given back
        _attend("window step", "bf16", 64, 32, 1, 128, 16, 1, 8192, 1020, 4),
        # four ragged prompts of up to 4096 tokens under the same rule
        _attend("window prompts", "bf16", 4, 32, 1, 128, 64, 4096, 4096, 1020, 4),
        # the next 500 tokens of long prompts that are taken in pieces
        _attend("prompt pieces", "bf16", 4, 8, 4, 128, 32, 500, 8192),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _cut(rng, pairs, axes):
    """`pairs` pairs of channels shared out to the axes, each at least one."""
    at = sorted(rng.sample(range(1, pairs), axes - 1))
    return tuple(b - a for a, b in zip([0] + at, at + [pairs]))


def draw(rng):
    op = rng.choice(["rotate", "append step", "append prompts", "step", "step", "window step", "window prompts", "prompt pieces"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([64, 128, 128])
    rotary = rng.choice([dim, dim, dim // 2, dim // 4])
    sections = _cut(rng, rotary // 2, rng.choice([1, 1, 2, 3]))
    pairs = rng.choice(["halves", "halves", "neighbours"])
    group = rng.choice([1, 1, 2, 4, 8])
    heads = _log(rng, 1, 32 // group)
    page = rng.choice([8, 16, 16, 24, 32, 64, 64, 128])
    if op == "rotate":
        c = _rotate("", dtype, _log(rng, 1, 4500 if dtype == "f32" else 9000), _log(rng, 1, 32), dim, rotary, sections, pairs,
                    _log(rng, 10, 1000000), rng.random() < 0.3)
    elif op.startswith("append"):
        if op == "append step":
            c = _append("", dtype, _log(rng, 1, 64), heads, group, dim, page, 1, _log(rng, 1, 1000), rotary, sections, pairs, rng.random() < 0.5)
        else:
            c = _append("", dtype, _log(rng, 1, 16), heads, group, dim, page, _log(rng, 2, 700), rng.choice([0, 0, _log(rng, 1, 500)]), rotary,
                        sections, pairs, rng.random() < 0.5)
    elif op == "step":
        c = _attend("", dtype, _log(rng, 1, 64), heads, group, dim, page, 1, _log(rng, 1, 3500 if dtype == "bf16" else 1700))
    elif op == "window step":
        c = _attend("", dtype, _log(rng, 1, 64), heads, group, dim, page, 1, _log(rng, 1, 8192 if dtype == "bf16" else 4096),
                    _log(rng, 1, 2000 if dtype == "bf16" else 900),
                    rng.choice([0, 4, _log(rng, 1, 100)]))
    elif dtype == "f32":
        c = _attend("", dtype, _log(rng, 1, 4), heads, group, dim, page, _log(rng, 2, 200), _log(rng, 200, 1000), rng.choice([0, _log(rng, 1, 500)]),
                    rng.choice([0, 4]))
    elif op == "window prompts":
        n = _log(rng, 2, 2048)
        c = _attend("", dtype, _log(rng, 1, 4), heads, group, dim, page, n, n + rng.choice([0, _log(rng, 1, 2000)]), _log(rng, 1, 1000),
                    rng.choice([0, 4, _log(rng, 1, 200)]))
    else:
        n = _log(rng, 2, 400)
        c = _attend("", dtype, _log(rng, 1, 4), heads, group, dim, page, n, n + _log(rng, 1, 5000))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------
# Lengths (of the case alone) and inputs (of the seed)
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case, what, most, least):
    """A length of up to `most` for each sequence; one of them is `most`."""
    r = random.Random("%s %d %d %d" % (what, case["batch"], most, case["dim"] * case["heads"]))
    got = [r.randint(min(most, max(least, most // 4)), most) for _ in range(case["batch"])]
    got[r.randrange(case["batch"])] = most
    return got


def _tokens_and_rows(case):
    """New tokens and rows (theirs included) of each sequence."""
    new = _lengths(case, "new", case["new"], 1)
    if case["op"] == "append":
        return new, [a + b for a, b in zip(new, _lengths(case, "held", case["held"], 0))]
    return new, [max(a, b) for a, b in zip(new, _lengths(case, "rows", case["length"], 1))]


def _first_seen(case, new, rows):
    """The first row behind the sinks that a sequence's new tokens see."""
    return max(0, rows - new - case["window"] + 1) if case["window"] else 0


def _sums(lengths):
    got = [0]
    for n in lengths:
        got.append(got[-1] + n)
    return got


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _device(values, dtype):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _frequencies(rotary):
    """Radians per position of each pair."""
    return [10000.0 ** (-2.0 * i / rotary) for i in range(rotary // 2)]


def _axis_of(case):
    return [a for a, n in enumerate(case["sections"].split("/")) for _ in range(int(n))]


def _positions(gen, axes, tokens, reach):
    """Positions below `reach`: they grow by time or text, and go over a picture's rows and columns on further axes."""
    t = torch.arange(tokens, device="cuda")
    start = int(torch.randint(0, max(1, reach - tokens + 1), (1,), generator=gen, device="cuda"))
    p = [start + t % max(1, reach - start)]
    if axes > 1:
        p.append(start // 2 + t // 31 % 40)
    if axes > 2:
        p.append(start // 2 + t % 31)
    return torch.stack(p).contiguous()


def _tables(case, rows, new, seed):
    """Shuffled pages of a pool with a few to spare; -1 where a sequence has no page, or has given it back."""
    page, r = case["page"], random.Random(seed)
    need, first, last = [], [], []
    for n, m in zip(new, rows):
        kept = list(range((m + page - 1) // page))
        if case["op"] == "attend" and case["window"]:
            a, s = _first_seen(case, n, m), min(case["sinks"], m)
            kept = [i for i in kept if (i + 1) * page > a or i * page < s]
        need.append(kept)
    total = sum(map(len, need))
    pool = list(range(total + 3))
    r.shuffle(pool)
    width = max(1, max((k[-1] + 1 if k else 0) for k in need))
    table = [[-1] * width for _ in rows]
    at = 0
    for b, kept in enumerate(need):
        for i in kept:
            table[b][i] = pool[at]
            at += 1
    return table, total + 3


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, heads, dim, dtype = case["op"], case["heads"], case["dim"], TYPES[case["dtype"]]
    s = {"case": case}
    if op != "attend":
        s["frequency"], s["axis"] = _frequencies(case["rotary"]), _axis_of(case)
        if own:
            from paper_2306_14048_b200 import H2ORotary

            s["rotary"] = H2ORotary(dim, rotary_dim=case["rotary"], frequencies=s["frequency"], axes=s["axis"], pairs=case["pairs"])
    if op == "rotate":
        s["x"] = _normal(gen, (case["tokens"], heads, dim), dtype)
        s["out"] = torch.empty_like(s["x"])
        s["positions"] = _positions(gen, case["axes"], case["tokens"], case["reach"])
        return s
    new, rows = _tokens_and_rows(case)
    tokens, cu = sum(new), _sums(new)
    table, pages = _tables(case, rows, new, seed)
    s["table"], s["length"], s["cu"] = _device(table, torch.int32), _device(rows, torch.int32), _device(cu, torch.int32)
    # keys with a shared direction on a few rows, as attention sinks have it
    u = torch.nn.functional.normalize(torch.randn((heads, dim), generator=gen, device="cuda"), dim=-1)
    pool = torch.randn((pages, case["page"], heads, dim), generator=gen, device="cuda")
    pool += (torch.rand((pages, case["page"], 1, 1), generator=gen, device="cuda") < 0.02) * 4.0 * u
    s["pk"], s["pv"] = pool.to(dtype), _normal(gen, pool.shape, dtype)
    del pool
    hq = heads * case["group"]
    s["q"] = (_normal(gen, (tokens, hq, dim), torch.float32) + 1.5 * u.repeat_interleave(case["group"], 0)).to(dtype)
    s["out"] = torch.empty_like(s["q"])
    if op == "append":
        s["k"], s["v"] = _normal(gen, (tokens, heads, dim), dtype), _normal(gen, (tokens, heads, dim), dtype)
        s["positions"] = _positions(gen, case["axes"], tokens, 4000000) if case["explicit"] else None
    else:
        s["lse"] = torch.empty((tokens, hq), dtype=torch.float32, device="cuda")
    if own:
        from paper_2306_14048_b200 import H2OPages

        s["pages"] = H2OPages(s["pk"], s["pv"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def _turned(s, x, positions, inverse=False):
    """x [tokens, heads, dim] rotated; positions [axes, tokens].  Angles in 64 bits: 32 lose those of far positions."""
    case = s["case"]
    half = case["rotary"] // 2
    angle = positions.double()[s["axis"]].T * torch.tensor(s["frequency"], dtype=torch.float64, device="cuda")
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    if inverse:
        sin = -sin
    y = x.float().clone()
    if case["pairs"] == "halves":
        a, b = y[..., :half].clone(), y[..., half:2 * half].clone()
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., 0:2 * half:2].clone(), y[..., 1:2 * half:2].clone()
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    return y.to(x.dtype)


def _places(s):
    """The sequence and the row of every new token."""
    cu = s["cu"].long()
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, s["length"][b] - cu[b + 1] + t


def _one_sequence(s, b, n, at, rows):
    """Attention of the n tokens from `at` on to `rows` rows of sequence b."""
    case = s["case"]
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    x = torch.arange(rows, device="cuda")
    entry = s["table"][b, x // page].long()
    k, v = (torch.where((entry >= 0)[:, None, None], s[p][entry.clamp(min=0), x % page].float(), 0.0).transpose(0, 1) for p in ("pk", "pv"))
    q = s["q"][at:at + n].float().view(n, heads, group, dim).permute(1, 2, 0, 3).reshape(heads, group * n, dim)
    p = (rows - n + torch.arange(n, device="cuda")).unsqueeze(1)
    seen = x <= p
    if case["window"]:
        seen = seen & ((x < case["sinks"]) | (x > p - case["window"]))
    z = ((q @ k.transpose(1, 2)) * (1.0 / math.sqrt(dim))).view(heads, group, n, rows)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    z = torch.exp(z - top)
    total = z.sum(-1, keepdim=True)
    out = (z.view(heads, group * n, rows) @ v).view(heads, group, n, dim) / total
    s["out"][at:at + n] = out.permute(2, 0, 1, 3).flatten(1, 2).to(s["out"].dtype)
    s["lse"][at:at + n] = (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).flatten(1, 2)


def _all_steps(s, new, rows):
    """Attention of one token of each sequence, all sequences together."""
    case = s["case"]
    heads, group, dim, page, batch = case["heads"], case["group"], case["dim"], case["page"], case["batch"]
    x = torch.arange(max(rows), device="cuda")
    entry = s["table"][:, x // page].long()
    k, v = (s[p][entry.clamp(min=0), x % page].transpose(1, 2) for p in ("pk", "pv"))
    p = s["length"].unsqueeze(1) - 1
    seen = (x <= p) & (entry >= 0)
    if case["window"]:
        seen = seen & ((x < case["sinks"]) | (x > p - case["window"]))
    z = (s["q"].float().view(batch, heads, group, dim) @ k.float().transpose(2, 3)) * (1.0 / math.sqrt(dim))
    z = torch.where(seen[:, None, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    z = torch.exp(z - top)
    total = z.sum(-1, keepdim=True)
    s["out"].copy_(((z @ v.float()) / total).flatten(1, 2))
    s["lse"].copy_((top + torch.log(total)).squeeze(-1).flatten(1, 2))


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "rotate":
        if own:
            s["rotary"].apply(s["x"], s["positions"], s["out"], inverse=case["inverse"])
            return s["out"]
        return _turned(s, s["x"], s["positions"], case["inverse"])
    many = {} if case["new"] == 1 else {"cu": s["cu"]}
    if op == "append":
        if own:
            s["pages"].append(s["k"], s["v"], s["table"], s["length"], rotary=s["rotary"], positions=s["positions"], q=s["q"], q_out=s["out"], **many)
            return s["pk"], s["pv"], s["out"]
        b, row = _places(s)
        positions = s["positions"] if case["explicit"] else row.expand(case["axes"], -1)
        entry = s["table"][b, row // case["page"]].long()
        s["pk"][entry, row % case["page"]] = _turned(s, s["k"], positions)
        s["pv"][entry, row % case["page"]] = s["v"]
        s["out"].copy_(_turned(s, s["q"], positions))
        return s["pk"], s["pv"], s["out"]
    if own:
        if many:
            many["max_q"] = case["new"]
        s["pages"].attend(s["q"], s["table"], s["length"], s["out"], max_len=case["length"], window=case["window"], sinks=case["sinks"],
                          lse=s["lse"], **many)
        return s["out"], s["lse"]
    new, rows = _tokens_and_rows(case)
    if case["new"] == 1:
        _all_steps(s, new, rows)
    else:
        for b, at in enumerate(_sums(new)[:-1]):
            _one_sequence(s, b, new[b], at, rows[b])
    return s["out"], s["lse"]


# ---------------------------------------------------------------------------------------------------------------
# What one pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    heads, dim, wide = case["heads"], case["dim"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotate":
        return {"bytes": case["tokens"] * (2 * heads * dim * wide + 8 * case["axes"]), "flops": 0}
    hq = heads * case["group"]
    new, rows = _tokens_and_rows(case)
    tokens = sum(new)
    if case["op"] == "append":
        return {"bytes": tokens * (2 * (2 * heads + hq) * dim * wide + (8 * case["axes"] if case["explicit"] else 0)), "flops": 0}
    pairs = seen = 0
    for n, m in zip(new, rows):
        a, s = _first_seen(case, n, m), case["sinks"]
        seen += m - max(0, a - s)  # rows that some query sees
        for p in range(m - n, m):
            pairs += p + 1 - (max(0, p - case["window"] + 1 - s) if case["window"] else 0)
    return {"bytes": 2 * seen * heads * dim * wide + tokens * hq * (2 * dim * wide + 4), "flops": 4 * pairs * hq * dim}


def _exact_turn(case, x, positions, inverse=False):
    """The rotation as a product of complex numbers, one pair of channels at a time."""
    x = x.double()
    y, half = x.clone(), case["rotary"] // 2
    axis, frequency = _axis_of(case), _frequencies(case["rotary"])
    for i in range(half):
        a, b = (i, i + half) if case["pairs"] == "halves" else (2 * i, 2 * i + 1)
        angle = positions[axis[i]].double() * frequency[i]
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), -angle if inverse else angle).unsqueeze(1)
        y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotate":
        return _exact_turn(case, s["x"], s["positions"], case["inverse"])
    new, rows = _tokens_and_rows(case)
    cu, page = _sums(new), case["page"]
    if op == "append":
        pk, pv = s["pk"].double(), s["pv"].double()
        positions = s["positions"]
        if positions is None:
            positions = _device([[m - n + i for n, m in zip(new, rows) for i in range(n)]] * case["axes"], torch.int64)
        k, v = _exact_turn(case, s["k"], positions), s["v"].double()
        table = s["table"].tolist()
        for b, (n, m) in enumerate(zip(new, rows)):
            x = m - n
            while x < m:  # page by page
                end = min(m, (x // page + 1) * page)
                to, at = table[b][x // page], cu[b] + x - (m - n)
                pk[to, x % page:x % page + end - x] = k[at:at + end - x]
                pv[to, x % page:x % page + end - x] = v[at:at + end - x]
                x = end
        return pk, pv, _exact_turn(case, s["q"], positions)
    heads, group, dim = case["heads"], case["group"], case["dim"]
    q = s["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(zip(new, rows)):
        # the rows that some query sees, in order
        first = _first_seen(case, n, m)
        x = torch.tensor([i for i in range(m) if i >= first or i < case["sinks"]], device="cuda")
        at = s["table"][b].long()[x // page] * page + x % page
        k, v = (s[p].flatten(0, 1)[at].double() for p in ("pk", "pv"))
        p = torch.arange(m - n, m, device="cuda").unsqueeze(1)
        hidden = x > p
        if case["window"]:
            hidden |= (x >= case["sinks"]) & (p - x >= case["window"])
        for h in range(heads * group):
            z = (q[cu[b]:cu[b] + n, h] @ k[:, h // group].T / math.sqrt(dim)).masked_fill(hidden, -math.inf)
            lse[cu[b]:cu[b] + n, h] = torch.logsumexp(z, -1)
            out[cu[b]:cu[b] + n, h] = torch.softmax(z, -1) @ v[:, h // group]
    return out, lse
