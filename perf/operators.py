"""Operators on a K/V store that many queries read: cases, inputs, plain forms and the framework's calls.

A *store* holds K and V rows that are written once and read often: an encoder's states, a prompt that a whole
batch shares, a sequence's own tokens.  Its rows are float32 or bfloat16 ([rows, heads, dim]), or 8-bit floating
point ("kv8": codes [heads, rows, dim] in e4m3 and one power of two for each row and head).  Operators:

  write   quantise rows as they are written into an 8-bit store
  read    read rows of an 8-bit store back
  cross   attention of each sequence's queries to that sequence's range of the store (no causal mask)
  prefix  attention of a batch whose groups of sequences share a long prefix, computed once for all, and whose
          sequences have rows of their own (causal, the last query sees all of them)

`run` computes an operator in elementary torch operations, or, where `own` is true, with the framework's calls.
"""
import math
import random

import torch

own = False

FORMATS = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _write(name, tokens, heads, dim, dtype="bf16", rows=0):
    return {"name": name, "op": "write", "tokens": tokens, "heads": heads, "dim": dim, "dtype": dtype, "rows": rows or 2 * tokens}


def _read(name, tokens, heads, dim, dtype="bf16", rows=0):
    return {"name": name, "op": "read", "tokens": tokens, "heads": heads, "dim": dim, "dtype": dtype, "rows": rows or 2 * tokens}


def _cross(name, fmt, batch, heads, group, dim, max_q, max_kv, ragged=True):
    return {"name": name, "op": "cross", "fmt": fmt, "batch": batch, "heads": heads, "group": group, "dim": dim,
            "max_q": max_q, "max_kv": max_kv, "ragged": ragged}


def _prefix(name, fmt, batch, groups, heads, group, dim, max_q, prefix, max_own):
    return {"name": name, "op": "prefix", "fmt": fmt, "batch": batch, "groups": groups, "heads": heads, "group": group,
            "dim": dim, "max_q": max_q, "prefix": prefix, "max_own": max_own, "ragged": True}


def listed():
    return [
        # the new token of each of 64 sequences enters an 8-bit store: one such call for each layer and token
        _write("write step", 64, 32, 128, rows=8192),
        # a batch of prompts, 16391 tokens in all, enters the store at once
        _write("write prompts", 16391, 32, 128),
        # scattered rows of a store back in bfloat16, as for moving a sequence to a store of another format
        _read("read rows", 5003, 32, 128),
        # decoder prompts of up to 512 tokens against encoder states of up to 2048, both ragged
        _cross("cross prompts", "bf16", 8, 32, 1, 128, 512, 2048),
        # the largest: four decoder prompts of 2048 tokens against 4096 encoder states each
        _cross("cross long", "bf16", 4, 32, 1, 128, 2048, 4096, ragged=False),
        # a small float32 model, odd sizes, heads of 64
        _cross("cross float32", "f32", 2, 8, 1, 64, 131, 515),
        # one token of each of 64 sequences against its encoder states: every layer, every token
        _cross("cross step", "bf16", 64, 32, 1, 128, 1, 2048),
        # the same from an 8-bit store with four query heads to a K/V head
        _cross("cross step 8-bit", "kv8", 32, 8, 4, 128, 1, 4096),
        # 64 samples drawn from one prompt of 8192 tokens, one token each
        _prefix("prefix step", "bf16", 64, 1, 32, 1, 128, 1, 8192, 512),
        # 16 sequences on a document of 32768 tokens in an 8-bit store, grouped heads
        _prefix("prefix step 8-bit", "kv8", 16, 1, 8, 4, 128, 1, 32768, 1024),
        # a handful of short sequences with a short instruction: latency is all
        _prefix("prefix step small", "bf16", 4, 1, 8, 1, 64, 1, 1000, 100),
        # user prompts of up to 200 tokens behind one of two shared instructions of up to 4096
        _prefix("prefix prompts", "bf16", 32, 2, 32, 1, 128, 200, 4096, 200),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["write", "read", "cross step", "cross prompts", "prefix step", "prefix prompts"])
    dim = rng.choice([64, 128, 128])
    if op in ("write", "read"):
        tokens, heads = _log(rng, 1, 16000), _log(rng, 1, 32)
        c = (_write if op == "write" else _read)("", tokens, heads, dim, rng.choice(["bf16", "bf16", "f32"]), tokens + _log(rng, 1, 16000))
    else:
        fmt = rng.choice(["bf16", "bf16", "kv8", "kv8", "f32"])
        group = rng.choice([1, 1, 2, 4, 8])
        heads = _log(rng, 1, 32 // group)
        if op == "cross step":
            c = _cross("", fmt, _log(rng, 1, 64), heads, group, dim, 1, _log(rng, 1, 4096))
        elif op == "cross prompts":
            c = _cross("", fmt, _log(rng, 1, 8), heads, group, dim, _log(rng, 2, 512), _log(rng, 1, 4096))
        else:
            batch = _log(rng, 1, 64)
            groups = rng.choice([1, 1, 2, 5])
            q = 1 if op == "prefix step" else _log(rng, 2, 200)
            c = _prefix("", fmt, batch, min(batch, groups), heads, group, dim, q, _log(rng, 1, 16384 if q == 1 else 4096),
                        q + _log(rng, 1, 512) - 1)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------
# Lengths (of the case alone) and inputs (of the seed)
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case, what, count, most, least=1):
    """`count` lengths of up to `most`; one of them is `most`."""
    if not case.get("ragged"):
        return [most] * count
    r = random.Random("%s %d %d %d" % (what, count, most, case["dim"] * case["heads"]))
    got = [r.randint(min(most, max(least, most // 4)), most) for _ in range(count)]
    got[r.randrange(count)] = most
    return got


def _sums(lengths):
    got = [0]
    for n in lengths:
        got.append(got[-1] + n)
    return got


def _cross_lengths(case):
    q = _lengths(case, "q", case["batch"], case["max_q"])
    return q, _lengths(case, "kv", case["batch"], case["max_kv"])


def _prefix_lengths(case):
    """Query tokens and own rows of each sequence, sequences of each group, length of each prefix."""
    batch, groups = case["batch"], case["groups"]
    q = _lengths(case, "q", batch, case["max_q"])
    mine = [max(a, b) for a, b in zip(q, _lengths(case, "own", batch, case["max_own"]))]
    members = [batch // groups + (1 if g < batch % groups else 0) for g in range(groups)]
    return q, mine, members, _lengths(case, "prefix", groups, case["prefix"])


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _keys_values(gen, rows, heads, dim, dtype):
    """K with a shared direction on a few rows, as attention sinks have it, and V; and the direction of each head."""
    u = torch.nn.functional.normalize(torch.randn((heads, dim), generator=gen, device="cuda"), dim=-1)
    k = torch.randn((rows, heads, dim), generator=gen, device="cuda")
    k += (torch.rand((rows, 1, 1), generator=gen, device="cuda") < 0.02) * 4.0 * u
    return k.to(dtype), _normal(gen, (rows, heads, dim), dtype), u


def _exponents(x):
    """The power of two of each row and head: the smallest e with max |x| <= 448 * 2^e, within [-15, 7]."""
    big = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(big)  # big = m * 2^e, m in [0.5, 1)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(big > 0, e, -15).clamp(-15, 7)


def _power(e):
    """2^e in float32, from its bits: exact, which pow() does not promise."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """[tokens, heads, dim] -> e4m3 codes [heads, tokens, dim], exponents + 127 [heads, tokens], both as bytes."""
    x = x.float().transpose(0, 1)
    e = _exponents(x)
    y = (x * _power(-e).unsqueeze(-1)).clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scale):
    """The float32 values that codes [heads, ..., dim] and scale [heads, ...] stand for."""
    return codes.view(torch.float8_e4m3fn).float() * _power(scale.int() - 127).unsqueeze(-1)


def _device(values, dtype):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _spread(lengths, at, gen_seed):
    """First rows of ranges of these lengths, in a shuffled order from row `at` on, with a gap before each; and the end."""
    r = random.Random(gen_seed)
    order = list(range(len(lengths)))
    r.shuffle(order)
    begin = [0] * len(lengths)
    for i in order:
        at += r.randrange(4)
        begin[i] = at
        at += lengths[i]
    return begin, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, heads, dim = case["op"], case["heads"], case["dim"]
    s = {"case": case}
    if op in ("write", "read"):
        n, rows, dtype = case["tokens"], case["rows"], FORMATS[case["dtype"]]
        s["rows"] = torch.randperm(rows, generator=gen, device="cuda")[:n].contiguous()
        held = rows if op == "read" else 0
        k, v, _ = _keys_values(gen, held or n, heads, dim, dtype)
        s["sk"], s["sk_scale"] = (torch.zeros((heads, rows, dim), dtype=torch.uint8, device="cuda"),
                                  torch.full((heads, rows), 127, dtype=torch.uint8, device="cuda"))
        s["sv"], s["sv_scale"] = s["sk"].clone(), s["sk_scale"].clone()
        if held:
            (s["sk"], s["sk_scale"]), (s["sv"], s["sv_scale"]) = (tuple(t.contiguous() for t in _quantise(x)) for x in (k, v))
            s["k"], s["v"] = (torch.empty((n, heads, dim), dtype=dtype, device="cuda") for _ in range(2))
        else:
            s["k"], s["v"] = k, v
    else:
        dtype = FORMATS.get(case["fmt"], torch.bfloat16)
        group = case["group"]
        if op == "cross":
            q_len, kv_len = _cross_lengths(case)
            begin, rows = _spread(kv_len, 0, seed)
            s["begin"], s["length"] = _device(begin, torch.int64), _device(kv_len, torch.int32)
        else:
            q_len, own_len, members, prefix_len = _prefix_lengths(case)
            begin, rows = _spread(prefix_len, 0, seed)
            own_begin, rows = _spread(own_len, rows, seed + 1)
            s["prefix_begin"], s["prefix_len"] = _device(begin, torch.int64), _device(prefix_len, torch.int32)
            s["own_begin"], s["own_len"] = _device(own_begin, torch.int64), _device(own_len, torch.int32)
            s["cu_group"] = _device(_sums(members), torch.int32)
            s["max_group"] = max(members)
        s["cu_q"] = _device(_sums(q_len), torch.int32)
        tokens = sum(q_len)
        k, v, u = _keys_values(gen, rows, heads, dim, dtype)
        s["sk"], s["sv"] = k, v
        if case["fmt"] == "kv8":
            (s["sk"], s["sk_scale"]), (s["sv"], s["sv_scale"]) = (tuple(t.contiguous() for t in _quantise(x)) for x in (k, v))
        s["q"] = (_normal(gen, (tokens, heads * group, dim), torch.float32) + 1.5 * u.repeat_interleave(group, 0)).to(dtype)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((tokens, heads * group), dtype=torch.float32, device="cuda")
    if own:
        from paper_2306_14048_b200 import H2OStore

        s["store"] = H2OStore(s["sk"], s["sv"], s.get("sk_scale"), s.get("sv_scale"))
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def _ranges(begin, length, most):
    """Row indexes [count, most] of ranges, and which of them there are (the others are 0)."""
    i = torch.arange(most, device="cuda")
    there = i < length.unsqueeze(1)
    return torch.where(there, begin.unsqueeze(1) + i, 0), there


def _stored(s, index):
    """K and V of store rows `index` [count, most] in float32, [count, heads, most, dim]."""
    if s["case"]["fmt"] == "kv8":
        return tuple(_values(s[x][:, index], s[x + "_scale"][:, index]).transpose(0, 1) for x in ("sk", "sv"))
    return tuple(s[x][index].float().transpose(1, 2) for x in ("sk", "sv"))


def _part(s, q_index, begin, length, most, limit):
    """Attention of the query tokens q_index [count, queries] to ranges of the store: maximum, sum and weighted values,
    each [count, heads, queries, group(, dim)].  limit [count, queries]: rows of its range that a query sees."""
    case = s["case"]
    heads, group, dim = case["heads"], case["group"], case["dim"]
    count, queries = q_index.shape
    index, there = _ranges(begin, length, most)
    k, v = _stored(s, index)
    v = torch.where(there[:, None, :, None], v, 0.0)
    q = s["q"][q_index].float().view(count, queries, heads, group, dim).transpose(1, 2).reshape(count, heads, queries * group, dim)
    x = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(dim))
    seen = (torch.arange(most, device="cuda") < limit.unsqueeze(2)).repeat_interleave(group, 1)
    x = torch.where(seen.unsqueeze(1), x, -math.inf)
    top = x.amax(-1)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top).unsqueeze(-1))
    shape = (count, heads, queries, group)
    return top.view(shape), p.sum(-1).view(shape), (p @ v).view(shape + (dim,))


def _of_tokens(s, part, cu, most):
    """A part's results in the order of the query tokens: [tokens, heads * group(, dim)].  cu: first token of each range."""
    t = torch.arange(s["q"].shape[0], device="cuda")
    which = torch.searchsorted(cu, t, right=True) - 1
    local = t - cu[which]
    return tuple(x[which, :, local].flatten(1, 2) for x in part)


def _joined(parts, dtype):
    """Output and log of the sum of exponentials, from the parts of the keys."""
    top = torch.stack([p[0] for p in parts]).amax(0)
    base = torch.where(top == -math.inf, 0.0, top)
    total, value = 0.0, 0.0
    share = [torch.exp(p[0] - base) for p in parts]
    total = sum(a * p[1] for a, p in zip(share, parts))
    value = sum(a.unsqueeze(-1) * p[2] for a, p in zip(share, parts))
    out = torch.where(total.unsqueeze(-1) > 0, value / total.unsqueeze(-1), 0.0)
    return out.to(dtype), base + torch.log(total)


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "write":
        if own:
            s["store"].write(s["k"], s["v"], rows=s["rows"])
        else:
            for x, to in ((s["k"], "sk"), (s["v"], "sv")):
                codes, scale = _quantise(x)
                s[to].index_copy_(1, s["rows"], codes)
                s[to + "_scale"].index_copy_(1, s["rows"], scale)
        return {x: s[x].view(torch.float8_e4m3fn) for x in ("sk", "sv")} | {x: s[x] for x in ("sk_scale", "sv_scale")}
    if op == "read":
        if own:
            s["store"].read(s["k"], s["v"], rows=s["rows"])
            return s["k"], s["v"]
        return tuple(_values(s[x][:, s["rows"]], s[x + "_scale"][:, s["rows"]]).transpose(0, 1).to(s["k"].dtype).contiguous()
                     for x in ("sk", "sv"))
    many = {} if case["max_q"] == 1 else {"cu_q": s["cu_q"], "max_q": case["max_q"]}
    if op == "cross":
        if own:
            s["store"].cross_attend(s["q"], s["begin"], s["length"], s["out"], max_len=case["max_kv"], lse=s["lse"], **many)
            return s["out"], s["lse"]
        index, _ = _ranges(s["cu_q"][:-1], s["cu_q"].diff(), case["max_q"])
        part = _part(s, index, s["begin"], s["length"], case["max_kv"], s["length"].unsqueeze(1).expand(-1, case["max_q"]))
        return _joined([_of_tokens(s, part, s["cu_q"], case["max_q"])], s["q"].dtype)
    if own:
        s["store"].prefix_attend(s["q"], s["prefix_begin"], s["prefix_len"], s["own_begin"], s["own_len"], s["out"],
                                 max_prefix=case["prefix"], max_own=case["max_own"], cu_group=s["cu_group"],
                                 max_group=s["max_group"], lse=s["lse"], **many)
        return s["out"], s["lse"]
    # the prefix: all the query tokens of a group together
    cu = s["cu_q"][s["cu_group"]]
    most = s["max_group"] * case["max_q"]
    index, _ = _ranges(cu[:-1], cu.diff(), most)
    shared = _part(s, index, s["prefix_begin"], s["prefix_len"], case["prefix"], s["prefix_len"].unsqueeze(1).expand(-1, most))
    # a sequence's own rows: query i of n sees all but the last n - 1 - i
    n = s["cu_q"].diff()
    index, _ = _ranges(s["cu_q"][:-1], n, case["max_q"])
    limit = (s["own_len"] - n).unsqueeze(1) + 1 + torch.arange(case["max_q"], device="cuda")
    mine = _part(s, index, s["own_begin"], s["own_len"], case["max_own"], torch.minimum(limit, s["own_len"].unsqueeze(1)))
    return _joined([_of_tokens(s, shared, cu, most), _of_tokens(s, mine, s["cu_q"], case["max_q"])], s["q"].dtype)


# ---------------------------------------------------------------------------------------------------------------
# What one pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    heads, dim, op = case["heads"], case["dim"], case["op"]
    if op in ("write", "read"):
        wide = 4 if case["dtype"] == "f32" else 2
        # the row's values, its codes and its scale, of K and of V, and the row's index
        return {"bytes": case["tokens"] * (2 * heads * (dim * (wide + 1) + 1) + 8), "flops": 0}
    group = case["group"]
    wide = 4 if case["fmt"] == "f32" else 2
    row = 2 * heads * ((dim + 1) if case["fmt"] == "kv8" else dim * wide)
    if op == "cross":
        q_len, kv_len = _cross_lengths(case)
        rows, pairs = sum(kv_len), sum(a * b for a, b in zip(q_len, kv_len))
    else:
        q_len, own_len, members, prefix_len = _prefix_lengths(case)
        rows = sum(prefix_len) + sum(own_len)
        cu, pairs = _sums(members), 0
        for g, n in enumerate(prefix_len):
            pairs += n * sum(q_len[cu[g]:cu[g + 1]])
        pairs += sum(n * m - n * (n - 1) // 2 for n, m in zip(q_len, own_len))
    return {"bytes": rows * row + sum(q_len) * heads * group * (2 * dim * wide + 4), "flops": 4 * pairs * heads * group * dim}


def _two_to(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x):
    """Quantised rows [tokens, heads, dim] by the definition: scale 2^e, value rounded to 4 significant bits, ties to even."""
    x = x.double().transpose(0, 1)
    big = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(big, -15.0)
    for power in range(-15, 7):  # the smallest power of two that holds the row
        e = torch.where(big > 448.0 * 2.0 ** power, float(power + 1), e)
    y = x / _two_to(e)
    step = _two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 1 - 3)  # 8 to 15 steps to a value; fewer below 2^-6
    return (torch.round(y / step) * step).clamp(-448.0, 448.0), (e + 127).squeeze(-1)


def _exact_rows(s, name, first, count):
    """Rows first .. first + count of the store in 64 bits, [heads, count, dim]."""
    x = s[name]
    if s["case"].get("fmt", "kv8") != "kv8":
        return x[first:first + count].double().transpose(0, 1)
    b = x[:, first:first + count].int()
    mantissa, exponent = b & 7, (b >> 3) & 15
    value = torch.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * _two_to(exponent - 10))
    value = torch.where(b >= 128, -value, value)
    return value * _two_to(s[name + "_scale"][:, first:first + count].int() - 127).unsqueeze(-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "write":
        got = {x: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in ("sk", "sv")}
        for x in ("sk", "sv"):
            codes, scale = _exact_codes(s["k" if x == "sk" else "v"])
            got[x][:, s["rows"]] = codes
            got[x + "_scale"] = s[x + "_scale"].clone()
            got[x + "_scale"][:, s["rows"]] = scale.to(torch.uint8)
        return got
    if op == "read":
        return tuple(_exact_rows(s, x, 0, case["rows"])[:, s["rows"]].transpose(0, 1) for x in ("sk", "sv"))
    heads, group, dim = case["heads"], case["group"], case["dim"]
    q = s["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    q_len = _cross_lengths(case)[0] if op == "cross" else _prefix_lengths(case)[0]
    cu, group_of = _sums(q_len), []
    if op == "prefix":
        for g, n in enumerate(_prefix_lengths(case)[2]):
            group_of += [g] * n
    for b in range(case["batch"]):
        n, at = q_len[b], cu[b]
        if op == "cross":
            parts = [(int(s["begin"][b]), int(s["length"][b]))]
            hidden = 0
        else:
            g = group_of[b]
            parts = [(int(s["prefix_begin"][g]), int(s["prefix_len"][g])), (int(s["own_begin"][b]), int(s["own_len"][b]))]
            hidden = n - 1
        k, v = (torch.cat([_exact_rows(s, x, *p) for p in parts], 1) for x in ("sk", "sv"))
        total = k.shape[1]
        i, j = torch.arange(n, device="cuda"), torch.arange(total, device="cuda")
        masked = (j >= (total - hidden + i).unsqueeze(1)) if hidden else None
        for h in range(heads):
            for r in range(group):
                x = q[at:at + n, h * group + r] @ k[h].T / math.sqrt(dim)
                if masked is not None:
                    x = x.masked_fill(masked, -math.inf)
                lse[at:at + n, h * group + r] = torch.logsumexp(x, -1)
                out[at:at + n, h * group + r] = torch.softmax(x, -1) @ v[h]
    return out, lse
