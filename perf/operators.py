"""Cases of the operators that score a member: its keys and values appended to
a paged cache, read back, and attended to.

A program that scores the members of a population runs prompts and then single
tokens through the weights between two moves of the parameters.  Two kinds of
calls are measured here:

    place    queries and keys normalised for each head and rotated by position,
             keys and values stored in the cache (bf16, int8 or E4M3 with a
             scale for each token and head), and the stored rows read back
    attend   attention over the cache, for one or a few rows of each sequence
             ("step") and for whole prompts ("prompt")

Head layouts are those of the package's parameter sets (40 query heads over 8,
32 over 8 and 16 over 16) and one with wide heads.

    own                   False: the plain form; True: the package's kernels
    listed()              the fixed cases
    draw(rng)             one more case of the same ranges
    prepare(case, seed)   what a program has in hand before the call
    run(state)            one pass; returns its outputs
    work(case)            bytes and operations a pass cannot do without
    exact(case, seed)     the outputs from the definition, in 64 bits
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6                     # of the norms
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100             # rows below this are stored as zeros
SCORES_MAX = 2.68e9            # of a case, padded: the longest prompt's
FLOPS_MAX = 6.8e11             # of a case: the longest prompt's


# ---------------------------------------------------------------- the cases --

def _heads(q_heads, kv_heads, dim):
    return {"q_heads": q_heads, "kv_heads": kv_heads, "dim": dim}


WIDE_MODEL = _heads(40, 8, 128)
MID_MODEL = _heads(32, 8, 128)
SMALL_MODEL = _heads(16, 16, 64)
WIDE_HEADS = _heads(16, 4, 256)


def listed():
    return [
        # one token of one rollout: latency is all there is
        dict(WIDE_MODEL, name="place one token", op="place", format="e4m3", page=64,
             seqs=1, longest=1, shortest=1, rot=128, adjacent=False, context=1900),
        # one token of each of a generation step's 32 tasks, half of each head rotated
        dict(MID_MODEL, name="place 32 tokens", op="place", format="int8", page=128,
             seqs=32, longest=1, shortest=1, rot=64, adjacent=False, context=4001),
        # the prompts of 32 tasks, packed without padding
        dict(WIDE_MODEL, name="place 32 prompts", op="place", format="e4m3", page=64,
             seqs=32, longest=1021, shortest=19, rot=128, adjacent=False, context=0),
        # one long document through narrow heads, kept as it is
        dict(SMALL_MODEL, name="place a document", op="place", format="bf16", page=256,
             seqs=1, longest=32771, shortest=32771, rot=64, adjacent=True, context=0),
        # the next token of a single short rollout
        dict(MID_MODEL, name="step 1 short", op="attend", format="bf16", page=64, seqs=1,
             longest=777, shortest=777, rows=1, mask="causal", cap=0.0, slopes=False),
        # the next token of 32 tasks whose histories differ widely
        dict(WIDE_MODEL, name="step 32 ragged", op="attend", format="e4m3", page=64, seqs=32,
             longest=16384, shortest=201, rows=1, mask="causal", cap=0.0, slopes=False),
        # long-horizon histories, capped scores
        dict(MID_MODEL, name="step 8 long", op="attend", format="int8", page=128, seqs=8,
             longest=65537, shortest=49999, rows=1, mask="causal", cap=50.0, slopes=False),
        # four rows of each task at once (an observation's few tokens), bias by distance
        dict(WIDE_MODEL, name="step 16 of 4 rows", op="attend", format="bf16", page=64, seqs=16,
             longest=4099, shortest=1023, rows=4, mask="causal", cap=0.0, slopes=True),
        # a short prompt of the narrow-headed model
        dict(SMALL_MODEL, name="prompt 517", op="attend", format="bf16", page=64, seqs=1,
             longest=517, shortest=517, rows=517, mask="causal", cap=0.0, slopes=False),
        # documents packed into one sequence, each with a prefix its rows all see
        dict(MID_MODEL, name="prompt of documents", op="attend", format="e4m3", page=64, seqs=1,
             longest=6001, shortest=6001, rows=6001, mask="documents", cap=30.0, slopes=False),
        # the prompts of 16 tasks, bias by distance
        dict(WIDE_MODEL, name="prompts ragged", op="attend", format="int8", page=128, seqs=16,
             longest=2039, shortest=65, rows=2039, mask="causal", cap=0.0, slopes=True),
        # the longest prompt
        dict(WIDE_MODEL, name="prompt 8192", op="attend", format="bf16", page=64, seqs=1,
             longest=8192, shortest=8192, rows=8192, mask="causal", cap=0.0, slopes=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = dict(rng.choice([WIDE_MODEL, MID_MODEL, SMALL_MODEL, WIDE_HEADS]))
    case["format"] = rng.choice(["bf16", "int8", "e4m3"])
    case["page"] = rng.choice([64, 128, 256])
    kind = rng.choice(["place", "step", "step", "prompt", "prompt"])
    if kind == "place":
        tokens = _log_int(rng, 1, 16000)
        seqs = _log_int(rng, 1, min(64, tokens))
        longest = max(1, tokens // seqs)
        case.update(op="place", seqs=seqs, longest=longest, shortest=_log_int(rng, 1, longest),
                    rot=rng.choice([case["dim"], case["dim"] // 2]),
                    adjacent=rng.choice([False, True]),
                    context=rng.choice([0, _log_int(rng, 1, 9000)]))
        return case
    case.update(op="attend", mask=rng.choice(["causal", "causal", "window", "documents"]),
                cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.choice([False, False, True]))
    if kind == "step":
        seqs = _log_int(rng, 1, 64)
        longest = _log_int(rng, 1, 230000 // seqs)
        case.update(seqs=seqs, longest=longest, shortest=_log_int(rng, 1, longest),
                    rows=min(longest, rng.choice([1, 1, 1, 2, 3, 5, 8])))
    else:
        rows = _log_int(rng, 9, 6000)
        seqs = _log_int(rng, 1, max(1, min(24, 12000 // rows)))
        longest = rows if rng.random() < 0.6 else min(24000, rows + _log_int(rng, 1, 12000))
        case.update(seqs=seqs, longest=longest, shortest=_log_int(rng, max(1, longest // 20), longest),
                    rows=rows)
        while _scores(case) > SCORES_MAX or work(case)["flops"] > FLOPS_MAX:
            if case["seqs"] > 1:
                case["seqs"] -= 1
            else:
                case["longest"] = int(0.9 * case["longest"])
                case["shortest"] = min(case["shortest"], case["longest"])
    return case


def _lengths(case):
    """The sequences' lengths: from the longest to the shortest in equal ratios."""
    n, hi, lo = case["seqs"], case["longest"], case["shortest"]
    if n == 1:
        return [hi]
    return [max(1, int(round(hi * (lo / hi) ** (i / (n - 1))))) for i in range(n)]


def _scores(case):
    """The scores of a case: every row of every query head against every key, padded."""
    return case["q_heads"] * case["seqs"] * min(case["rows"], case["longest"]) * case["longest"]


def _rows(case):
    return [min(case["rows"], n) for n in _lengths(case)]


def _intervals(case):
    """For each row of each sequence: its position, and the keys [first, limit) that it sees.

    documents: of 1, 2, 3 ... 9 parts in turn of length // 12, the last one
    whatever is left; the first fifth of each is a prefix that all of its rows see.
    window: the last 1000 keys."""
    out = []
    for length, n in zip(_lengths(case), _rows(case)):
        pos = np.arange(length - n, length, dtype=np.int64)
        first, limit = np.zeros_like(pos), pos + 1
        if case["mask"] == "window":
            first = np.maximum(0, pos - 999)
        elif case["mask"] == "documents":
            unit = max(1, length // 12)
            starts, at, k = [], 0, 1
            while at < length:
                starts.append(at)
                at += unit * k
                k = k % 9 + 1
            starts = np.array(starts, dtype=np.int64)
            ends = np.append(starts[1:], length)
            doc = np.searchsorted(starts, pos, side="right") - 1
            first = starts[doc]
            limit = np.maximum(limit, first + (ends[doc] - first) // 5)
        out.append((pos, first, limit))
    return out


# --------------------------------------------------------------- the inputs --

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _ints(values, dtype=torch.int32):
    return torch.tensor(np.asarray(values, dtype=np.int64), dtype=dtype, device="cuda")


def _quantise(x, form):
    """Codes and scales of the rows of x (float32, the last dimension a row)."""
    if form == "bf16":
        return x.to(torch.bfloat16), None
    top = x.abs().amax(-1, keepdim=True)
    live = top >= TINY
    inv = torch.where(live, CODE_MAX[form] / top, torch.zeros_like(top))
    scale = torch.where(live, top / CODE_MAX[form], torch.zeros_like(top))
    y = x * inv
    y = y.round().to(torch.int8) if form == "int8" else y.to(torch.float8_e4m3fn)
    return y, scale.squeeze(-1)


def _raw(t):
    """The cache's bytes, where indexing knows no 8-bit floats."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _value(codes, like):
    return (codes.view(torch.float8_e4m3fn) if like.dtype == torch.float8_e4m3fn
            else codes).float()


def _cache(case, gen, pages, fill):
    """A cache of `pages` pages: keys [pages, heads, page, dim], values
    [pages, heads, dim, page] and their scales [pages, heads, page]."""
    h, p, d, form = case["kv_heads"], case["page"], case["dim"], case["format"]
    if fill:
        k, ks = _quantise(_normal(gen, pages, h, p, d), form)
        v, vs = _quantise(_normal(gen, pages, h, p, d), form)
        return k, _raw(v).transpose(2, 3).contiguous().view(v.dtype), ks, vs
    dt = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[form]
    k = torch.zeros(pages, h, p, d, dtype=torch.uint8, device="cuda").to(dt)
    v = torch.zeros(pages, h, d, p, dtype=torch.uint8, device="cuda").to(dt)
    scales = [None if form == "bf16" else torch.zeros(pages, h, p, device="cuda")
              for _ in range(2)]
    return k, v, scales[0], scales[1]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = np.random.default_rng(seed)
    hq, h, d, p = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    lengths = _lengths(case)
    before = case.get("context", 0) if case["op"] == "place" else 0
    per_seq = [-(-(n + before) // p) for n in lengths]
    pages = sum(per_seq) + 3
    order = host.permutation(pages)
    table = np.zeros((len(lengths), max(per_seq)), dtype=np.int64)
    at = 0
    for s, n in enumerate(per_seq):
        table[s, :n] = order[at:at + n]
        at += n
    c = {"case": case}
    c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"] = _cache(
        case, gen, pages, case["op"] == "attend")
    if case["op"] == "place":
        tokens = sum(lengths)
        # the packed projections of queries, keys and values
        qkv = (_normal(gen, tokens, (hq + 2 * h) * d) * 1.5).to(torch.bfloat16)
        c["q"] = qkv[:, :hq * d].view(tokens, hq, d)
        c["k"] = qkv[:, hq * d:(hq + h) * d].view(tokens, h, d)
        c["v"] = qkv[:, (hq + h) * d:].view(tokens, h, d)
        c["q_gain"] = (1 + 0.1 * _normal(gen, d)).to(torch.bfloat16)
        c["k_gain"] = (1 + 0.1 * _normal(gen, d)).to(torch.bfloat16)
        pos = np.concatenate([np.arange(before, before + n) for n in lengths])
        seq = np.repeat(np.arange(len(lengths)), lengths)
        c["positions"] = _ints(pos)
        c["slots"] = _ints(table[seq, pos // p] * p + pos % p, torch.int64)
        r = case["rot"]
        angle = np.arange(max(lengths) + before)[:, None] * 10000.0 ** (-np.arange(r // 2) * 2 / r)
        c["rope"] = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
        return c
    rows = _rows(case)
    iv = _intervals(case)
    c["q"] = (_normal(gen, sum(rows), hq, d) * 1.5).to(torch.bfloat16)
    c["tables"] = _ints(table)
    c["lengths"] = _ints(lengths)
    c["starts"] = _ints(np.concatenate([[0], np.cumsum(rows)]))
    c["max_rows"], c["max_length"] = max(rows), max(lengths)
    plain = case["mask"] == "causal"
    c["first"] = None if plain else _ints(np.concatenate([f for _, f, _ in iv]))
    c["limit"] = None if plain else _ints(np.concatenate([m for _, _, m in iv]))
    c["scale"], c["cap"] = d ** -0.5, case["cap"]
    c["slopes"] = None
    if case["slopes"]:
        c["slopes"] = torch.from_numpy(2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).float().cuda()
    return c


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        from paper_2608_17310_amd.kvcache import KVCache
        state["cache"] = KVCache(state["k_pages"], state["v_pages"], state["k_scales"],
                                 state["v_scales"])
    return state


# ------------------------------------------------------------------ running --

def run(state):
    place = state["case"]["op"] == "place"
    if own:
        return _own_place(state) if place else _own_attend(state)
    return _plain_place(state) if place else _plain_attend(state)


def _own_place(c):
    cache = c["cache"]
    q = cache.append(c["k"], c["v"], c["slots"], q=c["q"], q_gain=c["q_gain"],
                     k_gain=c["k_gain"], eps=EPS, rope=c["rope"], positions=c["positions"],
                     adjacent=c["case"]["adjacent"])
    k, v = cache.read(c["slots"])
    return {"q": q, "k": k, "v": v}


def _own_attend(c):
    return c["cache"].attend(c["q"], c["tables"], c["lengths"], c["starts"],
                             max_rows=c["max_rows"], max_length=c["max_length"],
                             first=c["first"], limit=c["limit"], scale=c["scale"], cap=c["cap"],
                             slopes=c["slopes"])


def _normed(x, gain, cos, sin, adjacent):
    """Rows of x [tokens, heads, dim] normalised and rotated, in float32."""
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    r = 2 * cos.shape[-1]
    if adjacent:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_place(c):
    case = c["case"]
    p, r, form = case["page"], case["rot"], case["format"]
    turn = c["rope"][c["positions"].long()][:, None, :]
    cos, sin = turn[..., :r // 2], turn[..., r // 2:]
    q = _normed(c["q"], c["q_gain"], cos, sin, case["adjacent"]).to(torch.bfloat16)
    k, ks = _quantise(_normed(c["k"], c["k_gain"], cos, sin, case["adjacent"]), form)
    v, vs = _quantise(c["v"].float(), form)
    page, off = c["slots"] // p, c["slots"] % p
    k_pages, v_pages = _raw(c["k_pages"]), _raw(c["v_pages"])
    k_pages[page, :, off] = _raw(k)
    v_pages[page, :, :, off] = _raw(v)
    if ks is not None:
        c["k_scales"][page, :, off] = ks
        c["v_scales"][page, :, off] = vs
    k = _value(k_pages[page, :, off], c["k_pages"])
    v = _value(v_pages[page, :, :, off], c["v_pages"])
    if ks is not None:
        k = k * c["k_scales"][page, :, off].unsqueeze(-1)
        v = v * c["v_scales"][page, :, off].unsqueeze(-1)
    return {"q": q, "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attend(c):
    case = c["case"]
    hq, h, d, p = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    g, tables, width, tokens = hq // h, c["tables"].long(), c["max_rows"], len(c["q"])
    b, keys = tables.shape[0], tables.shape[1] * p
    # the rows of all sequences as one rectangle; its padding reads row 0 and
    # writes one row past the last
    row = torch.arange(width, device="cuda")
    n_rows = (c["starts"][1:] - c["starts"][:-1]).long()[:, None]
    at = torch.where(row < n_rows, c["starts"][:-1].long()[:, None] + row, tokens)
    read = torch.where(at < tokens, at, 0)

    k = _value(_raw(c["k_pages"])[tables], c["k_pages"])             # b, pages, h, p, d
    v = _value(_raw(c["v_pages"])[tables], c["v_pages"])             # b, pages, h, d, p
    if c["k_scales"] is not None:
        k = k * c["k_scales"][tables].unsqueeze(-1)
        v = v * c["v_scales"][tables].unsqueeze(-2)
    k = k.permute(0, 2, 4, 1, 3).reshape(b * h, d, keys)
    v = v.permute(0, 2, 1, 4, 3).reshape(b * h, keys, d)
    q = c["q"].float()[read].view(b, width, h, g, d).permute(0, 2, 3, 1, 4)
    t = torch.bmm(q.reshape(b * h, g * width, d), k).view(b, h, g, width, keys)
    t *= c["scale"]
    if c["cap"]:
        t = torch.tanh(t / c["cap"]) * c["cap"]
    key = torch.arange(keys, device="cuda")
    pos = c["lengths"][:, None] - n_rows + row
    if c["slopes"] is not None:
        away = (pos[:, None, None, :, None] - key).abs()
        t = t - c["slopes"].view(1, h, g, 1, 1) * away
    first = torch.zeros_like(pos) if c["first"] is None else c["first"][read]
    limit = pos + 1 if c["limit"] is None else c["limit"][read]
    limit = torch.minimum(limit, c["lengths"][:, None])
    seen = (key >= first[..., None]) & (key < limit[..., None])      # b, width, keys
    t.masked_fill_(~seen[:, None, None], -math.inf)
    t -= t.amax(-1, keepdim=True).clamp_min(-3e38)
    t = t.exp_()
    total = t.sum(-1, keepdim=True)
    o = torch.bmm(t.view(b * h, g * width, keys), v).view(b, h, g, width, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    out = torch.zeros(tokens + 1, hq, d, dtype=torch.bfloat16, device="cuda")
    out[at] = o.permute(0, 3, 1, 2, 4).reshape(b, width, hq, d).to(torch.bfloat16)
    return out[:tokens]


# --------------------------------------------------------------------- work --

def work(case):
    hq, h, d = case["q_heads"], case["kv_heads"], case["dim"]
    token = 2 * h * (2 * d if case["format"] == "bf16" else d + 4)   # cache bytes of a token
    if case["op"] == "place":
        tokens = sum(_lengths(case))
        places = max(_lengths(case))
        in_out = 2 * d * (2 * hq + 2 * h) * tokens + 4 * case["rot"] * places
        back = 2 * 2 * h * d * tokens
        return {"bytes": in_out + 2 * token * tokens + back,
                "flops": 10.0 * d * (hq + 2 * h) * tokens}
    keys = pairs = 0
    for (pos, first, limit), length in zip(_intervals(case), _lengths(case)):
        limit = np.minimum(limit, length)
        pairs += int(np.maximum(0, limit - first).sum())
        mark = np.zeros(length + 1, dtype=np.int64)
        np.add.at(mark, first, 1)
        np.add.at(mark, limit, -1)
        keys += int((np.cumsum(mark)[:length] > 0).sum())
    return {"bytes": token * keys + 4.0 * d * hq * sum(_rows(case)), "flops": 4.0 * d * hq * pairs}


# -------------------------------------------------------------------- exact --

def _stored64(x, form):
    """What the cache holds of the rows of x (float64), as values."""
    if form == "bf16":
        return x
    big = CODE_MAX[form]
    scale = x.abs().max(dim=-1, keepdim=True).values / big
    y = torch.where(scale * big < TINY, torch.zeros_like(x), x / scale)
    if form == "int8":
        return torch.round(y) * scale
    # E4M3: 3 fraction bits, the smallest exponent -6; round to even
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -20))).clamp_min(-6.0)
    unit = torch.exp2(e - 3)
    return torch.round(y / unit) * unit * scale


def exact(case, seed):
    c = _inputs(case, seed)
    return _exact_place(c) if case["op"] == "place" else _exact_attend(c)


def _exact_place(c):
    case = c["case"]
    r = case["rot"]
    turn = c["rope"].double()[c["positions"].long()]

    def normed(x, gain):
        x = x.double()
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * gain.double()
        i = torch.arange(r // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + r // 2)
        z = torch.complex(x[..., a], x[..., b]) * torch.complex(turn[:, None, :r // 2],
                                                                turn[:, None, r // 2:])
        x[..., a], x[..., b] = z.real, z.imag
        return x

    return {"q": normed(c["q"], c["q_gain"]),
            "k": _stored64(normed(c["k"], c["k_gain"]), case["format"]),
            "v": _stored64(c["v"].double(), case["format"])}


def _exact_attend(c):
    case = c["case"]
    hq, h, d, p = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    g = hq // h
    out = torch.zeros(c["q"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for s, (length, (pos, first, limit)) in enumerate(zip(_lengths(case), _intervals(case))):
        n, pages = len(pos), c["tables"][s, :-(-length // p)].long()
        key = torch.arange(length, device="cuda")
        pos, first, limit = (torch.from_numpy(a).cuda()[:, None] for a in (pos, first, limit))
        hidden = (key < first) | (key >= limit)
        for j in range(h):
            k = _value(_raw(c["k_pages"])[pages, j], c["k_pages"]).double().reshape(-1, d)[:length]
            v = _value(_raw(c["v_pages"])[pages, j], c["v_pages"]).double()
            v = v.transpose(1, 2).reshape(-1, d)[:length]
            if c["k_scales"] is not None:
                k = k * c["k_scales"][pages, j].double().reshape(-1, 1)[:length]
                v = v * c["v_scales"][pages, j].double().reshape(-1, 1)[:length]
            for i in range(j * g, j * g + g):
                t = torch.mm(c["q"][start:start + n, i].double(), k.t()) * c["scale"]
                if c["cap"]:
                    t = c["cap"] * torch.tanh(t / c["cap"])
                if c["slopes"] is not None:
                    t = t - c["slopes"][i].double() * (pos - key).abs()
                t = t.masked_fill(hidden, -math.inf)
                out[start:start + n, i] = torch.softmax(t, -1) @ v
        start += n
    return out
