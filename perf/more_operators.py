"""Cases of the operators at a decoder's head and beside its projections, with
which the members of a population are scored, compared with a teacher and
evaluated side by side.

    score    log-probabilities of the targets of hidden rows over a large
             vocabulary, without keeping the logits; with "grad" also the
             gradients of their weighted sum for the rows and the head
    distill  the divergence from a teacher that is known by its top logits, and
             the student's log-probabilities there; with "grad" also the
             gradients of the weighted sum of the divergences
    adapt    a shared projection with the low-rank adapters of many members
             beside it, one member's for each row

Widths and vocabulary are those of the package's parameter sets (hidden 1024,
2560 and 5120, vocabulary 151936), and generic odd ones.

    own                   False: the plain form; True: the package's kernels
    listed()              the fixed cases
    draw(rng)             one more case of the same ranges
    prepare(case, seed)   what a program has in hand before the call
    run(state)            one pass; returns its outputs
    work(case)            bytes and operations a pass cannot do without
    exact(case, seed)     the outputs from the definition, in 64 bits
"""
import math

import torch

own = False

FLOPS_MAX = 6.6e12             # of a case: the largest listed one's
BYTES_MAX = 8.0e9


# ---------------------------------------------------------------- the cases --

def listed():
    return [
        # the next token of one rollout, under the small model: latency and the head's bytes
        dict(name="score 1 row", op="score", rows=1, hidden=1024, vocab=151936, masked=0.0,
             scale=1.0, grad=False),
        # one token of each of a generation step's 32 tasks, under the large model
        dict(name="score 32 rows", op="score", rows=32, hidden=5120, vocab=151936, masked=0.0,
             scale=1.0, grad=False),
        # the answers of a member's tasks at once; the prompts' rows are masked
        dict(name="score 1021 rows", op="score", rows=1021, hidden=2560, vocab=151936, masked=0.3,
             scale=1.0, grad=False),
        # a batch of long answers under the large model
        dict(name="score 4099 rows", op="score", rows=4099, hidden=5120, vocab=151936, masked=0.0,
             scale=1.0, grad=False),
        # a short supervised step of a model with an odd vocabulary and width
        dict(name="train 333 rows", op="score", rows=333, hidden=1000, vocab=32003, masked=0.2,
             scale=1.0, grad=True),
        # a supervised step of the middle model
        dict(name="train 2048 rows", op="score", rows=2048, hidden=2560, vocab=151936, masked=0.1,
             scale=1.0, grad=True),
        # a few answers held against a teacher's 20 likeliest tokens: a reward
        dict(name="distill 77 rows", op="distill", rows=77, hidden=1024, vocab=151936, masked=0.0,
             entries=20, scale=1.0, grad=False),
        # a distillation step at temperature 2
        dict(name="distill 1000 rows", op="distill", rows=1000, hidden=2560, vocab=151936,
             masked=0.1, entries=64, scale=0.5, grad=True),
        # one token of one member, through the large model's square projection
        dict(name="adapt 1 row", op="adapt", rows=1, inner=5120, outer=5120, rank=16, members=1,
             bare=0.0),
        # one token of each of 32 members, through its widest projection
        dict(name="adapt 32 rows", op="adapt", rows=32, inner=5120, outer=17408, rank=16,
             members=32, bare=0.0),
        # the prompts of 16 members, through the middle model's wide projection
        dict(name="adapt prompts", op="adapt", rows=8403, inner=2560, outer=9728, rank=32,
             members=16, bare=0.0),
        # long histories of 8 members, part of them under no adapter
        dict(name="adapt histories", op="adapt", rows=16384, inner=5120, outer=5120, rank=64,
             members=8, bare=0.2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A model's width: one of the package's sets, or any multiple of eight; an odd one now and then."""
    kind = rng.random()
    if kind < 0.4:
        return rng.choice([w for w in (1024, 2560, 5120, 9728, 17408) if lo <= w <= hi])
    n = _log_int(rng, lo, hi)
    return n if kind > 0.9 else max(lo, n // 8 * 8)


def draw(rng):
    op = rng.choice(["score", "score", "distill", "adapt"])
    while True:
        if op == "adapt":
            members = _log_int(rng, 1, 64)
            case = dict(op=op, rows=_log_int(rng, 1, 16384), inner=8 * (_width(rng, 64, 17408) // 8),
                        outer=_width(rng, 64, 17408), rank=rng.choice([8, 16, 16, 32, 64, 128]),
                        members=members, bare=rng.choice([0.0, 0.0, 0.3]))
        else:
            case = dict(op=op, rows=_log_int(rng, 1, 6000), hidden=_width(rng, 64, 6000),
                        vocab=rng.choice([151936, _log_int(rng, 500, 200000)]),
                        masked=rng.choice([0.0, 0.2, 0.7]), scale=rng.choice([1.0, 1.0, 0.5, 1.4]),
                        grad=rng.choice([False, True]))
            if op == "distill":
                case["entries"] = _log_int(rng, 1, 128)
        w = work(case)
        if w["flops"] <= FLOPS_MAX and w["bytes"] <= BYTES_MAX:
            return case


# --------------------------------------------------------------- the inputs --

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _weight(gen, rows, width, std):
    """A bf16 matrix of normal values, a slab of rows at a time in 32 bits."""
    out = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    for part in out.split(max(1, (1 << 27) // width)):
        part.copy_(_normal(gen, *part.shape) * std)
    return out


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n = case["rows"]
    c = {"case": case}
    if case["op"] == "adapt":
        m, r, i, o = case["members"], case["rank"], case["inner"], case["outer"]
        c["x"] = _normal(gen, n, i).to(torch.bfloat16)
        c["weight"] = _weight(gen, o, i, i ** -0.5)
        c["a"] = (_normal(gen, m, r, i) * i ** -0.5).to(torch.bfloat16)
        c["b"] = (_normal(gen, m, o, r) * 0.2 * r ** -0.5).to(torch.bfloat16)
        c["scales"] = 0.5 + _uniform(gen, m)
        # the rows of a member are adjacent, as packed sequences are; the members' shares differ
        cuts = (_uniform(gen, m).sort().values * n).long()
        member = (torch.arange(n, device="cuda")[:, None] >= cuts).sum(1)
        order = torch.randperm(m, generator=gen, device="cuda")
        if n <= 64:
            member = torch.arange(n, device="cuda")
        index = order[member % m]
        stretch = _uniform(gen, n // 64 + 1) < case["bare"]
        c["index"] = torch.where(stretch[torch.arange(n, device="cuda") // 64], -1, index).int()
        return c
    h, v = case["hidden"], case["vocab"]
    k = case.get("entries", 1)
    c["weight"] = _weight(gen, v, h, h ** -0.5)
    x = _normal(gen, n, h) * 2.0
    # tokens as a text has them: few often, many seldom; a row's are distinct, in no order
    ids = ((v - k) * _uniform(gen, n, k).pow(3.0)).long().clamp_(max=v - k).sort(1).values
    ids = ids + torch.arange(k, device="cuda")
    ids = ids.gather(1, _uniform(gen, n, k).argsort(1))
    # what a trained model gives its targets: a logit above the others'
    likely = c["weight"][ids[:, 0]].float()
    x += likely * (8.0 * _uniform(gen, n, 1))
    if k > 1:
        x += c["weight"][ids[:, 1]].float() * 5.0
    c["x"] = x.to(torch.bfloat16)
    skip = _uniform(gen, n) < case["masked"]
    skip[0] = False
    c["grad"] = torch.full((n,), 1.0 / n, device="cuda") * (0.5 + _uniform(gen, n))
    if case["op"] == "score":
        c["targets"] = torch.where(skip, -100, ids[:, 0])
        return c
    # the teacher's entries: falling, and for some rows fewer than there is room for
    c["logits"] = (_normal(gen, n, k) * 2.0 + 10.0).sort(1, descending=True).values
    have = (k * (0.5 + 0.75 * _uniform(gen, n, 1))).ceil().clamp_(1, k)
    absent = (torch.arange(k, device="cuda") >= have) | skip[:, None]
    c["ids"] = torch.where(absent, -1, ids)
    return c


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        if case["op"] == "adapt":
            from paper_2608_17310_amd.adapters import Adapters
            state["adapters"] = Adapters(state["a"], state["b"], state["scales"])
        else:
            from paper_2608_17310_amd.head import Head
            state["head"] = Head(state["weight"])
    return state


# ------------------------------------------------------------------ running --

def run(state):
    op = state["case"]["op"]
    if own:
        return {"score": _own_score, "distill": _own_distill, "adapt": _own_adapt}[op](state)
    return {"score": _plain_score, "distill": _plain_distill, "adapt": _plain_adapt}[op](state)


def _own_score(c):
    head, scale = c["head"], c["case"]["scale"]
    logp, lse = head.score(c["x"], c["targets"], scale=scale)
    out = {"logp": logp, "lse": lse}
    if c["case"]["grad"]:
        out["d_hidden"], out["d_weight"] = head.score_gradient(
            c["x"], c["targets"], logp, lse, c["grad"], scale=scale)
    return out


def _own_distill(c):
    head, scale = c["head"], c["case"]["scale"]
    loss, logp, lse = head.distill(c["x"], c["ids"], c["logits"], scale=scale)
    out = {"loss": loss, "logp": logp, "lse": lse}
    if c["case"]["grad"]:
        out["d_hidden"], out["d_weight"] = head.distill_gradient(
            c["x"], c["ids"], c["logits"], logp, lse, c["grad"], scale=scale)
    return out


def _own_adapt(c):
    return {"y": c["adapters"].project(c["x"], c["weight"], c["index"])}


def _plain_logits(c):
    """Scaled logits and their normalisers, in 32 bits."""
    x, w = c["x"].float(), c["weight"].float()
    z = (x @ w.t()) * c["case"]["scale"]
    top = z.amax(-1, keepdim=True)
    return x, w, z, (z - top).exp().sum(-1).log() + top[:, 0]


def _plain_grads(c, x, w, dz):
    return {"d_hidden": (dz @ w).to(torch.bfloat16), "d_weight": (dz.t() @ x).to(torch.bfloat16)}


def _plain_score(c):
    live = c["targets"] >= 0
    at = c["targets"].clamp(min=0)[:, None]
    x, w, z, lse = _plain_logits(c)
    logp = z.gather(1, at)[:, 0] - lse
    out = {"logp": torch.where(live, logp, 0.0), "lse": torch.where(live, lse, 0.0)}
    if c["case"]["grad"]:
        g = torch.where(live, c["grad"] * c["case"]["scale"], 0.0)[:, None]
        dz = (z - lse[:, None]).exp_().mul_(-g)
        dz.scatter_add_(1, at, g)
        out.update(_plain_grads(c, x, w, dz))
    return out


def _plain_distill(c):
    here = c["ids"] >= 0
    at = c["ids"].clamp(min=0)
    live = here.any(1)
    t = torch.where(here, c["logits"] * c["case"]["scale"], -math.inf)
    top = t.amax(1, keepdim=True).clamp_min(-3e38)
    e = (t - top).exp()
    total = e.sum(1, keepdim=True)
    q = torch.where(here, e / total, 0.0)
    log_q = torch.where(here, t - top - total.log(), 0.0)
    x, w, z, lse = _plain_logits(c)
    logp = torch.where(here, z.gather(1, at) - lse[:, None], 0.0)
    out = {"loss": (q * (log_q - logp)).sum(1), "logp": logp, "lse": torch.where(live, lse, 0.0)}
    if c["case"]["grad"]:
        g = torch.where(live, c["grad"] * c["case"]["scale"], 0.0)[:, None]
        dz = (z - lse[:, None]).exp_().mul_(g)
        dz.scatter_add_(1, at, -g * q)
        out.update(_plain_grads(c, x, w, dz))
    return out


def _plain_adapt(c):
    m, r = c["case"]["members"], c["case"]["rank"]
    x = c["x"].float()
    y = x @ c["weight"].float().t()
    # every member's small products, and of them each row's own
    u = x @ c["a"].float().view(m * r, -1).t()
    mine = c["index"][:, None] == torch.arange(m, device="cuda")
    u = u.view(-1, m, r) * torch.where(mine, c["scales"], 0.0)[..., None]
    y += u.view(-1, m * r) @ c["b"].float().permute(0, 2, 1).reshape(m * r, -1)
    return {"y": y.to(torch.bfloat16)}


# --------------------------------------------------------------------- work --

def work(case):
    n = case["rows"]
    if case["op"] == "adapt":
        # (members beside bare rows are counted as if all rows had one)
        m, r, i, o = min(case["members"], n), case["rank"], case["inner"], case["outer"]
        return {"bytes": 2.0 * (n * (i + o) + i * o + m * r * (i + o)),
                "flops": 2.0 * n * (i * o + r * (i + o))}
    h, v, k = case["hidden"], case["vocab"], case.get("entries", 1)
    live = max(1.0, n * (1.0 - case["masked"]))     # masked rows need neither reading nor products
    once = 2.0 * live * h * v
    read = 2.0 * (live * h + v * h) + (8.0 if k == 1 else 12.0) * n * k
    return {"bytes": read + 4.0 * n * (2 + k) + (2.0 * (n * h + v * h) if case["grad"] else 0.0),
            # the logits, and the two products of their gradient with rows and head
            "flops": once * (3 if case["grad"] else 1)}


# -------------------------------------------------------------------- exact --

def exact(case, seed):
    c = _inputs(case, seed)
    return {"score": _exact_head, "distill": _exact_head, "adapt": _exact_adapt}[case["op"]](c)


def _exact_head(c):
    case = c["case"]
    score, n, s = case["op"] == "score", case["rows"], case["scale"]
    ids = c["targets"][:, None] if score else c["ids"]
    k = ids.shape[1]
    here = ids >= 0
    # the wanted distribution over the entries; one entry has all of it
    if score:
        log_q = torch.zeros(n, 1, dtype=torch.float64, device="cuda")
    else:
        t = (c["logits"].double() * s).masked_fill(~here, -1e300)
        log_q = t - torch.logsumexp(t, 1, keepdim=True)
    q = log_q.exp() * here
    w = c["weight"].double()
    logp = torch.zeros(n, k, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n, dtype=torch.float64, device="cuda")
    dx = torch.zeros(n, case["hidden"], dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w) if case["grad"] else None
    step = max(1, (1 << 28) // case["vocab"])
    for a in range(0, n, step):
        b = min(n, a + step)
        rows = torch.nonzero(here[a:b].any(1)).flatten() + a
        if not len(rows):
            continue
        x = c["x"][rows].double()
        lp = torch.mm(x, w.t()) * s
        lse[rows] = torch.logsumexp(lp, -1)
        lp -= lse[rows][:, None]
        at = ids[rows].clamp(min=0)
        logp[rows] = lp.gather(1, at) * here[rows]
        if case["grad"]:
            # of sum q log p: q minus p; a divergence is its negative
            d = -lp.exp_() * q[rows].sum(1, keepdim=True)
            d.scatter_add_(1, at, q[rows])
            d *= c["grad"][rows].double()[:, None] * (s if score else -s)
            dx[rows] = torch.mm(d, w)
            dw += torch.mm(d.t().contiguous(), x)
            del d
        del lp
    out = {"logp": logp[:, 0] if score else logp, "lse": lse}
    if not score:
        out["loss"] = (q * torch.where(here, log_q - logp, 0.0)).sum(1)
    if case["grad"]:
        out.update(d_hidden=dx, d_weight=dw)
    return out


def _exact_adapt(c):
    w, x = c["weight"].double(), c["x"].double()
    y = torch.mm(x, w.t())
    for i in range(c["case"]["members"]):
        rows = torch.nonzero(c["index"] == i).flatten()
        u = torch.mm(x[rows], c["a"][i].double().t()) * c["scales"][i].double()
        y[rows] += torch.mm(u, c["b"][i].double().t())
    return {"y": y}
