"""A decoder scored through its head and evaluated under many members' adapters:
rewards against a plain decoder in 64 bits, members side by side against members
one by one, a teacher's divergence, and a population scored in one batch.

The bf16 decoder rounds about 14 times a layer on its way to the hidden states; each
rounding is off by up to 2^-8 relative, about 2^-9 in the mean square, and they add as
independent errors: for 2 layers sqrt(28) 2^-9, about 1 % of the logits' norm.  The
bounds are four times that; with adapters a projection rounds once more, u: sqrt(56) 2^-9,
and four times that is 6 %.
"""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2608_17310_amd import esopt, workloads as wl
from paper_2608_17310_amd.adapters import Adapters
from paper_2608_17310_amd.generation import run_generation
from paper_2608_17310_amd.rollout import PROJECTIONS, Decoder

pytestmark = pytest.mark.gpu

LAYERS, HIDDEN, INTER, HQ, H, D, VOCAB = 2, 128, 192, 4, 2, 64, 97
SHAPES = {"q": (HQ * D, HIDDEN), "k": (H * D, HIDDEN), "v": (H * D, HIDDEN), "o": (HIDDEN, HQ * D),
          "gate": (INTER, HIDDEN), "up": (INTER, HIDDEN), "down": (HIDDEN, INTER)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def bf16(rng, *shape, std=1.0, mean=0.0):
    return torch.from_numpy((mean + rng.standard_normal(shape) * std).astype(np.float32)).bfloat16().cuda()


def make_params(seed):
    rng = np.random.default_rng(seed)
    return [bf16(rng, *s, std=0.15) if len(s) == 2 else bf16(rng, *s, std=0.1, mean=1.0)
            for s in wl.decoder_shapes(LAYERS, HIDDEN, INTER, HQ * D, H * D, VOCAB, tied=False)]


def make_adapters(seed, members, rank=8, names=PROJECTIONS, std=0.1):
    rng = np.random.default_rng(seed)
    return [{n: Adapters(bf16(rng, members, rank, SHAPES[n][1], std=std),
                         bf16(rng, members, SHAPES[n][0], rank, std=std),
                         torch.from_numpy(rng.uniform(0.5, 1.5, members).astype(np.float32)).cuda())
             for n in names} for _ in range(LAYERS)]


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def plain_logits(params, tokens, adapters=None, member=-1):
    """Logits of every position of one sequence, in 64 bits, with merged weights."""
    p = [f64(t) for t in params]

    def norm(x, g):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * g

    def weight(w, layer, name):
        if adapters is None or member < 0 or name not in adapters[layer]:
            return w
        a = adapters[layer][name]
        return w + f64(a.scales)[member] * f64(a.b)[member] @ f64(a.a)[member]
    n = len(tokens)
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(D // 2) * 2.0 / D)
    turn = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    x = p[0][tokens]
    for i in range(LAYERS):
        ws = [weight(w, i, name) for w, name in zip(p[1 + 9 * i:8 + 9 * i], PROJECTIONS)]
        wq, wk, wv, wo, gate, up, down = ws
        n1, n2 = p[8 + 9 * i:10 + 9 * i]
        y = norm(x, n1)
        q = oa.norm_rotate((y @ wq.T).reshape(n, HQ, D), np.ones(D), turn=turn)
        k = oa.norm_rotate((y @ wk.T).reshape(n, H, D), np.ones(D), turn=turn)
        v = (y @ wv.T).reshape(n, H, D)
        out = np.empty((n, HQ, D))
        for h in range(HQ):
            s = q[:, h] @ k[:, h // (HQ // H)].T * D ** -0.5
            s = np.where(np.tri(n, dtype=bool), s, -np.inf)
            e = np.exp(s - s.max(-1, keepdims=True))
            out[:, h] = e / e.sum(-1, keepdims=True) @ v[:, h // (HQ // H)]
        x = x + out.reshape(n, -1) @ wo.T
        y = norm(x, n2)
        g = y @ gate.T
        x = x + (g / (1 + np.exp(-g)) * (y @ up.T)) @ down.T
    return norm(x, p[-2]) @ p[-1].T


def log_softmax(z):
    z = z - z.max(-1, keepdims=True)
    return z - np.log(np.exp(z).sum(-1, keepdims=True))


def make_prompts(rng, sizes):
    return [rng.integers(0, VOCAB, n).tolist() for n in sizes]


def near(got, z, want, tokens, part):
    """A sum over `tokens` tokens, of logits z that are off by `part` of their norm:
    each token's logit and its normaliser."""
    spread = np.linalg.norm(z - z.mean(-1, keepdims=True), axis=-1).max() / np.sqrt(VOCAB)
    return abs(got - want) <= max(1, tokens) * max(2 * part * spread, 0.05)


def test_scores_without_logits():
    rng = np.random.default_rng(1)
    params = make_params(2)
    model = Decoder(params, HQ, H, D, False, seqs=3, length=100, format="bf16")
    prompts, targets = make_prompts(rng, [20, 3, 64]), make_prompts(rng, [5, 30, 1])
    got = model.score(prompts, targets)
    assert torch.equal(got, model.score(prompts, targets)) and got.dtype == torch.float32
    again = model.log_likelihood(prompts, targets)
    for s in range(3):
        z = plain_logits(params, prompts[s] + targets[s])[len(prompts[s]) - 1:-1]
        want = log_softmax(z)[np.arange(len(targets[s])), targets[s]].sum()
        assert near(got[s].item(), z, want, len(targets[s]), 0.04)
        # the same hidden states: the logits' rounding to bf16 apart, 2^-8 of a logit for each of a
        # token's two
        assert abs((got - again)[s].item()) <= 2 * len(targets[s]) * 2.0 ** -8 * np.abs(z).max() * 1.1
    assert not model.score(prompts, [[], [], []]).any()
    for bad in (([[1], [], [2]], [[3], [4], [5]]), ([[1], [2], [3]], [[4], [5]])):
        with pytest.raises(ValueError):
            model.score(*bad)


def test_scores_take_rows_to_the_head_in_slabs(monkeypatch):
    from paper_2608_17310_amd import rollout
    rng = np.random.default_rng(3)
    model = Decoder(make_params(4), HQ, H, D, False, seqs=2, length=200, format="bf16")
    prompts, targets = make_prompts(rng, [20, 3]), make_prompts(rng, [150, 100])
    want = model.score(prompts, targets)
    teacher = model.top_logits(prompts, targets, 5)
    far = model.divergence(prompts, targets, *teacher)
    monkeypatch.setattr(rollout, "ROWS_AT_A_TIME", 70)
    # the rows' sums run in another order: binary32's error of 250 terms of up to 2^4
    assert torch.allclose(model.score(prompts, targets), want, rtol=0, atol=250 * 2.0 ** -18)
    assert torch.allclose(model.divergence(prompts, targets, *teacher), far, rtol=0, atol=250 * 2.0 ** -18)


def test_divergence_from_a_teacher():
    rng = np.random.default_rng(5)
    params, others = make_params(6), make_params(7)
    teacher = Decoder(others, HQ, H, D, False, seqs=2, length=64, format="bf16")
    student = Decoder(params, HQ, H, D, False, seqs=2, length=64, format="bf16")
    prompts, targets = make_prompts(rng, [9, 30]), make_prompts(rng, [20, 7])
    ids, logits = teacher.top_logits(prompts, targets, 12)
    assert ids.shape == logits.shape == (27, 12)
    got = student.divergence(prompts, targets, ids, logits, scale=0.5)
    at = 0
    for s in range(2):
        n = len(targets[s])
        z = plain_logits(params, prompts[s] + targets[s])[len(prompts[s]) - 1:-1] * 0.5
        q = log_softmax(f64(logits)[at:at + n] * 0.5)
        logp = np.take_along_axis(log_softmax(z), ids.cpu().numpy()[at:at + n], 1)
        want = (np.exp(q) * (q - logp)).sum()
        assert near(got[s].item(), z, want, n, 0.04)
        at += n
    # its own distribution, all of it: nothing (terms of up to 2^4 that cancel, in bf16 logits 2^-8 off)
    ids, logits = student.top_logits(prompts, targets, VOCAB)
    z = logits.abs().max().item()
    assert student.divergence(prompts, targets, ids, logits).abs().max().item() <= 27 * 2 * z * 2.0 ** -8
    for bad in ((ids[:-1], logits[:-1]), (ids[0], logits[0]), (ids, logits[:, :3])):
        with pytest.raises(ValueError):
            student.divergence(prompts, targets, *bad)


@pytest.mark.parametrize("names", [PROJECTIONS, ("q", "v"), ("down",)])
def test_members_side_by_side(names):
    """Each sequence under its own member, and none: prompts and steps against a plain
    decoder with that member's merged weights."""
    rng = np.random.default_rng(8)
    params, adapters = make_params(9), make_adapters(10, 3, names=names)
    model = Decoder(params, HQ, H, D, False, seqs=5, length=120, format="bf16", adapters=adapters)
    members = [2, -1, 0, 1, 2]
    model.assign(members)
    prompts = make_prompts(rng, [70, 5, 33, 1, 12])
    more = rng.integers(0, VOCAB, (5, 3))
    logits = [model.prefill(prompts)]
    for t in range(3):
        logits.append(model.step(torch.from_numpy(more[:, t]).cuda()))
    assert model.status.item() == 0 and model.member_status.item() == 0
    for s, prompt in enumerate(prompts):
        want = plain_logits(params, prompt + more[s].tolist(), adapters, members[s])[len(prompt) - 1:]
        got = np.stack([f64(l[s]) for l in logits])
        assert np.linalg.norm(got - want) <= 0.06 * np.linalg.norm(want), s
        if members[s] >= 0:                                # and the member matters
            bare = plain_logits(params, prompt + more[s].tolist())[len(prompt) - 1:]
            assert np.linalg.norm(want - bare) > 0.12 * np.linalg.norm(want)


def test_what_assign_and_adapters_refuse():
    params, adapters = make_params(11), make_adapters(12, 2)
    with pytest.raises(ValueError):
        Decoder(params, HQ, H, D, False, seqs=2, length=64, adapters=adapters[:1])
    with pytest.raises(ValueError):
        Decoder(params, HQ, H, D, False, seqs=2, length=64, adapters=[{"w": adapters[0]["q"]}, {}])
    plain = Decoder(params, HQ, H, D, False, seqs=2, length=64)
    with pytest.raises(ValueError):
        plain.assign([0, 1])
    model = Decoder(params, HQ, H, D, False, seqs=2, length=64, adapters=adapters)
    for bad in ([0], [0, 1, 1], [0, 2], [0.0, 1.0], [0, 1 << 32], [[0, 1]]):
        with pytest.raises(ValueError):
            model.assign(bad)
        assert model.members.tolist() == [-1, -1]
    model.assign([-(1 << 40), 1])
    assert model.members.tolist() == [-1, 1]
    model.assign(torch.tensor([0, 1 << 32]).cuda())        # not read back, but reported
    model.prefill([[1, 2], [3]])
    assert model.member_status.item() == 1


def test_a_population_scored_in_one_batch():
    """A generation of low-rank members: each perturbed by a plan over its own adapters,
    all scored at once, the centre updated by theirs; what each scores alone is what it
    scores among the others."""
    rng = np.random.default_rng(13)
    params = make_params(14)
    n, sigma = 8, 3e-2
    adapters = make_adapters(15, n + 1, names=("q", "v", "up", "down"), std=0.05)
    tensors = lambda i: [t[i] for layer in adapters for a in layer.values() for t in (a.a, a.b)]
    centre = tensors(n)
    plan = esopt.Plan(centre)
    prompt, target = make_prompts(rng, [12])[0], make_prompts(rng, [6])[0]
    model = Decoder(params, HQ, H, D, False, seqs=n + 1, length=32, format="bf16", adapters=adapters)
    one = Decoder(params, HQ, H, D, False, seqs=1, length=32, format="bf16", adapters=adapters)
    before = [t.clone() for t in centre]
    for g in range(2):
        seeds = [100 * g + i // 2 for i in range(n)]
        signs = [1, -1] * (n // 2)
        for i in range(n):
            for t, c in zip(tensors(i), centre):
                t.copy_(c)
            for layer in adapters:
                for a in layer.values():
                    a.scales[:] = 1.0
            member = esopt.Plan(tensors(i))
            member.perturb(seeds[i], signs[i], sigma)
            member.close()
        model.assign(list(range(n + 1)))
        rewards = model.score([prompt] * (n + 1), [target] * (n + 1))
        assert rewards.isfinite().all()
        if g == 0:
            assert len({round(r, 4) for r in rewards[:n].tolist()}) > n // 2
            for i in (0, 3, n):
                one.assign([i])
                # sums of bf16 rows of another shape: four of a layer's roundings
                assert abs(one.score([prompt], [target]).item() - rewards[i].item()) <= 0.05 * len(target)
        plan.update(seeds, signs, rewards[:n].contiguous(), alpha=sigma)
    plan.close()
    assert all(t.isfinite().all() and not torch.equal(t, b) for t, b in zip(centre, before))


def test_a_generation_scored_without_logits():
    rng = np.random.default_rng(16)
    params = make_params(17)
    plan = esopt.Plan(params)
    model = Decoder(params, HQ, H, D, False, seqs=4, length=64, format="e4m3")
    prompts, targets = make_prompts(rng, [17, 30, 5, 9]), make_prompts(rng, [4] * 4)
    rec = run_generation(plan, [1, 1, 2, 2], [1, -1, 1, -1], 1e-2, 1e-2,
                         lambda i: model.score(prompts, targets).mean().item())
    assert len(set(rec.rewards)) > 2
    plan.close()


@pytest.mark.parametrize("slab", [1 << 28, 97 * 10])
def test_a_teachers_logits_are_not_rounded(monkeypatch, slab):
    """They are binary32 sums of exact products of the hidden states and the head (off by at most a
    step of 2^-23 of the sum of the products' sizes each), and the largest of them."""
    from paper_2608_17310_amd import rollout
    monkeypatch.setattr(rollout, "LOGITS_AT_A_TIME", slab)
    rng = np.random.default_rng(18)
    model = Decoder(make_params(19), HQ, H, D, False, seqs=2, length=64, format="bf16")
    prompts, targets = make_prompts(rng, [9, 30]), make_prompts(rng, [20, 7])
    ids, logits = model.top_logits(prompts, targets, 12)
    x, rows, *_ = model._answers(prompts, targets)
    X, W = x[rows].double(), model.head.double()
    z = X @ W.t()
    tol = (HIDDEN + 2) * 2.0 ** -23 * (X.abs() @ W.abs().t()).amax()
    assert logits.dtype == torch.float32 and ((z.gather(1, ids) - logits).abs() <= tol).all()
    assert ((z.topk(12, -1).values - logits).abs() <= tol).all()
