"""A decoder evaluated through the cache: logits against a plain decoder in 64
bits, prompts against single tokens, and a generation scored by it.

The bf16 decoder rounds about 14 times a layer on its way to the logits; each
rounding is off by up to 2^-8 relative, about 2^-9 in the mean square, and they
add as independent errors: for 2 layers sqrt(28) 2^-9, about 1 % of the logits'
norm.  The bound is four times that; E4M3 keys and values add 2^-4 / sqrt(12)
each, 2.6 % in the mean square together, and get four times the sum.
"""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2608_17310_amd import esopt, workloads as wl
from paper_2608_17310_amd.generation import replay, run_generation
from paper_2608_17310_amd.rollout import Decoder

pytestmark = pytest.mark.gpu

LAYERS, HIDDEN, INTER, HQ, H, D, VOCAB = 2, 128, 192, 4, 2, 64, 97


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def _params(seed, std=0.15):
    rng = np.random.default_rng(seed)
    out = []
    for s in wl.decoder_shapes(LAYERS, HIDDEN, INTER, HQ * D, H * D, VOCAB, tied=False):
        x = rng.standard_normal(s) * std if len(s) == 2 else 1 + 0.1 * rng.standard_normal(s)
        out.append(torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda())
    return out


def _plain(params, tokens, cap):
    """Logits of every position of one sequence, in 64 bits."""
    p = [t.float().cpu().numpy().astype(np.float64) for t in params]

    def norm(x, g):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * g
    n = len(tokens)
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(D // 2) * 2.0 / D)
    turn = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    x = p[0][tokens]
    for i in range(LAYERS):
        wq, wk, wv, wo, gate, up, down, n1, n2 = p[1 + 9 * i:10 + 9 * i]
        y = norm(x, n1)
        q = oa.norm_rotate((y @ wq.T).reshape(n, HQ, D), np.ones(D), 1e-6, turn)
        k = oa.norm_rotate((y @ wk.T).reshape(n, H, D), np.ones(D), 1e-6, turn)
        a, _ = oa.attend(q, k, (y @ wv.T).reshape(n, H, D), D ** -0.5, cap)
        x = x + a.reshape(n, HQ * D) @ wo.T
        y = norm(x, n2)
        g = y @ gate.T
        x = x + (g / (1 + np.exp(-g)) * (y @ up.T)) @ down.T
    return norm(x, p[-2]) @ p[-1].T


def _prompts(rng, sizes):
    return [rng.integers(0, VOCAB, n).tolist() for n in sizes]


@pytest.mark.parametrize("form,bound", [("bf16", 0.04), ("e4m3", 0.15)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_prompts_and_steps_against_a_plain_decoder(form, bound, cap):
    rng = np.random.default_rng(30)
    params = _params(31)
    model = Decoder(params, HQ, H, D, False, seqs=4, length=150, format=form, cap=cap)
    prompts = _prompts(rng, [70, 1, 128, 33])
    more = rng.integers(0, VOCAB, (4, 6))
    logits = [model.prefill(prompts)]
    for t in range(6):
        logits.append(model.step(torch.from_numpy(more[:, t]).cuda()))
    assert model.status.item() == 0
    for s, prompt in enumerate(prompts):
        want = _plain(params, prompt + more[s].tolist(), cap)[len(prompt) - 1:]
        got = np.stack([l[s].double().cpu().numpy() for l in logits])
        assert np.linalg.norm(got - want) <= bound * np.linalg.norm(want), (s, form)


def test_likelihood_and_greedy_tokens():
    rng = np.random.default_rng(32)
    params = _params(33)
    model = Decoder(params, HQ, H, D, False, seqs=3, length=100, format="bf16")
    prompts, targets = _prompts(rng, [20, 3, 64]), _prompts(rng, [5, 9, 1])
    got = model.log_likelihood(prompts, targets).double().cpu().numpy()
    for s in range(3):
        z = _plain(params, prompts[s] + targets[s], 0.0)[len(prompts[s]) - 1:-1]
        z = z - z.max(-1, keepdims=True)
        logp = z - np.log(np.exp(z).sum(-1, keepdims=True))
        want = logp[np.arange(len(targets[s])), targets[s]]
        # 4 % of the logits' norm over the vocabulary, for each token and its normaliser
        slack = 2 * 0.04 * np.linalg.norm(z - z.mean(-1, keepdims=True)) / np.sqrt(VOCAB)
        assert abs(got[s] - want.sum()) <= max(1, len(want)) * max(slack, 0.05)
    out = model.generate(prompts, 7)
    assert out.shape == (3, 7)
    logits = model.prefill([p + o for p, o in zip(prompts, out[:, :-1].tolist())])
    best, chosen = logits.max(-1).values, logits.gather(1, out[:, -1:])[:, 0]
    assert torch.all(best - chosen <= 0.04 * logits.std(-1) * 4)
    with pytest.raises(ValueError):
        model.prefill(prompts[:2])
    with pytest.raises(ValueError):
        model.prefill([[1]] * 2 + [[1] * 101])


def test_a_generation_scored_by_the_decoder_replays():
    rng = np.random.default_rng(34)
    params = _params(35)
    start = [p.clone() for p in params]
    plan = esopt.Plan(params)
    model = Decoder(params, HQ, H, D, False, seqs=4, length=64, format="e4m3")
    prompts, targets = _prompts(rng, [17, 30, 5, 9]), _prompts(rng, [4] * 4)
    before = model.log_likelihood(prompts, targets)
    assert torch.equal(before, model.log_likelihood(prompts, targets))
    records = []
    for g in range(6):
        seeds = [100 * g + i for i in range(8) for _ in (0, 1)]
        signs = [1, -1] * 8
        records.append(run_generation(
            plan, seeds, signs, 2e-2, 4e-2,
            lambda i: model.log_likelihood(prompts, targets).mean().item(), checksum=True))
    assert len(set(records[0].rewards)) > 8                # members differ
    after = model.log_likelihood(prompts, targets)
    assert after.mean() > before.mean()                    # and the parameters learn from it
    end = [p.clone() for p in params]
    for p, s in zip(params, start):
        p.copy_(s)
    replay(plan, records)
    for p, e in zip(params, end):
        assert torch.equal(p.view(torch.int16), e.view(torch.int16))
    plan.close()


def test_long_likelihoods_are_the_same_every_time():
    """The sum over a target's tokens has one order: the same bits on every
    call, and next to the sum in 64 bits."""
    rng = np.random.default_rng(36)
    params = _params(37)
    model = Decoder(params, HQ, H, D, False, seqs=4, length=4096, format="bf16")
    sizes = [4000, 3001, 1, 2500]
    prompts, targets = _prompts(rng, [3, 17, 64, 1]), _prompts(rng, sizes)
    tokens = sum(len(p) + n for p, n in zip(prompts, sizes))
    hidden = torch.from_numpy(rng.standard_normal((tokens, HIDDEN)).astype(np.float32)).to(
        torch.bfloat16).cuda()
    model._forward = lambda *args: hidden                  # the sum alone is looked at
    got = model.log_likelihood(prompts, targets)
    for _ in range(20):
        assert torch.equal(model.log_likelihood(prompts, targets), got)
    logp = (hidden @ params[-1].t()).float().log_softmax(-1).double().cpu().numpy()
    at = 0
    for s in range(4):
        ids = prompts[s] + targets[s]
        r = np.arange(len(prompts[s]) - 1, len(ids) - 1)
        want = logp[at + r, np.array(ids)[r + 1]].sum()
        # terms as float32 (2^-24 of each, half of it at most lost), the logits' rounding to bf16
        # the same in both but for products summed in another order (one bf16 step, 2^-8 of a logit
        # of at most 20, in a row)
        assert abs(got[s].item() - want) <= sizes[s] * 20 * 2.0 ** -8
        at += len(ids)
