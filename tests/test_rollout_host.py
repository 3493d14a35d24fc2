"""The decoder's bookkeeping without a GPU: what a call refuses, what it leaves
as it was, and the sums of log-probabilities over given hidden states."""
import numpy as np
import pytest
import torch

from paper_2608_17310_amd import rollout
from paper_2608_17310_amd.rollout import Decoder

VOCAB, HIDDEN, SEQS, LENGTH = 11, 5, 3, 40


@pytest.fixture
def model():
    """A decoder on the CPU with hidden states of its own in place of the layers."""
    gen = torch.Generator().manual_seed(1)
    m = Decoder.__new__(Decoder)
    m.embedding = torch.randn(VOCAB, HIDDEN, generator=gen)
    m.head = torch.randn(VOCAB, HIDDEN, generator=gen)
    m.length = LENGTH
    m.lengths = torch.zeros(SEQS, dtype=torch.int32)
    m.longest = 0
    m.calls = []
    m.hidden = torch.randn(SEQS * LENGTH, HIDDEN, generator=gen)

    def forward(tokens, seq, positions, starts, max_rows):
        m.calls.append((tokens.tolist(), starts.tolist(), max_rows))
        return m.hidden[:len(tokens)]
    m._forward = forward
    return m


def _state(m):
    return m.lengths.tolist(), m.longest, len(m.calls)


def test_likelihood_refuses_what_has_no_prediction(model):
    """The first token of a sequence is predicted by nothing, and prompts and
    targets go in pairs."""
    model.prefill([[1, 2], [3], [4, 5, 6]])
    before = _state(model)
    for prompts, targets in (([[1], [], [2]], [[3], [4], [5]]),
                             ([[1], [2], [3]], [[4], [5], [6], [7]]),
                             ([[1], [2], [3], [4]], [[4], [5], [6]]),
                             ([[1], [2]], [[4], [5]])):
        with pytest.raises(ValueError):
            model.log_likelihood(prompts, targets)
        assert _state(model) == before


def test_likelihood_sums_the_targets_terms(model):
    prompts, targets = [[1, 2], [3], [4, 5, 6]], [[7, 8, 9], [], iter([10])]
    got = model.log_likelihood(prompts, targets)
    logp = (model.hidden @ model.head.t()).double().log_softmax(-1)
    # rows: 0 .. 4 of the first sequence, 5 of the second, 6 .. 9 of the third
    want = [logp[1, 7] + logp[2, 8] + logp[3, 9], 0.0, logp[8, 10]]
    # three terms of float32 logits and logarithms, each off by a few 2^-24 of up to 2^4
    np.testing.assert_allclose(got.numpy(), [float(w) for w in want], rtol=0, atol=2.0 ** -16)
    assert got.dtype == torch.float32
    assert not model.log_likelihood(prompts, [[], [], []]).any()


@pytest.mark.parametrize("count", [0, 1, 2, 4])
def test_a_refused_step_leaves_the_decoder_as_it_was(model, count):
    model.prefill([[1, 2], [3], [4, 5, 6]])
    before = _state(model)
    for tokens in (torch.zeros(count, dtype=torch.long), torch.zeros(SEQS, 1, dtype=torch.long)):
        with pytest.raises(ValueError):
            model.step(tokens)
        assert _state(model) == before
    model.step(torch.zeros(SEQS, dtype=torch.long))
    assert model.lengths.tolist() == [3, 2, 4] and model.longest == 4
    model.longest = LENGTH                                 # and when the cache is full
    with pytest.raises(ValueError):
        model.step(torch.zeros(SEQS, dtype=torch.long))
    assert model.lengths.tolist() == [3, 2, 4]


def test_no_tokens_can_be_generated(model):
    prompts = [[1, 2], [3], [4, 5, 6]]
    out = model.generate(prompts, 0)
    assert out.shape == (SEQS, 0) and out.dtype == torch.long
    assert model.generate(prompts, 2).shape == (SEQS, 2)
    with pytest.raises(ValueError):
        model.generate(prompts, -1)


@pytest.mark.parametrize("bad", [-1, VOCAB, 1 << 40])
def test_tokens_outside_the_vocabulary_are_refused(model, bad):
    """-1 would read the embedding's last row, and others past its end."""
    model.prefill([[1, 2], [3], [4, 5, 6]])
    before = _state(model)
    for prompts in ([[bad], [1], [2]], [[1, 2], [3, 4, bad], [5]]):
        for call in (lambda: model.prefill(prompts), lambda: model.generate(prompts, 1),
                     lambda: model.log_likelihood(prompts, [[1], [2], [3]]),
                     lambda: model.log_likelihood([[1], [2], [3]], prompts),
                     lambda: model.prefill([torch.tensor(p) for p in prompts])):
            with pytest.raises(ValueError):
                call()
            assert _state(model) == before
    with pytest.raises(ValueError):
        model.step(torch.tensor([1, bad, 2]))
    assert _state(model) == before
    model.prefill([[0, VOCAB - 1], [0], [VOCAB - 1]])


@pytest.mark.parametrize("rows", [1, 2, 4, 100])
def test_likelihood_holds_few_logits_at_a_time(model, monkeypatch, rows):
    """Logits are made a slab of rows at a time, whatever the targets' lengths,
    and the sums do not depend on it."""
    prompts, targets = [[1, 2], [3], [4, 5, 6]], [[7, 8, 9, 0, 1], [2], [10, 4]]
    want = model.log_likelihood(prompts, targets)
    sizes = []
    linear = rollout.F.linear

    def counted(x, w):
        sizes.append(len(x))
        return linear(x, w)
    monkeypatch.setattr(rollout.F, "linear", counted)
    monkeypatch.setattr(rollout, "LOGITS_AT_A_TIME", rows * VOCAB + VOCAB - 1)
    got = model.log_likelihood(prompts, targets)
    assert sum(sizes) == 8 and max(sizes) <= rows
    # float32 logits of products summed in another order: 2^-24 of up to 2^5, five terms and their
    # normalisers
    np.testing.assert_allclose(got.numpy(), want.numpy(), rtol=0, atol=10 * 2.0 ** -19)
    monkeypatch.setattr(rollout, "LOGITS_AT_A_TIME", VOCAB - 1)
    assert torch.isfinite(model.log_likelihood(prompts, targets)).all()


@pytest.mark.parametrize("kind", [list, tuple, np.array, lambda t: torch.tensor(t, dtype=torch.int32)])
def test_a_steps_tokens_may_be_any_sequence(model, kind):
    model.prefill([[1, 2], [3], [4, 5, 6]])
    want = model.step(torch.tensor([7, 8, 9]))
    model.prefill([[1, 2], [3], [4, 5, 6]])
    assert torch.equal(model.step(kind([7, 8, 9])), want)
    assert model.calls[-1][0] == [7, 8, 9]
    with pytest.raises(ValueError):
        model.step(kind([7, 8]))
    with pytest.raises(ValueError):
        model.step(kind([7, 8, VOCAB]))
