"""Scores at a head and divergences from a teacher's top logits, with their
gradients (es_head_*), against the fp64 oracle.

Tolerances are the kernels' roundings.  E = 2^-24 is half a binary32 step.  A logit
is a binary32 sum of H exact products: off by at most H steps of 2 E (a matrix unit's
sum may be cut instead of rounded) of the sum S of their sizes; Z below.  A
normaliser is off by its logits' error, by exp2's (2 E of a value below
2^6 and the function's own 2 E, all relative to the sum) and by the sum's over a
tile's 64 values and 6 joins, and its logarithm by 4 E of it.  A log-probability
takes two logits.  bf16's rounding is off by at most U = 2^-8 of a value.  Gradients:
one rounding of each logit's gradient d (U sum |d w|), its binary32 errors (that of
exp(z - lse), twice a logit's), and one of the result.
"""
import numpy as np
import pytest
import torch

from oracle import head as oh
from paper_2608_17310_amd import esopt
from paper_2608_17310_amd.head import ES_HEAD_BAD_ID, Head

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def mat(rng, rows, width, std=1.0, stride=None, at=0):
    """A bf16 matrix of `rows` rows, `stride` elements apart, `at` elements into its memory."""
    stride = width if stride is None else stride
    room = torch.full((at + rows * stride + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    t = room[at:at + rows * stride].view(rows, stride)[:, :width]
    t.copy_(torch.from_numpy((rng.standard_normal((rows, width)) * std).astype(np.float32)))
    return t


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def slack(x, w, scale):
    """The error of a row's logits, and of its normaliser beside theirs."""
    s = (np.abs(x) @ np.abs(w).T).max(1) * abs(scale)
    z = 2 * E * x.shape[1] * s + 4 * E * s
    return z, 2 * E * 64 + 100 * E + 8 * E * s


def make(rng, rows, vocab, hidden, entries=None, masked=0.2, std=None, **kw):
    x = mat(rng, rows, hidden, **kw)
    w = mat(rng, vocab, hidden, (3.0 if std is None else std) / np.sqrt(hidden), **kw)
    k = entries or 1
    ids = rng.integers(0, vocab, (rows, k))
    if entries:
        ids[rng.random((rows, k)) < 0.25] = -1
    ids[rng.random(rows) < masked] = -100
    ids[rows // 2] = rng.integers(0, vocab, k)
    teacher = rng.standard_normal((rows, k)).astype(np.float32) * 3 if entries else None
    grad = rng.standard_normal(rows).astype(np.float32)
    return x, w, ids, teacher, grad


def check(x, w, ids, teacher, grad, scale, status=None):
    """A call of each direction against the oracle; its outputs."""
    head = Head(w)
    X, W = np.where((ids >= 0).any(1)[:, None], f64(x), 0.0), f64(w)
    T = None if teacher is None else teacher.astype(np.float64)
    d_ids = dev(ids if teacher is not None else ids[:, 0], torch.int64)
    d_grad = dev(grad, torch.float32)
    s = float(np.float32(scale))
    loss, logp, lse = oh.score(X, W, ids, s, T)
    if teacher is None:
        g_logp, g_lse = head.score(x, d_ids, scale=scale, status=status)
        outs = (g_logp, g_lse)
        dx, dw = head.score_gradient(x, d_ids, g_logp, g_lse, d_grad, scale=scale)
    else:
        d_t = dev(teacher, torch.float32)
        g_loss, g_logp, g_lse = head.distill(x, d_ids, d_t, scale=scale, status=status)
        outs = (g_loss, g_logp, g_lse)
        dx, dw = head.distill_gradient(x, d_ids, d_t, g_logp, g_lse, d_grad, scale=scale)
    z, norm = slack(X, W, s)
    live, void = oh.kinds(ids, len(W))
    np.testing.assert_array_equal(np.isnan(f64(g_lse)), void)
    ok = ~void
    assert np.all(np.abs(f64(g_lse) - lse)[ok] <= (z + norm + 4 * E * np.abs(lse))[ok])
    got = f64(g_logp).reshape(logp.shape)
    tol = (2 * z + norm)[:, None] + 8 * E * (np.abs(logp) + np.abs(lse)[:, None])
    assert np.all(np.abs(got - logp)[ok] <= tol[ok])
    if teacher is not None:
        q, log_q = oh.weights(ids, T, s)
        # q's own error: its exponent's, of a product rounded once, and its sum's
        q_err = q * (4 * E * (np.abs(np.where(q > 0, T, 0.0)) * s + 64))
        some = np.where(q > 0, np.abs(log_q - logp), 0.0)
        tol = (q * (tol + 16 * E * (1 + np.abs(log_q)))).sum(1) + (q_err * (some + 1)).sum(1) + \
            300 * E * (q * some).sum(1)
        assert np.all(np.abs(f64(g_loss) - loss)[ok] <= tol[ok] + 1e-37)
    d = oh.logit_gradients(X, W, ids, grad, s, T)
    want_x, want_w = oh.gradients(X, W, ids, grad, s, T)
    # of f p: both logits' and the normaliser's errors, and a few roundings
    f = np.abs(np.where(live, grad, 0.0) * s)[:, None]
    p_err = (2 * z + norm + 32 * E)[:, None] + 4 * E * np.abs(lse)[:, None]
    p_err = np.where(ok[:, None], p_err, 0.0)
    q, _ = oh.weights(ids, T, s)
    full = np.zeros_like(d)
    for r in range(len(ids)):
        if live[r]:
            for e in np.flatnonzero(ids[r] >= 0):
                full[r, ids[r, e]] += q[r, e]
    # (what is below binary32's smallest normal value, 2^-126, may be zero)
    d_err = U * np.abs(d) + (np.abs(d) + 2 * f * full) * (p_err + 64 * E * 3) + 2.0 ** -126
    k = 2 * E * (len(W) + 64)
    tol = U * np.abs(want_x) + (d_err + k * np.abs(d)) @ np.abs(W) + 2.0 ** -126
    np.testing.assert_array_equal(np.isnan(f64(dx)).any(1), void)
    assert np.all(np.abs(f64(dx) - want_x)[ok] <= tol[ok] * (1 + U))
    k = 2 * E * (len(X) + 64)
    tol = U * np.abs(want_w) + (d_err + k * np.abs(d)).T @ np.abs(X) + 2.0 ** -126
    assert np.all(np.abs(f64(dw) - want_w) <= tol * (1 + U))
    return outs + (dx, dw)


SIZES = [(1, 97, 128), (2, 1, 8), (7, 500, 64), (33, 256, 72), (64, 513, 104), (65, 1031, 1000),
         (256, 300, 320), (257, 1030, 192), (300, 5003, 64), (130, 777, 2056)]


@pytest.mark.parametrize("rows,vocab,hidden", SIZES)
@pytest.mark.parametrize("entries", [None, 1, 20])
def test_scores_and_gradients(rows, vocab, hidden, entries):
    rng = np.random.default_rng([rows, vocab, hidden, entries or 0])
    check(*make(rng, rows, vocab, hidden, entries), float(rng.choice([1.0, 0.5, 1.7])))


@pytest.mark.parametrize("rows,vocab,hidden", [(1, 97, 5), (3, 50, 1), (40, 300, 63), (70, 600, 1001),
                                               (259, 511, 130)])
@pytest.mark.parametrize("entries", [None, 7])
def test_odd_widths_strides_and_alignments(rows, vocab, hidden, entries):
    """Rows that start anywhere, between NaN that no row holds."""
    rng = np.random.default_rng([hidden, entries or 0])
    args = make(rng, rows, vocab, hidden, entries, stride=hidden + int(rng.integers(1, 9)),
                at=int(rng.integers(1, 8)))
    check(*args, 1.0)


@pytest.mark.parametrize("rows,vocab,hidden", [
    (1, 20000, 64), (17, 16400, 200), (64, 20001, 72), (65, 17000, 64), (128, 16385, 136),   # streamed
    (70, 900, 72), (128, 16384, 64), (128, 33, 264),                                         # in rings
    (129, 40001, 64), (260, 30000, 72)])                                                     # large tiles
@pytest.mark.parametrize("entries", [None, 5])
def test_large_and_small_vocabularies(rows, vocab, hidden, entries):
    rng = np.random.default_rng([rows, vocab])
    check(*make(rng, rows, vocab, hidden, entries), 1.0)


@pytest.mark.parametrize("rows,vocab,hidden", [(1500, 100003, 64), (1500, 100003, 65), (5000, 30000, 72)])
def test_vocabularies_of_several_pieces(rows, vocab, hidden):
    """Gradients of logits beyond what a call holds at a time, against the formula
    in 64 bits on the card."""
    rng = np.random.default_rng([rows, hidden])
    x, w, ids, _, grad = make(rng, rows, vocab, hidden)
    head, t, g = Head(w), dev(ids[:, 0], torch.int64), dev(grad, torch.float32)
    logp, lse = head.score(x, t)
    dx, dw = head.score_gradient(x, t, logp, lse, g)
    live, X, W = t >= 0, x.double(), w.double()
    z = X @ W.t()
    want = torch.logsumexp(z, -1)
    s = X.abs().amax() * W.abs().sum(1).amax()           # no product's sizes add up to more
    z_err = (2 * E * hidden + 4 * E) * s
    assert ((lse - want).abs()[live] <= z_err + 200 * E + 8 * E * s + 4 * E * want.abs()[live]).all()
    d = z.sub_(want[:, None]).exp_()
    d[torch.arange(rows, device="cuda"), t.clamp(min=0)] -= 1
    d *= torch.where(live, -g.double(), 0.0)[:, None]
    full = torch.zeros_like(d)
    full[torch.arange(rows, device="cuda"), t.clamp(min=0)] = torch.where(live, g.double().abs(), 0.0)
    p_err = 2 * z_err + 12 * E * s + 300 * E + 8 * E * want.abs().amax()
    d_err = U * d.abs() + (d.abs() + 2 * full) * p_err + 2.0 ** -126
    for got, ref, size, n in ((dx, d @ W, lambda a: a @ W.abs(), vocab),
                              (dw, d.t() @ X, lambda a: a.t() @ X.abs(), rows)):
        tol = U * ref.abs() + size(d_err) + 2 * E * (n + 64) * size(d.abs()) + 2.0 ** -126
        assert ((got.double() - ref).abs() <= tol * (1 + U)).all()


@pytest.mark.parametrize("rows", [3, 64, 65, 300])
def test_aligned_rows_between_others(rows):
    rng = np.random.default_rng(rows)
    check(*make(rng, rows, 400, 128, None, stride=144, at=8), 1.0)
    check(*make(rng, rows, 400, 128, 5, stride=144, at=8), 1.0)


@pytest.mark.parametrize("rows", [5, 64, 100, 600])
@pytest.mark.parametrize("entries", [None, 6])
def test_rows_without_ids_reach_nothing(rows, entries):
    """Dead rows hold NaN and infinities: results zero, gradients zero, and no
    other row's or the head's differ by a bit from those without them."""
    rng = np.random.default_rng([rows, entries or 0])
    x, w, ids, teacher, grad = make(rng, rows, 700, 136, entries, masked=0.6)
    dead = (ids < 0).all(1)
    assert dead.any() and not dead.all()
    outs = check(x, w, ids, teacher, grad, 1.0)
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[dev(dead, torch.bool)] = bad
        g = grad.copy()
        g[dead] = bad
        t = None if teacher is None else np.where(ids < 0, np.float32(bad), teacher)
        again = check(y, w, ids, t, g, 1.0)
        for a, b in zip(outs, again):
            assert torch.equal(a, b)
    for out in outs[:-1]:
        assert not out[dev(dead, torch.bool)].any()


@pytest.mark.parametrize("rows", [1, 64, 129])
@pytest.mark.parametrize("entries", [None, 3])
def test_no_row_has_an_id(rows, entries):
    rng = np.random.default_rng(rows)
    x, w, ids, teacher, grad = make(rng, rows, 333, 64, entries)
    ids[:] = -1
    for out in check(x, w, ids, teacher, grad, 1.0):
        assert not out.any()


@pytest.mark.parametrize("rows", [4, 90])
@pytest.mark.parametrize("entries", [None, 4])
def test_ids_past_the_vocabulary_are_reported(rows, entries):
    rng = np.random.default_rng(rows)
    x, w, ids, teacher, grad = make(rng, rows, 100, 64, entries)
    ids[1, -1], ids[3, 0] = 100, 1 << 40
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(x, w, ids, teacher, grad, 1.0, status=status)
    assert status.item() == ES_HEAD_BAD_ID
    status.zero_()
    ids[ids >= 100] = 99
    check(x, w, ids, teacher, grad, 1.0, status=status)
    assert status.item() == 0


def test_a_teacher_that_leaves_nothing_and_repeated_ids():
    rng = np.random.default_rng(5)
    x, w, ids, teacher, grad = make(rng, 70, 200, 96, 9, masked=0.0)
    teacher[3] = -np.inf
    teacher[4, 2:] = -np.inf
    ids[6] = 17
    ids[7, :4] = ids[7, 5]
    loss, logp, lse, dx, dw = check(x, w, ids, teacher, grad, 1.0)
    assert loss[3].item() == 0.0 and not dx[3].any() and lse[3].item() != 0.0
    assert torch.equal(logp[6], logp[6, :1].expand(9))


def test_a_student_that_is_the_teacher():
    """Where every id is given and the teacher's logits are the student's, the
    divergence is a sum of terms that cancel and its gradient nearly nothing."""
    rng = np.random.default_rng(6)
    x, w, _, _, grad = make(rng, 80, 200, 64)
    ids = np.stack([rng.permutation(200) for _ in range(80)])
    z = f64(x) @ f64(w).T
    teacher = np.take_along_axis(z, ids, 1).astype(np.float32)
    loss, *_ = check(x, w, ids, teacher, grad, 1.0)
    assert loss.abs().max().item() <= 1e-5


@pytest.mark.parametrize("rows", [3, 100])
def test_wide_logits(rows):
    """Logits of some thousands: one token has all of the weight, or none."""
    rng = np.random.default_rng(7)
    x, w, ids, teacher, grad = make(rng, rows, 500, 64, None, std=3000.0)
    z = f64(x) @ f64(w).T
    ids[:rows // 2, 0] = z.argmax(1)[:rows // 2]
    logp, lse, *_ = check(x, w, ids, teacher, grad, 1.0)
    assert torch.isfinite(logp).all() and torch.isfinite(lse).all()


def test_rows_that_are_not_finite_are_nan_alone():
    rng = np.random.default_rng(8)
    x, w, ids, _, _ = make(rng, 300, 500, 64, masked=0.0)
    t = dev(ids[:, 0], torch.int64)
    want = Head(w).score(x, t)
    x[5, 3], x[299, 0] = float("nan"), float("inf")
    got = Head(w).score(x, t)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[5, 299]] = False
    for a, b in zip(got, want):
        assert torch.isnan(a[~keep]).all() and torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("entries", [None, 5])
def test_gradients_against_differences(entries):
    """The gradient along a direction against the outputs' difference over it, both
    from the kernels: the gradient's roundings (U of sum |d w| |v|) and the loss's
    binary32 errors over the step."""
    rng = np.random.default_rng(9)
    x, w, ids, teacher, grad = make(rng, 40, 300, 64, entries, masked=0.1)
    head = Head(w)
    d_ids = dev(ids if entries else ids[:, 0], torch.int64)
    t = dev(teacher, torch.float32) if entries else None
    g = dev(grad, torch.float32)

    def out(h, y):
        if entries:
            loss, logp, lse = h.distill(y, d_ids, t)
            return loss, logp, lse
        logp, lse = h.score(y, d_ids)
        return logp, logp, lse

    o, logp, lse = out(head, x)
    args = (d_ids, t, logp, lse, g) if entries else (d_ids, logp, lse, g)
    dx, dw = (head.distill_gradient if entries else head.score_gradient)(x, *args)
    h = 2.0 ** -4                                          # steps that bf16 inputs take exactly
    for _ in range(3):
        for at, grads in ((x, dx), (w, dw)):
            v = torch.from_numpy(rng.integers(-1, 2, tuple(at.shape)).astype(np.float32)).cuda()
            step = h * at.abs().max().item() * 2.0 ** -3
            up, down = (at.float() + step * v).bfloat16(), (at.float() - step * v).bfloat16()
            real = (up.double() - down.double())
            if at is x:
                hi, lo = out(head, up)[0], out(head, down)[0]
            else:
                hi, lo = out(Head(up), x)[0], out(Head(down), x)[0]
            diff = ((hi.double() - lo.double()) * g.double()).sum().item()
            got = (grads.double() * real).sum().item()
            scale = (grads.double().abs() * real.abs()).sum().item()
            # second differences cancel; the third's share of a step of a 50th of the logits' spread
            assert abs(diff - got) <= (2 * U + 0.02) * scale


def test_only_the_wanted_gradients():
    rng = np.random.default_rng(10)
    x, w, ids, _, grad = make(rng, 50, 400, 64)
    head, t, g = Head(w), dev(ids[:, 0], torch.int64), dev(grad, torch.float32)
    logp, lse = head.score(x, t)
    dx, dw = head.score_gradient(x, t, logp, lse, g)
    assert head.score_gradient(x, t, logp, lse, g, weight_grad=False)[1] is None
    assert torch.equal(head.score_gradient(x, t, logp, lse, g, weight_grad=False)[0], dx)
    only = head.score_gradient(x, t, logp, lse, g, hidden_grad=False)
    assert only[0] is None and torch.equal(only[1], dw)
    assert head.score_gradient(x, t, logp, lse, g, hidden_grad=False, weight_grad=False) == (None, None)


def test_no_rows():
    w = torch.randn(100, 64, device="cuda").bfloat16()
    x, t = w[:0], torch.zeros(0, dtype=torch.int64, device="cuda")
    head = Head(w)
    logp, lse = head.score(x, t)
    assert logp.shape == lse.shape == (0,)
    e = torch.zeros(0, device="cuda")
    dx, dw = head.score_gradient(x, t, logp, lse, e)
    assert dx.shape == (0, 64) and dw.shape == w.shape and not dw.any()
    loss, logp, lse = head.distill(x, t.view(0, 1), e.view(0, 1))
    assert loss.shape == (0,) and logp.shape == (0, 1)


def test_the_same_bits_every_time_and_under_a_graph():
    """Replays among eager calls of the same and of other sizes, new inputs in place."""
    rng = np.random.default_rng(11)
    x, w, ids, teacher, grad = make(rng, 130, 900, 192, 6)
    head = Head(w)
    t, q, g = dev(ids, torch.int64), dev(teacher, torch.float32), dev(grad, torch.float32)

    def step():
        loss, logp, lse = head.distill(x, t, q, scale=0.5)
        return (loss, logp, lse) + head.distill_gradient(x, t, q, logp, lse, g, scale=0.5)

    want = [o.clone() for o in step()]
    for _ in range(3):
        for a, b in zip(step(), want):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for round_ in range(4):
        y, _, ids2, teacher2, grad2 = make(rng, 130, 900, 192, 6, masked=0.3 * round_)
        x.copy_(y)
        t.copy_(dev(ids2, torch.int64))
        q.copy_(dev(teacher2, torch.float32))
        g.copy_(dev(grad2, torch.float32))
        want = [o.clone() for o in step()]
        for o in outs:
            o.fill_(7.0)
        Head(w[:77]).score(x[:9], t[:9, 0].clamp(max=76))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    """A workspace each: calls on one head overlap without a trace."""
    rng = np.random.default_rng(12)
    sets = [make(rng, n, 3000, 256, None) for n in (70, 300)]
    w = sets[0][1]
    head = Head(w)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    args = [(x, dev(ids[:, 0], torch.int64), dev(grad, torch.float32)) for x, _, ids, _, grad in sets]
    want = []
    for x, t, g in args:
        logp, lse = head.score(x, t)
        want.append((logp, lse) + head.score_gradient(x, t, logp, lse, g))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (x, t, g) in enumerate(args):
            logp, lse = head.score(x, t, stream=streams[i])
            grads = head.score_gradient(x, t, logp, lse, g, stream=streams[i])
            got[i].append((logp, lse) + grads)
    torch.cuda.synchronize()
    for i in range(2):
        for outs in got[i]:
            for a, b in zip(outs, want[i]):
                assert torch.equal(a, b)


def test_refusals():
    w = torch.zeros(100, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    head = Head(w)
    f = torch.zeros(4, device="cuda")
    for call in (lambda: Head(w.float()), lambda: Head(w.cpu()), lambda: Head(w.t()),
                 lambda: Head(w[:0]), lambda: Head(w[None]), lambda: Head(w[:1].expand(5, 64)),
                 lambda: head.score(x.float(), t), lambda: head.score(x[:, :32], t),
                 lambda: head.score(x, t.int()), lambda: head.score(x, t[:3]),
                 lambda: head.score(x, t[:, None]), lambda: head.score(x, t.cpu()),
                 lambda: head.score(x.cpu(), t), lambda: head.score(x[0], t[:1]),
                 lambda: head.score(x[:, ::2], t),
                 lambda: head.distill(x, t, f), lambda: head.distill(x, t[:, None], f),
                 lambda: head.distill(x, t[:, None], f[:, None].double()),
                 lambda: head.score_gradient(x, t, f[:3], f, f),
                 lambda: head.score_gradient(x, t, f, f, f.double()),
                 lambda: head.score(x, t, status=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: head.score(x, t, scale=float("nan")),
                 lambda: head.score(x, t, scale=float("inf")),
                 lambda: head.distill(x, t[:, None].expand(4, 257).contiguous(),
                                      torch.zeros(4, 257, device="cuda")),
                 lambda: head.distill(x, t[:, None][:, :0].contiguous(), f[:, None][:, :0].contiguous())):
        with pytest.raises(esopt.EsError):
            call()


@pytest.mark.parametrize("entries", [1, 6])
@pytest.mark.parametrize("rows", [9, 140])
def test_rows_whose_teacher_leaves_nothing(rows, entries):
    """Their loss and their gradient are 0, and what x holds there reaches nothing: the
    others' are those of a call without them."""
    rng = np.random.default_rng([rows, entries])
    x, w, ids, teacher, grad = make(rng, rows, 300, 128, entries, masked=0.0)
    ids[:, 0] = rng.integers(0, 300, rows)                 # every row has one
    empty = rng.random(rows) < 0.4
    empty[1] = True
    teacher[empty] = -np.inf
    x[torch.from_numpy(empty).cuda()] = float("nan")
    head, d_t, d_grad = Head(w), dev(teacher, torch.float32), dev(grad, torch.float32)
    got = []
    for i in (ids, np.where(empty[:, None], -1, ids)):
        d_ids = dev(i, torch.int64)
        loss, logp, lse = head.distill(x, d_ids, d_t)
        got.append((loss,) + head.distill_gradient(x, d_ids, d_t, logp, lse, d_grad))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    assert not got[0][0][torch.from_numpy(empty).cuda()].any()


@pytest.mark.parametrize("scale", [0.0, -0.5])
def test_a_teachers_infinities_at_any_scale(scale):
    """-infinity leaves an id no weight: the divergence without it."""
    rng = np.random.default_rng(31)
    x, w, ids, teacher, grad = make(rng, 40, 300, 128, 6, masked=0.0)
    ids = np.abs(ids) % 300
    teacher[:, 2] = -np.inf
    teacher[5] = -np.inf
    without = np.where(np.isneginf(teacher), -1, ids)
    head, d_t = Head(w), dev(teacher, torch.float32)
    loss, logp, lse = head.distill(x, dev(ids, torch.int64), d_t, scale=scale)
    assert torch.equal(loss, head.distill(x, dev(without, torch.int64), d_t, scale=scale)[0])
    assert loss.isfinite().all() and loss[5] == 0
    for t in head.distill_gradient(x, dev(ids, torch.int64), d_t, logp, lse, dev(grad, torch.float32),
                                   scale=scale):
        assert t.isfinite().all()


@pytest.mark.parametrize("entries", [None, 1, 5])
@pytest.mark.parametrize("rows", [511, 512, 513, 700])
def test_lists_of_rows(rows, entries):
    """Live rows among dead and void ones, where their list has a launch of its own and
    where it has none."""
    rng = np.random.default_rng([rows, entries or 0])
    args = make(rng, rows, 200, 64, entries, masked=0.5)
    args[2][rng.random(rows) < 0.1, 0] = 200
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(*args, 1.0, status)
    assert status.item() == ES_HEAD_BAD_ID


@pytest.mark.parametrize("entries", [None, 2])
def test_more_rows_than_a_list_takes_at_a_time(entries):
    rng = np.random.default_rng(20001)
    check(*make(rng, 20001, 70, 16, entries, masked=0.3), 1.0)


@pytest.mark.parametrize("vocab", [16400, 25000, 40003, 48000, 56001, 65000, 80009])
@pytest.mark.parametrize("rows,hidden,entries", [(2, 72, None), (33, 40, 3), (96, 64, None), (97, 8, None)])
def test_streams_of_any_number_of_waves(vocab, rows, hidden, entries):
    rng = np.random.default_rng([vocab, rows])
    check(*make(rng, rows, vocab, hidden, entries), 1.0)


@pytest.mark.parametrize("vocab", [300, 20000])
@pytest.mark.parametrize("entries", [None, 4])
def test_a_row_out_of_a_larger_array(vocab, entries):
    """The last token of one long sequence: its row stride is beyond what several rows may have."""
    rng = np.random.default_rng(vocab)
    x, w, ids, teacher, grad = make(rng, 1, vocab, 2056, entries, masked=0.0)
    ids[:, 0] = 7
    room = torch.empty(1, 2200, 2056, device="cuda").bfloat16()
    room[:, -1] = x
    assert room[:, -1].stride(0) > 1 << 22
    for a, b in zip(check(room[:, -1], w, ids, teacher, grad, 1.0), check(x, w, ids, teacher, grad, 1.0)):
        assert torch.equal(a, b)


def test_a_head_of_one_token():
    rng = np.random.default_rng(41)
    for rows in (3, 70, 200):
        x, w, ids, _, grad = make(rng, rows, 1, 264)
        column = w.view(264, 1).clone()
        for a, b in zip(check(x, column.t(), ids, None, grad, 1.0), check(x, w, ids, None, grad, 1.0)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [5, 70, 128, 129, 300])
@pytest.mark.parametrize("vocab,hidden", [(500, 72), (501, 200), (20001, 72), (40003, 136), (300, 1001)])
def test_an_infinity_in_the_head(rows, vocab, hidden):
    """A token whose logit is -infinity: the scores and the other columns of the rows' gradient
    are those of a head that has the type's largest number there (its logit's exponential
    is 0 as well), and in the infinity's own column a row whose target the token is has the
    infinity that its definition gives.  The infinity stands where the sums' last parts begin."""
    rng = np.random.default_rng([rows, vocab, hidden])
    x, w, ids, _, grad = make(rng, rows, vocab, hidden, masked=0.0)
    at, token = (hidden - 1) // 64 * 64, vocab - 1
    x[:, at] = -1.0
    ids[ids == token] = 0
    grad[1] = 0.75
    outs = []
    for value, target in ((float("inf"), 3), (3.3895e38, 3), (float("inf"), token)):
        w[token, at] = value
        ids[1] = target
        t = dev(ids[:, 0], torch.int64)
        logp, lse = Head(w).score(x, t)
        dx, _ = Head(w).score_gradient(x, t, logp, lse, dev(grad, torch.float32), weight_grad=False)
        outs.append((logp, lse, dx))
    (logp, lse, dx), (logp2, lse2, dx2), (logp3, lse3, dx3) = outs
    assert torch.isfinite(lse).all() and torch.equal(lse, lse2) and torch.equal(logp, logp2)
    keep = torch.arange(hidden, device="cuda") != at
    assert torch.equal(dx[:, keep], dx2[:, keep])
    assert torch.equal(lse3, lse) and logp3[1] == -float("inf") and dx3[1, at] == float("inf")


@pytest.mark.parametrize("rows", [1, 5, 70, 129, 300])
@pytest.mark.parametrize("vocab,hidden", [(500, 64), (501, 200), (40003, 136)])
@pytest.mark.parametrize("entries", [None, 4])
def test_an_infinity_in_the_head_and_its_gradient(rows, vocab, hidden, entries):
    """A token whose logit is -infinity has no gradient, and the others have theirs: those
    of a head that has the type's largest number there."""
    rng = np.random.default_rng([rows, vocab])
    x, w, ids, teacher, grad = make(rng, rows, vocab, hidden, entries, masked=0.3)
    x[:, 3] = -1.0
    ids[ids == 11] = 12
    head = Head(w)
    d_ids, d_grad = dev(ids if entries else ids[:, 0], torch.int64), dev(grad, torch.float32)
    got = []
    for value in (float("inf"), 3.3895e38):
        w[11, 3] = value
        if entries:
            t = dev(teacher, torch.float32)
            _, logp, lse = head.distill(x, d_ids, t)
            got.append(head.distill_gradient(x, d_ids, t, logp, lse, d_grad, hidden_grad=False)[1])
        else:
            logp, lse = head.score(x, d_ids)
            got.append(head.score_gradient(x, d_ids, logp, lse, d_grad, hidden_grad=False)[1])
    assert torch.isfinite(got[0]).all() and torch.equal(*got) and not got[0][11].any()


@pytest.mark.parametrize("scale", [1.4, 1.0, 0.5, 0.0, -1.5])
@pytest.mark.parametrize("rows", [7, 140])
def test_a_teachers_largest_numbers(rows, scale):
    """Masks of the type's lowest value throughout leave equal weights, and so does its highest;
    one above the other leaves one entry all of them, or none: the results are those of
    small logits that do."""
    rng = np.random.default_rng([rows, 43])
    x, w, _, _, grad = make(rng, rows, 300, 128)
    ids = np.stack([rng.permutation(300)[:5] for _ in range(rows)])
    far = np.tile(np.arange(5, dtype=np.float32) / 4, (rows, 1))
    near = far.copy()
    low, most = np.finfo(np.float32).min, np.finfo(np.float32).max
    far[1::4], near[1::4] = low, 0
    far[2::4], near[2::4] = most, 0
    far[3::4], near[3::4] = low, -np.inf if scale > 0 else 0
    far[3::4, 2], near[3::4, 2] = most, -np.inf if scale < 0 else 0
    head, d_ids, d_grad = Head(w), dev(ids, torch.int64), dev(grad, torch.float32)
    got = []
    for t in (far, near):
        d_t = dev(t, torch.float32)
        loss, logp, lse = head.distill(x, d_ids, d_t, scale=scale)
        got.append((loss,) + head.distill_gradient(x, d_ids, d_t, logp, lse, d_grad, scale=scale))
    for a, b in zip(*got):
        assert a.isfinite().all() and torch.equal(a, b)


@pytest.mark.parametrize("scale", [0.7, 0.0, -0.7])
@pytest.mark.parametrize("rows,entries", [(7, 1), (7, 5), (140, 70), (600, 1), (600, 3)])
def test_a_teacher_that_is_no_number(rows, entries, scale):
    """Such a row's loss and its logits' gradients are NaN, the rows' gradients beside it are
    those without it, and the head's is NaN throughout, as its definition gives."""
    rng = np.random.default_rng([rows, entries])
    x, w, _, _, grad = make(rng, rows, 300, 64)
    ids = rng.integers(0, 300, (rows, entries))
    clean = rng.standard_normal(ids.shape).astype(np.float32)
    head, d_grad = Head(w), dev(grad, torch.float32)

    def run(i, t):
        d_ids, d_t = dev(i, torch.int64), dev(t, torch.float32)
        loss, logp, lse = head.distill(x, d_ids, d_t, scale=scale)
        return (loss, logp, lse) + head.distill_gradient(x, d_ids, d_t, logp, lse, d_grad, scale=scale)
    want = run(ids, clean)
    for value in (np.nan, np.inf):
        t = clean.copy()
        t[1, 0] = value
        loss, logp, lse, dx, dw = run(ids, t)
        # an infinity at a scale below 0 has no weight
        lost = np.isnan(value) or scale >= 0
        with np.errstate(invalid="ignore"):
            W, X = f64(w), f64(x)
            assert np.isnan(oh.gradients(X, W, ids, grad, scale, t.astype(np.float64))[1]).all() == lost
        assert torch.isnan(loss[1]) == lost and torch.isnan(dx[1]).all() == lost
        assert torch.isnan(dw).all() == lost and torch.isnan(dw).any() == lost
        others = torch.arange(rows, device="cuda") != 1
        assert torch.equal(loss[others], want[0][others]) and torch.equal(dx[others], want[3][others])
        assert torch.equal(logp, want[1]) and torch.equal(lse, want[2])
        if entries > 1:                                    # absent, it is not looked at
            gone = ids.copy()
            gone[1, 0] = -1
            for a in run(gone, t):
                assert torch.isfinite(a).all()


@pytest.mark.parametrize("rows", [1, 33, 70, 129, 300])
@pytest.mark.parametrize("vocab,hidden", [(500, 72), (501, 64), (20001, 72), (40003, 136), (300, 63)])
def test_a_logit_of_infinity(rows, vocab, hidden):
    """Its row's results are NaN, as the differences of infinities that define them are; rows where
    that logit is -infinity are finite."""
    rng = np.random.default_rng([rows, vocab])
    x, w, ids, _, _ = make(rng, rows, vocab, hidden, masked=0.0)
    ids[ids == 7] = 8
    w[7, 5] = float("inf")
    x[:, 5] = torch.where(torch.arange(rows, device="cuda") % 3 == 1, -1.0, 1.0)
    up = x[:, 5] > 0
    logp, lse = Head(w).score(x, dev(ids[:, 0], torch.int64))
    loss, *_ = Head(w).distill(x, dev(ids, torch.int64), torch.zeros(rows, 1, device="cuda"))
    for out in (logp, lse, loss):
        assert torch.equal(torch.isnan(out), up) and torch.isfinite(out[~up]).all()


@pytest.mark.parametrize("scale", [1.0, 0.5])
@pytest.mark.parametrize("rows,vocab,hidden", [(1, 20001, 8), (40, 20001, 8), (100, 20001, 8), (3, 500, 8),
                                               (70, 500, 8), (33, 500, 7), (200, 500, 8), (300, 40003, 8)])
def test_normalisers_of_large_logits(rows, vocab, hidden, scale):
    """Integers, whose logits of some thousands are exact: a normaliser is off by its own rounding
    and by its sum's errors alone (as in `slack`)."""
    rng = np.random.default_rng([rows, vocab])
    x, w = (torch.from_numpy(rng.integers(-90, 91, (n, hidden)).astype(np.float32)).cuda().bfloat16()
            for n in (rows, vocab))
    t = torch.from_numpy(rng.integers(0, vocab, rows)).cuda()
    logp, lse = Head(w).score(x, t, scale=scale)
    z = x.double() @ w.double().t() * scale
    want = torch.logsumexp(z, -1)
    assert want.amax() > 3000
    assert ((lse - want).abs() <= E * want.abs() + 2 * E * 64 + 100 * E).all()
    got = z.gather(1, t[:, None])[:, 0] - want
    assert ((logp - got).abs() <= E * (want.abs() + got.abs()) + 2 * E * 64 + 100 * E).all()


@pytest.mark.parametrize("rows,vocab,hidden", [(3, 500, 200), (40, 500, 1001), (100, 20001, 64), (64, 20001, 2056),
                                               (300, 700, 2056)])
def test_no_probability_is_above_one(rows, vocab, hidden):
    """Targets with all of the weight, at logits of some thousands, whose sums round."""
    rng = np.random.default_rng([rows, hidden])
    x, w, _, _, _ = make(rng, rows, vocab, hidden, masked=0.0, std=1000.0)
    z = x.double() @ w.double().t()
    t = z.argmax(1)
    logp, lse = Head(w).score(x, t)
    sure = torch.logsumexp(z, -1) - z.amax(1) == 0
    assert sure.sum() > rows // 2
    assert (logp <= 0).all() and not torch.isnan(logp).any()
    loss, logp, _ = Head(w).distill(x, t[:, None], torch.zeros(rows, 1, device="cuda"))
    assert (logp <= 0).all() and (loss >= 0).all()


def check_on_the_card(x, w, ids, grad):
    """Scores and gradients without a teacher against the formula in 64 bits on the card, with the
    bounds of test_vocabularies_of_several_pieces."""
    rows, vocab, hidden = len(x), len(w), x.shape[1]
    assert -(-vocab // 128) * -(-rows // 128) > 512        # (so many small tiles are large ones)
    head, t, g = Head(w), dev(ids[:, 0], torch.int64), dev(grad, torch.float32)
    logp, lse = head.score(x, t)
    dx, dw = head.score_gradient(x, t, logp, lse, g)
    live, X, W = t >= 0, x.double(), w.double()
    here = torch.arange(rows, device="cuda")
    z = X @ W.t()
    want = torch.logsumexp(z, -1)
    s = X.abs().amax() * W.abs().sum(1).amax()
    z_err = (2 * E * hidden + 4 * E) * s
    norm = 200 * E + 8 * E * s
    assert ((lse - want).abs()[live] <= z_err + norm + 4 * E * want.abs()[live]).all()
    right = z[here, t.clamp(min=0)] - want
    assert ((logp - right).abs()[live] <= 2 * z_err + norm + 8 * E * (want.abs() + right.abs())[live]).all()
    assert not lse[~live].any() and not logp[~live].any()
    d = z.sub_(want[:, None]).exp_()
    d[here, t.clamp(min=0)] -= 1
    d *= torch.where(live, -g.double(), 0.0)[:, None]
    full = torch.zeros_like(d)
    full[here, t.clamp(min=0)] = torch.where(live, g.double().abs(), 0.0)
    p_err = 2 * z_err + 12 * E * s + 300 * E + 8 * E * want.abs().amax()
    d_err = U * d.abs() + (d.abs() + 2 * full) * p_err + 2.0 ** -126
    for got, ref, size, n in ((dx, d @ W, lambda a: a @ W.abs(), vocab),
                              (dw, d.t() @ X, lambda a: a.t() @ X.abs(), rows)):
        tol = U * ref.abs() + size(d_err) + 2 * E * (n + 64) * size(d.abs()) + 2.0 ** -126
        assert ((got.double() - ref).abs() <= tol * (1 + U)).all()


@pytest.mark.parametrize("rows,vocab,hidden", [(700, 40003, 520), (700, 40003, 1001), (1100, 20000, 2056)])
def test_long_sums_in_large_tiles(rows, vocab, hidden):
    """Tiles of 256 x 256 whose sums have many stages, for the logits, both gradients and (over the
    live rows) the head's: rings that wrap, and ends in the middle of a stage."""
    rng = np.random.default_rng([rows, hidden, 47])
    x, w, ids, _, grad = make(rng, rows, vocab, hidden, masked=0.2)
    check_on_the_card(x, w, ids, grad)


@pytest.mark.parametrize("rows,hidden", [(129, 136), (191, 192), (192, 193), (193, 200), (256, 256), (257, 264),
                                         (319, 320), (320, 328), (321, 384), (384, 385), (385, 448)])
def test_every_number_of_stages_in_large_tiles(rows, hidden):
    """Sums of three to eight stages, whole and not: along hidden for the logits, over the rows for
    the head's gradient."""
    rng = np.random.default_rng([rows, hidden, 53])
    x, w, ids, _, grad = make(rng, rows, 33000, hidden, masked=0.0)
    check_on_the_card(x, w, ids, grad)


@pytest.mark.parametrize("entries", [None, 5])
def test_gradients_against_differences_along_themselves(entries):
    """The outputs' difference over a step against the gradient, in directions where it is large:
    a step in a quarter of the places, each to its gradient's side.  Inputs and steps are multiples of
    2^-6, so the logits are exact; what is left is the gradients' rounding (U of a result, and U of
    each d in it), the scores' binary32 errors, and the third difference: of a logarithm of a sum
    of exponentials the third derivative is a third central moment, at most R^3 / (6 sqrt 3) of
    logits whose changes span R.  Along such directions a gradient of another size or sign, or one
    without its softmax, is told apart."""
    rng = np.random.default_rng([59, entries or 0])
    rows, vocab, hidden, step = 40, 300, 64, 2.0 ** -6
    x, w = (torch.from_numpy(rng.integers(-64, 65, (n, hidden)).astype(np.float32) / 64).cuda().bfloat16()
            for n in (rows, vocab))
    _, _, ids, teacher, grad = make(rng, rows, vocab, hidden, entries, masked=0.1)
    d_ids = dev(ids if entries else ids[:, 0], torch.int64)
    t = dev(teacher, torch.float32) if entries else None
    d_grad = dev(grad, torch.float32)

    def out(y, v):
        if entries:
            return Head(v).distill(y, d_ids, t)
        logp, lse = Head(v).score(y, d_ids)
        return logp, logp, lse

    first, logp, lse = out(x, w)
    if entries:
        grads = Head(w).distill_gradient(x, d_ids, t, logp, lse, d_grad)
    else:
        grads = Head(w).score_gradient(x, d_ids, logp, lse, d_grad)
    X, W, T = f64(x), f64(w), None if teacher is None else teacher.astype(np.float64)
    live, _ = oh.kinds(ids, vocab)
    g = np.where(live, np.abs(grad), 0.0)
    d = np.abs(oh.logit_gradients(X, W, ids, grad, 1.0, T))
    # without the softmax: the wanted weights alone
    bare = np.zeros_like(d)
    q, _ = oh.weights(ids, T, 1.0)
    for r in np.flatnonzero(live):
        for e in np.flatnonzero(ids[r] >= 0):
            bare[r, ids[r, e]] += q[r, e] * grad[r] * (-1 if entries else 1)
    error = 2 * E * 64 + 100 * E + 16 * E * (np.abs(f64(lse)) + np.abs(f64(logp)).reshape(rows, -1).max(1))
    for at, G in enumerate(map(f64, grads)):
        v = np.sign(G) * (rng.random(G.shape) < 0.25) * step
        up, down = (dev(a, torch.float32).bfloat16() for a in ((X, W)[at] + v, (X, W)[at] - v))
        assert np.array_equal(f64(up) - f64(down), 2 * v)
        hi, lo = (out(x, y)[0] if at else out(y, w)[0] for y in (up, down))
        diff = ((f64(hi) - f64(lo)) * grad).sum()
        got = (2 * v * G).sum()
        change = X @ v.T if at else v @ W.T
        span = change.max(1) - change.min(1)
        size = d.T @ np.abs(X) if at else d @ np.abs(W)
        tol = (2 * np.abs(v) * U * (np.abs(G) + size) * (1 + U)).sum() + (g * 2 * error).sum() + \
            (g * span ** 3).sum() / (3 * 6 * 3 ** 0.5)
        assert abs(diff - got) <= tol
        without = (2 * v * (bare.T @ X if at else bare @ W)).sum()
        assert tol <= 0.1 * abs(got) and abs(diff - without) > tol


@pytest.mark.parametrize("rows,vocab,hidden", [(30, 300, 64), (90, 20001, 136), (200, 400, 72), (140, 33000, 200)])
def test_rows_that_overlap(rows, vocab, hidden):
    """Windows of a sequence, 8 elements apart, as rows and as a head."""
    rng = np.random.default_rng([rows, 61])
    x, w, ids, _, grad = make(rng, rows, vocab, hidden)
    long, flat = (mat(rng, 1, 8 * n + hidden)[0] for n in (rows, vocab))
    y, v = long.as_strided((rows, hidden), (8, 1)), (flat * hidden ** -0.5).as_strided((vocab, hidden), (8, 1))
    for a, b in ((y, w), (x, v), (y, v)):
        t, g = dev(ids[:, 0], torch.int64), dev(grad, torch.float32)
        outs = []
        for p, q in ((a, b), (a.contiguous(), b.contiguous())):
            logp, lse = Head(q).score(p, t)
            outs.append((logp, lse) + Head(q).score_gradient(p, t, logp, lse, g))
        for got, want in zip(*outs):
            assert torch.equal(got, want)


def test_the_smallest_numbers():
    """Products of bf16's denormal numbers are exact as well."""
    for rows, vocab, hidden in ((3, 200, 64), (3, 200, 63), (40, 20001, 64), (200, 300, 64)):
        x, w = (torch.zeros(n, hidden, device="cuda").bfloat16() for n in (rows, vocab))
        x[:, 1], w[5, 1] = 2.0 ** -130, 2.0 ** 126
        x[:, 2], w[6, 2] = 2.0 ** 125, 3 * 2.0 ** -132
        t = torch.arange(rows, device="cuda") % 3 + 4
        logp, lse = Head(w).score(x, t, scale=8.0)
        z = x[:1].double() @ w.double().t() * 8
        want = torch.logsumexp(z, -1)
        assert z[0, 5] == 0.5 and z[0, 6] == 0.1875
        assert ((lse - want).abs() <= 300 * E).all() and ((logp - z[0, t] + want).abs() <= 300 * E).all()


@pytest.mark.parametrize("rows,hidden", [(2, 2560), (40, 2561), (100, 2560), (300, 2560)])
def test_a_head_beyond_32_bits(rows, hidden):
    """More than 2^32 bytes and 2^31 elements of the head, and of its gradient."""
    rng = np.random.default_rng([rows, 67])
    vocab = 900_001
    w = torch.empty(vocab, hidden, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    for part in w.split(100_000):
        part.copy_(torch.randn(*part.shape, device="cuda", generator=gen) * hidden ** -0.5)
    x = mat(rng, rows, hidden)
    t = torch.from_numpy(rng.integers(0, vocab, rows)).cuda()
    t[0], t[1] = vocab - 1, vocab - 2
    g = dev(rng.standard_normal(rows), torch.float32)
    logp, lse = Head(w).score(x, t)
    X = x.double()
    tops = []
    for part in w.split(100_000):
        tops.append(torch.logsumexp(X @ part.double().t(), -1))
    want = torch.logsumexp(torch.stack(tops), 0)
    s = X.abs().amax() * max(part.double().abs().sum(1).amax() for part in w.split(100_000))
    z_err = (2 * E * hidden + 4 * E) * s
    assert ((lse - want).abs() <= z_err + 200 * E + 8 * E * s + 4 * E * want.abs()).all()
    right = (X * w[t].double()).sum(1) - want
    assert ((logp - right).abs() <= 2 * z_err + 200 * E + 8 * E * (s + want.abs() + right.abs())).all()
    dx, dw = Head(w).score_gradient(x, t, logp, lse, g)
    p_err = 2 * z_err + 12 * E * s + 300 * E + 8 * E * want.abs().amax()
    ref, room, first = torch.zeros_like(X), torch.zeros_like(X), 0
    for part, got in zip(w.split(100_000), dw.split(100_000)):
        P = part.double()
        d = (X @ P.t() - want[:, None]).exp_()
        full = torch.zeros_like(d)
        for r in range(rows):
            if first <= t[r] < first + len(part):
                d[r, t[r] - first] -= 1
                full[r, t[r] - first] = g[r].double().abs()
        d *= -g.double()[:, None]
        d_err = U * d.abs() + (d.abs() + 2 * full) * p_err + 2.0 ** -126
        ref += d @ P
        room += (d_err + 2 * E * (vocab + 64) * d.abs()) @ P.abs()
        to = d.t() @ X
        tol = U * to.abs() + (d_err + 2 * E * (rows + 64) * d.abs()).t() @ X.abs() + 2.0 ** -126
        assert ((got.double() - to).abs() <= tol * (1 + U)).all()
        first += len(part)
    assert ((dx.double() - ref).abs() <= (U * ref.abs() + room) * (1 + U)).all()


@pytest.mark.parametrize("rows,vocab,hidden", [(256, 333, 72), (256, 33000, 136), (512, 301, 200), (512, 20003, 65)])
def test_live_rows_that_fill_their_tiles(rows, vocab, hidden):
    """The last packed row is a live one, and the sums end within a stage."""
    rng = np.random.default_rng([rows, vocab, 79])
    check(*make(rng, rows, vocab, hidden, masked=0.0), 1.0)
