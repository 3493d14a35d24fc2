"""Projections under the low-rank adapters of many members (es_adapt_*), against
the fp64 oracle.

Tolerances are the kernel's roundings: U = 2^-8 of u = s A x (its bf16), whose
binary32 sum is off by 2 E, E = 2^-24, a step of the sum of its products' sizes;
as much of the whole sum; and U of the result.
"""
import numpy as np
import pytest
import torch

from oracle import head as oh
from paper_2608_17310_amd import esopt
from paper_2608_17310_amd.adapters import ES_ADAPT_BAD_INDEX, Adapters

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


def bf16(rng, *shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).cuda().bfloat16()


def ints(x):
    return torch.from_numpy(np.asarray(x)).int().cuda()


def make(rng, rows, inner, outer, rank, members, how="mixed"):
    x, w = bf16(rng, rows, inner), bf16(rng, outer, inner, std=inner ** -0.5)
    a = bf16(rng, members, rank, inner, std=inner ** -0.5)
    b = bf16(rng, members, outer, rank, std=rank ** -0.5)
    scales = torch.from_numpy(rng.uniform(0.5, 3, members).astype(np.float32)).cuda()
    index = {"mixed": lambda: rng.integers(-1, members, rows),
             "runs": lambda: np.sort(rng.integers(-1, members, rows)),
             "each": lambda: np.arange(rows) % members,
             "one": lambda: np.full(rows, members - 1),
             "none": lambda: np.full(rows, -1 - rows)}[how]()
    return x, w, a, b, scales, index


def check(x, w, a, b, scales, index, got):
    X, W, A, B = map(f64, (x, w, a, b))
    S = None if scales is None else f64(scales)
    want = oh.project(X, W, A, B, index, S)
    size = np.abs(X) @ np.abs(W).T
    tol = 2 * E * (X.shape[1] + A.shape[1] + 16) * size
    for r, i in enumerate(index):
        if 0 <= i < len(A):
            s = 1.0 if S is None else S[i]
            u_err = U * np.abs(s * (A[i] @ X[r])) + s * 2 * E * (X.shape[1] + 16) * (
                np.abs(A[i]) @ np.abs(X[r])) * (1 + U)
            low = np.abs(B[i]) @ np.abs(s * (A[i] @ X[r]))
            tol[r] += np.abs(B[i]) @ u_err + 2 * E * (X.shape[1] + A.shape[1] + 16) * low
    tol = tol * (1 + U) + U * np.abs(want) + 2.0 ** -126
    got = f64(got)
    void = index >= len(A)
    np.testing.assert_array_equal(np.isnan(got).any(1), void)
    np.testing.assert_array_equal(np.isnan(got).all(1), void)
    assert np.all(np.abs(got - want)[~void] <= tol[~void])


@pytest.mark.parametrize("rows,inner,outer,rank,members", [
    (1, 64, 64, 8, 1), (1, 1000, 513, 16, 3), (3, 8, 1, 128, 2), (16, 512, 300, 16, 16),
    (17, 136, 100, 24, 5), (33, 1024, 257, 64, 40), (64, 328, 1025, 32, 7), (65, 256, 256, 16, 3),
    (129, 72, 771, 40, 200), (300, 1032, 520, 128, 4), (513, 192, 264, 8, 30),
    (2, 264, 8193, 16, 3), (16, 64, 9001, 24, 16), (20, 136, 8200, 16, 9), (33, 72, 9000, 64, 3),   # many outputs
    (70, 2104, 130, 32, 6), (200, 4096, 257, 16, 5),                                # divided sums
    (1300, 72, 6000, 16, 11), (2100, 64, 4100, 64, 6)])                             # large tiles
@pytest.mark.parametrize("how", ["mixed", "runs", "each", "one", "none"])
def test_project(rows, inner, outer, rank, members, how):
    rng = np.random.default_rng([rows, inner, outer, rank])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, rank, members, how)
    check(x, w, a, b, scales, index, Adapters(a, b, scales).project(x, w, ints(index)))
    if how in ("mixed", "one"):
        check(x, w, a, b, None, index, Adapters(a, b).project(x, w, ints(index)))


@pytest.mark.parametrize("outer", [8193, 16384, 20003, 24000, 28672, 32761, 40000, 70001])
@pytest.mark.parametrize("rows,inner,rank", [(1, 72, 8), (17, 200, 16), (33, 64, 40), (64, 136, 8)])
def test_a_matrix_of_many_rows(outer, rows, inner, rank):
    """Three to eight waves a compute unit, one round and several, shares that end early."""
    rng = np.random.default_rng([rows, outer])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, rank, 3)
    check(x, w, a, b, scales, index, Adapters(a, b, scales).project(x, w, ints(index)))


@pytest.mark.parametrize("rows", [1, 9, 64, 65, 200])
def test_strides_and_outputs(rows):
    """Rows inside wider ones at any alignment; nothing beside the output is written."""
    rng = np.random.default_rng(rows)
    x, w, a, b, scales, index = make(rng, rows, 264, 129, 16, 6)
    wide = bf16(rng, rows, 300)
    wide[:, 7:271] = x
    room = torch.full((rows + 2, 140), 5.0, device="cuda").bfloat16()
    w_room = torch.full((129, 280), float("nan"), device="cuda").bfloat16()
    w_room[:, :264] = w
    out = room[1:-1, 3:132]
    got = Adapters(a, b, scales).project(wide[:, 7:271], w_room[:, :264], ints(index), out=out)
    assert got.data_ptr() == out.data_ptr()
    check(x, w, a, b, scales, index, out)
    kept = room.clone()
    kept[1:-1, 3:132] = 5.0
    assert (kept == 5.0).all()


@pytest.mark.parametrize("rows", [5, 64, 100, 300])
def test_a_member_reaches_its_own_rows_alone(rows):
    """Adapters that have diverged, rows that are not finite."""
    rng = np.random.default_rng(rows)
    x, w, a, b, scales, index = make(rng, rows, 192, 200, 32, 4)
    index[:5] = [-1, 0, 1, 2, 3]
    want = Adapters(a, b, scales).project(x, w, ints(index))
    a2, b2, s2, x2 = a.clone(), b.clone(), scales.clone(), x.clone()
    a2[1, 3], b2[2, 7], s2[3] = float("nan"), float("inf"), float("nan")
    x2[0] = float("inf")
    got = Adapters(a2, b2, s2).project(x2, w, ints(index))
    keep = torch.from_numpy((index <= 0) & (np.arange(rows) > 0)).cuda()
    assert keep.any() and torch.equal(got[keep], want[keep])
    assert not torch.isfinite(got[~keep][:4]).all(1).any()


def test_indexes_past_the_members_are_reported():
    rng = np.random.default_rng(1)
    for rows in (4, 70):
        x, w, a, b, scales, index = make(rng, rows, 64, 100, 8, 3)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        index[1], index[3] = 3, 2 ** 31 - 1
        adapters = Adapters(a, b, scales)
        check(x, w, a, b, scales, index, adapters.project(x, w, ints(index), status=status))
        assert status.item() == ES_ADAPT_BAD_INDEX
        status.zero_()
        index[1] = index[3] = -2 ** 31
        check(x, w, a, b, scales, index, adapters.project(x, w, ints(index), status=status))
        assert status.item() == 0


def test_no_rows_and_one_member_moved_by_a_plan():
    """A member's adapters are tensors of a plan: perturbed and restored, the
    projection follows."""
    rng = np.random.default_rng(2)
    x, w, a, b, scales, index = make(rng, 40, 128, 96, 16, 3)
    adapters = Adapters(a, b, scales)
    assert adapters.project(x[:0], w, ints(index)[:0]).shape == (0, 96)
    before = adapters.project(x, w, ints(index))
    plan = esopt.Plan([a[1], b[1]])
    plan.perturb(7, 1, 1e-2)
    moved = adapters.project(x, w, ints(index))
    check(x, w, a, b, scales, index, moved)
    mine = torch.from_numpy(index == 1).cuda()
    assert torch.equal(moved[~mine], before[~mine]) and not torch.equal(moved[mine], before[mine])
    plan.close()


@pytest.mark.parametrize("rows", [1, 40, 200])
def test_the_same_bits_under_a_graph_and_on_streams(rows):
    rng = np.random.default_rng(3)
    x, w, a, b, scales, index = make(rng, rows, 520, 300, 16, 5)
    adapters, i = Adapters(a, b, scales), ints(index)
    want = adapters.project(x, w, i)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [adapters.project(x, w, i, stream=side) for _ in range(3)]
    again = [adapters.project(x, w, i) for _ in range(3)]
    torch.cuda.synchronize()
    for y in got + again:
        assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = adapters.project(x, w, i)
    for k in range(3):
        x.copy_(bf16(rng, rows, 520))
        i.copy_(ints(rng.integers(-1, 5, rows)))
        want = adapters.project(x, w, i)
        out.zero_()
        Adapters(a[:2], b[:2]).project(x[:1], w, i[:1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals():
    rng = np.random.default_rng(4)
    x, w, a, b, scales, index = make(rng, 4, 64, 96, 16, 3)
    i = ints(index)
    adapters = Adapters(a, b, scales)
    wide = bf16(rng, 96, 72)
    for call in (lambda: Adapters(a.float(), b), lambda: Adapters(a.cpu(), b), lambda: Adapters(a[0], b),
                 lambda: Adapters(a, b[:2]), lambda: Adapters(a, b[:, :, :8].contiguous()),
                 lambda: Adapters(a[:, :4].contiguous(), b[:, :, :4].contiguous()),
                 lambda: Adapters(a[:0], b[:0]), lambda: Adapters(a.transpose(1, 2), b),
                 lambda: Adapters(a, b, scales[:2]), lambda: Adapters(a, b, scales.double()),
                 lambda: adapters.project(x[:, :32], w, i), lambda: adapters.project(x.float(), w, i),
                 lambda: adapters.project(x, w[:50], i), lambda: adapters.project(x, w.t(), i),
                 lambda: adapters.project(x, w, i.long()), lambda: adapters.project(x, w, i[:3]),
                 lambda: adapters.project(x, w, i, out=torch.empty(4, 96, device="cuda")),
                 lambda: adapters.project(x, w, i, out=bf16(rng, 4, 95))):
        with pytest.raises(ValueError):
            call()
    odd = torch.empty(96 * 64 + 1, device="cuda").bfloat16()[1:].view(96, 64)
    for call in (lambda: adapters.project(x, odd, i),
                 lambda: adapters.project(x, wide.view(-1)[:96 * 68].view(96, 68)[:, :64], i),
                 lambda: Adapters(a[:, :, :60].contiguous(), b).project(x[:, :60], w[:, :60], i)):
        with pytest.raises(esopt.EsError):
            call()


@pytest.mark.parametrize("rows", [1, 20, 40, 70, 300])
def test_a_matrix_of_one_row(rows):
    """Its row stride means nothing: a column of words that are two bytes apart, seen as a row."""
    rng = np.random.default_rng(rows)
    x, w, a, b, scales, index = make(rng, rows, 264, 1, 16, 3)
    column = w.view(264, 1).clone()
    assert column.t().stride() == (1, 1)
    adapters = Adapters(a, b, scales)
    got = adapters.project(x, column.t(), ints(index))
    check(x, w, a, b, scales, index, got)
    assert torch.equal(got, adapters.project(x, w, ints(index)))


def test_a_row_out_of_a_larger_array():
    """One row, whose stride is beyond what several may have."""
    rng = np.random.default_rng(6)
    x, w, a, b, scales, index = make(rng, 1, 4104, 100, 16, 2)
    room, out_room = torch.empty(1, 1200, 4104, device="cuda").bfloat16(), torch.empty(1, 50000, 100).bfloat16().cuda()
    room[:, -1], out = x, out_room[:, -1]
    assert min(room[:, -1].stride(0), out.stride(0)) > 1 << 22
    adapters = Adapters(a, b, scales)
    assert adapters.project(room[:, -1], w, ints(index), out=out) is out
    assert torch.equal(out, adapters.project(x, w, ints(index)))


@pytest.mark.parametrize("rows,inner,outer", [(3, 72, 100), (64, 72, 9000), (65, 72, 100), (70, 2104, 130),
                                              (300, 1032, 520), (1300, 72, 6000)])
def test_an_infinity_in_the_weight(rows, inner, outer):
    """It reaches its own output, with the sign of the row's factor, and no other; it stands
    where the sum's last part begins."""
    rng = np.random.default_rng([rows, inner])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, 16, 3)
    at = (inner - 1) // 64 * 64
    assert (x[:, at] != 0).all()
    adapters = Adapters(a, b, scales)
    want = adapters.project(x, w, ints(index))
    w[outer // 2, at] = float("inf")
    got = adapters.project(x, w, ints(index))
    assert torch.equal(got[:, outer // 2], torch.sign(x[:, at]) * float("inf"))
    keep = torch.arange(outer, device="cuda") != outer // 2
    assert torch.equal(got[:, keep], want[:, keep])


@pytest.mark.parametrize("rows,inner,outer", [(1300, 1096, 6000), (1300, 128, 6000), (1290, 136, 6000),
                                              (1300, 192, 6001), (1400, 200, 5900), (1300, 256, 6000),
                                              (1300, 264, 6000), (1300, 320, 6000), (1300, 328, 6100)])
def test_every_number_of_stages_in_large_tiles(rows, inner, outer):
    assert -(-outer // 128) * -(-rows // 128) > 512        # (so many small tiles are large ones)
    rng = np.random.default_rng([rows, inner, outer])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, 24, 7, "runs")
    check(x, w, a, b, scales, index, Adapters(a, b, scales).project(x, w, ints(index)))


@pytest.mark.parametrize("rows,inner,outer,rank,members", [
    (270_000, 64, 8200, 8, 3),                             # more than 2^31 results
    (3, 2560, 900_001, 16, 3), (100, 2560, 900_001, 16, 3),           # elements of the weight
    (40, 64, 17408, 64, 3000), (40, 64, 5120, 128, 6000), (150, 64, 17408, 64, 3000)])   # of all b
def test_arrays_beyond_32_bits(rows, inner, outer, rank, members):
    """Rows among all of them, against 64 bits."""
    rng = np.random.default_rng([rows, outer])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)

    def normal(n, width, std):
        out = torch.empty(n, width, device="cuda", dtype=torch.bfloat16)
        for part in out.split(max(1, (1 << 28) // width)):
            part.copy_(torch.randn(*part.shape, device="cuda", generator=gen) * std)
        return out

    x, w = normal(rows, inner, 1.0), normal(outer, inner, inner ** -0.5)
    a = normal(members, rank * inner, inner ** -0.5).view(members, rank, inner)
    b = normal(members, outer * rank, rank ** -0.5).view(members, outer, rank)
    index = rng.integers(-1, members, rows)
    index[0], index[-1] = members - 1, members - 2
    got = Adapters(a, b).project(x, w, ints(index))
    assert max(got.numel(), w.numel(), b.numel()) > 1 << 31
    for r in [0, rows - 1] + rng.integers(0, rows, 8).tolist():
        X, W = x[r].double(), w.double()
        want, i = W @ X, index[r]
        tol = 2 * E * (inner + rank + 16) * (W.abs() @ X.abs())
        if i >= 0:
            A, B = a[i].double(), b[i].double()
            want += B @ (A @ X)
            u_err = U * (A @ X).abs() + 2 * E * (inner + 16) * (A.abs() @ X.abs()) * (1 + U)
            tol += B.abs() @ u_err + 2 * E * (inner + rank + 16) * (B.abs() @ (A @ X).abs())
        assert ((got[r].double() - want).abs() <= tol * (1 + U) + U * want.abs()).all()


def test_rows_and_results_side_by_side():
    """In the columns of one array; an output over its own input is refused."""
    rng = np.random.default_rng(71)
    for rows in (1, 30, 100, 700):
        x, w, a, b, scales, index = make(rng, rows, 128, 96, 16, 3)
        room = torch.zeros(rows, 224, device="cuda").bfloat16()
        room[:, :128] = x
        adapters = Adapters(a, b, scales)
        adapters.project(room[:, :128], w, ints(index), out=room[:, 128:])
        check(x, w, a, b, scales, index, room[:, 128:])
        assert torch.equal(room[:, :128], x)
        with pytest.raises(esopt.EsError):
            adapters.project(room[:, :128], w, ints(index), out=room[:, 127:223])


PATHS = [(1, 200, 300), (20, 72, 100), (50, 136, 9000), (64, 72, 9000), (70, 2104, 130), (100, 200, 300),
         (300, 136, 520), (1300, 200, 6000)]


@pytest.mark.parametrize("rows,inner,outer", PATHS)
@pytest.mark.parametrize("rank", [8, 16, 24, 128])
def test_the_small_product_is_not_rounded_to_bf16(rows, inner, outer, rank):
    """Without the shared part, of sums that nearly cancel: a result is off by its own rounding, and
    by 2^-15 of each term's u, and the sums' binary32 errors."""
    rng = np.random.default_rng([rows, inner, rank])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, rank, 5)
    w.zero_()
    got = f64(Adapters(a, b, scales).project(x, w, ints(index)))
    X, A, B, S = map(f64, (x, a, b, scales))
    for r, i in enumerate(index):
        if i < 0:
            assert not got[r].any()
            continue
        u = S[i] * (A[i] @ X[r])
        want = B[i] @ u
        u_err = 2.0 ** -15 * np.abs(u) + S[i] * 2 * E * (inner + 16) * (np.abs(A[i]) @ np.abs(X[r]))
        tol = np.abs(B[i]) @ u_err + 2 * E * (rank + 16) * (np.abs(B[i]) @ np.abs(u))
        assert np.all(np.abs(got[r] - want) <= tol * (1 + U) + U * np.abs(want) + 2.0 ** -126)


@pytest.mark.parametrize("rows,inner,outer", PATHS)
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_an_infinity_in_an_adapter(rows, inner, outer, rank):
    """It reaches its own output of its member's rows, with the sign of what it is multiplied by:
    a number that bf16 holds (integers here) or not."""
    rng = np.random.default_rng([rows, inner, rank, 73])
    x, w, a, b, scales, index = make(rng, rows, inner, outer, rank, 3)
    x, a = (torch.from_numpy(rng.integers(-3, 4, tuple(t.shape)).astype(np.float32)).cuda().bfloat16() for t in (x, a))
    scales[0], scales[1], scales[2] = 1.0, 0.3, -2.0
    index[0] = 1
    adapters = Adapters(a, b, scales)
    want = adapters.project(x, w, ints(index))
    b[1, outer // 2, rank - 3] = float("inf")
    got = adapters.project(x, w, ints(index))
    mine = torch.from_numpy(index == 1).cuda()
    u = x.double() @ a[1, rank - 3].double() * 0.3
    hit = got[mine, outer // 2].double()
    assert torch.equal(hit[u[mine] != 0], u[mine][u[mine] != 0].sign() * float("inf"))
    assert torch.isnan(hit[u[mine] == 0]).all()            # (0 times infinity)
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[mine, outer // 2] = False
    assert torch.equal(got[keep], want[keep])
