"""Distillation over lists that are too long for the kernels of short ones, at sizes that a definition in 64 bits reaches quickly: the path is asserted."""
import math

import pytest
import torch

import head_reference as R
from test_gpu_row_distillation import PAD, backward, check_backward, check_forward, definition, forward, teacher_lists
from test_gpu_row_logprobs import inputs, types

pytestmark = pytest.mark.gpu


def assert_long(ann, nq, n, d, t, k):
    """Short lists keep 8 bytes to a score and nothing else."""
    assert ann.ann_row_distillation_workspace(nq, n, d, types(ann)[t], k) != 8 * nq * n
    assert ann.ann_row_distillation_backward_workspace(nq, n, d, types(ann)[t], k) != 8 * nq * n


SHAPES = [(1, 1100, 1, 1), (3, 1025, 7, 64), (5, 1100, 100, 10), (40, 1500, 300, 20), (128, 1152, 128, 5), (130, 1257, 96, 20), (200, 1300, 200, 8), (257, 1300, 200, 8),
          (300, 1029, 520, 33), (9, 1700, 1500, 7)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHAPES)
def test_forward_and_backward(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    assert_long(ann, nq, n, d, R.DTYPES[dtype], k)
    gen = torch.Generator().manual_seed(nq + n)
    for bias, pad, scale in (("none", 0, 10.0), ("plain", 8, 5.0), ("holes", 1, -3.0)):
        q, rows, b, _ = inputs(nq, n, d, dtype, n + d, bias)
        ids, given = teacher_lists(q, rows, b, scale, k, d)
        check_forward(ann, q, rows, b, ids, given, scale, pad)
        check_backward(ann, q, rows, b, ids, given, scale, 0.5 + torch.rand(nq, generator=gen), pad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", [(40, 1500, 300, 16), (200, 1300, 200, 8), (280, 1200, 136, 32), (60, 1400, 96, 5)])
def test_a_student_that_has_learnt(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    assert_long(ann, nq, n, d, R.DTYPES[dtype], k)
    q, rows, _, _ = inputs(nq, n, d, dtype, 3)
    ids, given = teacher_lists(q, rows, None, 20.0, k, d, near=0.0)
    check_forward(ann, q, rows, None, ids, given, 20.0)
    check_backward(ann, q, rows, None, ids, given, 20.0, torch.full((nq,), 1.0 / nq))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, d", [(40, 100), (40, 200), (300, 136)])
def test_given_rows_that_are_left_out(nq, d, dtype):
    import paper_2503_17911_amd as ann
    n, k = 1500, 6
    assert_long(ann, nq, n, d, R.DTYPES[dtype], k)
    q, rows, b, _ = inputs(nq, n, d, dtype, 5, "holes")
    ids, given = teacher_lists(q, rows, b, 20.0, k, 1)
    out = torch.nonzero(b == -math.inf)[:, 0]
    ids[10, 2], given[10, 2] = out[0], -1.0          # counts: the loss is infinite, the others' gradient has its weight
    ids[11, 2], given[11, 2] = out[1], -math.inf     # does not count
    spoilt = rows.clone()
    spoilt[out] = float("nan")
    got = check_forward(ann, q, spoilt, b, ids, given, 20.0)
    assert got["loss"][10] == math.inf and got["loss"][11] < math.inf
    assert got["logprobs"][10, 2] == got["logprobs"][11, 2] == -math.inf
    g = torch.ones(nq)
    back = check_backward(ann, q, rows, b, ids, given, 20.0, g)
    again = backward(ann, q, spoilt, b, ids, given, 20.0, *(v.float() for v in definition(R.scores(q, rows, 20.0, b), ids, given)[:2]), g)
    for f in back:
        assert torch.equal(back[f], again[f]), f
    assert (back["drows"][out] == 0).all() and (back["drow_bias"][out] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [600, 1600])
def test_masks_of_the_lowest_value_are_ordinary_biases(n, dtype):
    """Rows with the lowest finite bias have no probability but can be given: their log probability is finite (or -infinity where fp32 has no number), the loss with it."""
    import paper_2503_17911_amd as ann
    nq, d, k = 30, 64, 4
    q, rows, _, _ = inputs(nq, n, d, dtype, 5)
    for lowest in (torch.finfo(torch.float32).min, -1e4):
        b = torch.zeros(n)
        b[::3] = lowest
        ids, given = teacher_lists(q, rows, b, 8.0, k, 1)
        ids[4:20, 1], given[4:20, 1] = 3 * torch.arange(16), -2.0
        got = check_forward(ann, q, rows, b, ids, given, 8.0)
        assert (got["logprobs"][4:20, 1] < -9e3).all() and (got["loss"][4:20] > 1e3).all()
        check_backward(ann, q, rows, b, ids, given, 8.0, torch.ones(nq))


@pytest.mark.parametrize("dtype, nq, d", [("bf16", 40, 100), ("bf16", 40, 200), ("f16", 40, 200), ("f16", 300, 136), ("f16", 70, 64), ("f32", 40, 70)])
def test_parts_and_nothing(dtype, nq, d):
    import paper_2503_17911_amd as ann
    n = 1500
    assert_long(ann, nq, n, d, R.DTYPES[dtype], 7)
    q, rows, b, _ = inputs(nq, n, d, dtype, 5, "holes")
    ids, given = teacher_lists(q, rows, b, 20.0, 7, 1)
    lse, logp = (v.float() for v in definition(R.scores(q, rows, 20.0, b), ids, given)[:2])
    g = torch.randn(nq, generator=torch.Generator().manual_seed(3))
    full = check_backward(ann, q, rows, b, ids, given, 20.0, g)
    for f in full:
        only = backward(ann, q, rows, b, ids, given, 20.0, lse, logp, g, dq=f == "dq", drows=f == "drows", dbias=f == "drow_bias")
        assert list(only) == [f] and torch.equal(only[f], full[f])
    # all rows left out; nothing given
    out = torch.full((n,), -math.inf)
    got = forward(ann, q, rows, out, ids, given, 20.0)
    counts = ((ids >= 0) & (ids < n) & (given > -math.inf)).any(1)
    assert (got["lse"] == -math.inf).all() and (got["loss"][counts] == math.inf).all() and (got["loss"][~counts] == 0).all()
    for v in backward(ann, q, rows, out, ids, given, 20.0, got["lse"], got["logprobs"], g).values():
        assert (v == 0).all()
    none = torch.full_like(ids, PAD)
    got = forward(ann, q, rows, b, none, given, 20.0)
    assert (got["loss"] == 0).all() and (got["logprobs"] == 0).all()
    for v in backward(ann, q, rows, b, none, given, 20.0, lse, logp, g).values():
        assert (v == 0).all()


def test_gradient_against_differences():
    import paper_2503_17911_amd as ann
    assert_long(ann, 20, 1400, 48, torch.float32, 8)
    q, rows, b, _ = inputs(20, 1400, 48, "f32", 3, "plain")
    ids, given = teacher_lists(q, rows, b, 6.0, 8, 2)
    gen = torch.Generator().manual_seed(1)
    g = torch.randn(20, generator=gen)
    f = forward(ann, q, rows, b, ids, given, 6.0)
    got = backward(ann, q, rows, b, ids, given, 6.0, f["lse"], f["logprobs"], g)

    def loss(q, rows, b):
        return float((g.double() * definition(R.scores(q, rows, 6.0, b), ids, given)[2]).sum())

    q, rows, b = q.double(), rows.double(), b.double()
    step = 1e-5
    for _ in range(4):
        e = [torch.randn(v.shape, generator=gen, dtype=R.F64) for v in (q, rows, b)]
        slope = (loss(*(v + step * w for v, w in zip((q, rows, b), e))) - loss(*(v - step * w for v, w in zip((q, rows, b), e)))) / (2 * step)
        terms = [got[f].double() * w for f, w in zip(("dq", "drows", "drow_bias"), e)]
        # (a score errs by some 2^-17 at most here, its exponential by as much relative to itself)
        assert abs(sum(float(v.sum()) for v in terms) - slope) <= 2.0 ** -15 * sum(float(v.abs().sum()) for v in terms) + 1e-4
