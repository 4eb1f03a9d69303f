"""The gradients of distillation over long lists keep the bits of G that its rounding to 16 takes, for every row and query: in sums that cancel it would be all that is left."""
import math

import pytest
import torch

import head_reference as R
from test_gpu_row_distillation import backward, definition
from test_gpu_row_logprobs import inputs, unit

pytestmark = pytest.mark.gpu
LIVE = 6       # coordinates that are not zero


def sums_that_cancel(nq, n, d, dtype, seed):
    """Few rows with any probability, all with a coordinate of one (so that dq's is the sum of G over the rows: nothing), and queries in threes that are alike but
    for their weights, which add up to nothing (so that drows are nothing).  The teachers name one row of those that count."""
    g = torch.Generator().manual_seed(seed)
    t = R.DTYPES[dtype]
    rows, q = torch.zeros(n, d), torch.zeros(nq, d)
    rows[:, 0] = 1.0
    rows[:, 1] = -64.0                                    # the others: a score of -320 below
    live = torch.randperm(n, generator=g)[:8]
    rows[live, 1:LIVE] = torch.randint(-8, 9, (8, LIVE - 1), generator=g) / 8.0
    rows[live, 1] = 0.0
    of = torch.randint(-8, 9, (nq, LIVE - 2), generator=g) / 16.0
    q[:, 0], q[:, 1], q[:, 2:LIVE] = 1.0, 1.0, of
    threes = torch.randperm(nq // 3, generator=g)[:4] * 3
    weight = torch.zeros(nq)
    for i in threes.tolist():
        q[i + 1], q[i + 2] = q[i], q[i]
        weight[i:i + 3] = torch.tensor([0.3, 0.45, -0.75])
    ids = live[:1].expand(nq).clone()[:, None]
    return q.to(t), rows.to(t), ids, torch.full((nq, 1), -0.25), weight, live


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(30, 1500, 100), (300, 1500, 16), (300, 3000, 128), (30, 1500, 200), (300, 1500, 136), (700, 9000, 264), (1200, 20_000, 136)])
def test_sums_that_cancel(nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    scale = 5.0
    for bias in (False, True):
        q, rows, ids, given, g, live = sums_that_cancel(nq, n, d, dtype, nq + d)
        b = None
        if bias:
            b = torch.zeros(n)
            gen = torch.Generator().manual_seed(n)
            b[torch.randperm(n, generator=gen)[:n // 5]] = -math.inf
            b[live] = torch.randint(-4, 5, (8,), generator=gen) / 8.0
        z = R.scores(q, rows, scale, b)
        lse, logp, _, t, B = definition(z, ids, given)
        lse32 = lse.float()
        got = backward(ann, q, rows, b, ids, given, scale, lse32, logp.float(), g)
        A = (g.double() * t.sum(1))[:, None] * (z - lse32.double()[:, None]).exp()
        B = g.double()[:, None] * B
        # An element: its score's sum of LIVE products and its difference from lse (fp32: the parts' smaller products as well), a few roundings; two parts of G in 16
        # bits: half a step of half a step.  Sums: the terms that are not nothing, twice, and their parts; the others add nothing at all.
        half = R.half_step(R.DTYPES[dtype])
        most = z[:, live].abs().max() + lse.abs().max()
        err = (6 * LIVE + 16) * 2 * R.U32 * (1 + most) + (half * half if dtype != "f32" else 2.0 ** -23)
        x, qq = rows.double(), q.double()
        if b is not None:
            x = torch.where((b == -math.inf)[:, None], 0.0, x)
        counts = {"dq": 8, "drows": 12}
        for f, want, sizes, rest in (("dq", (A + B) @ x, (A.abs() + B.abs()) @ x.abs(), A.abs() @ x.abs()), ("drows", (A + B).T @ qq, (A.abs() + B.abs()).T @ qq.abs(), A.abs().T @ qq.abs())):
            products = 6 if dtype == "f32" else 2
            off = err * rest + (2 * R.U32 * (products * counts[f] + 64) + 4 * R.U32) * sizes
            # (1e-40: exp(-320), of the rows that do not count, is nothing in fp32)
            tol = half * scale * want.abs() + (1 + half) * scale * off + R.smallest_step(R.DTYPES[dtype]) + 1e-40
            assert ((got[f].double() - scale * want).abs() <= tol).all(), f
        # what the sums are: nothing beside their terms
        assert (((A + B) @ x)[:, 0].abs() <= 1e-6).all() and ((A + B).T @ qq)[live].abs().max() <= 1e-6


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, scale, k", [(400, 4000, 128, 20.0, 5), (400, 4000, 128, 20.0, 10), (200, 4000, 64, 50.0, 5), (400, 4000, 136, 20.0, 5), (200, 6000, 200, 50.0, 10)])
def test_rows_in_clusters_beside_a_teacher_who_names_few(nq, n, d, scale, k, dtype):
    """The gradients' errors are those of rounding them: within a tenth, all in all and of the worst query or row that counts (sums in fp32 take another 1e-5 or so of the terms)."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(d + k)
    t = R.DTYPES[dtype]
    centres = torch.randn(n // 20, d, generator=gen)
    rows = unit(centres[torch.arange(n) % len(centres)] + 0.3 * torch.randn(n, d, generator=gen))
    q = unit(rows[torch.randint(n, (nq,), generator=gen)] + 0.4 / math.sqrt(d) * torch.randn(nq, d, generator=gen))
    teacher = unit(q + 0.1 / math.sqrt(d) * torch.randn(nq, d, generator=gen))
    q, rows = q.to(t), rows.to(t)
    z = R.scores(teacher, rows, scale, None)
    val, ids = z.topk(k, 1)
    given = (val - torch.logsumexp(z, 1, keepdim=True)).float()
    z = R.scores(q, rows, scale, None)
    lse, logp, _, w, B = definition(z, ids, given)
    g = 0.5 + torch.rand(nq, generator=gen)
    got = backward(ann, q, rows, None, ids, given, scale, lse.float(), logp.float(), g)
    A = (g.double() * w.sum(1))[:, None] * (z - lse.float().double()[:, None]).exp()
    G = A + g.double()[:, None] * B
    # what a score in fp32, and lse, may be off moves an element of A by as much of itself (50 <q, x> of 200 columns: 264 * 2^-23 * 50)
    moved = (R.score_error(q, rows, scale, None) + 2 * R.U32 * (1 + lse.abs()))[:, None] * A
    sides = (("dq", G @ rows.double(), moved @ rows.double().norm(dim=1)), ("drows", G.T @ q.double(), moved.T @ q.double().norm(dim=1)))
    for f, want, slack in sides:
        want, slack = scale * want, scale * slack
        off, rounding = (got[f].double() - want).norm(dim=1), (want.to(t).double() - want).norm(dim=1)
        assert off.norm() <= 1.1 * rounding.norm(), f
        counts = want.norm(dim=1) > 0.1 * want.norm(dim=1).max()
        # a line's own rounding is at most half a step of each element
        assert (off <= 1.1 * R.half_step(t) * want.norm(dim=1) + slack)[counts].all(), f
