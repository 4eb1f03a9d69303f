"""Distillation over rows' scores and its gradients against their definitions in 64 bits."""
import math

import pytest
import torch

import head_reference as R
from test_gpu_row_logprobs import inputs, strided, stream, types, unit

pytestmark = pytest.mark.gpu
PAD = -1


def teacher_lists(q, rows, b, scale, k, seed, near=0.3):
    """A teacher's lists: its k likeliest rows and their log probabilities; some that end early, one without an entry, rows that are given twice,
    ids that are no row's, entries without weight."""
    g = torch.Generator().manual_seed(seed)
    nq, d = q.shape
    n = rows.shape[0]
    z = R.scores(unit(q.double() + near / math.sqrt(d) * torch.randn(nq, d, generator=g, dtype=R.F64)), rows, scale, b)
    val, ids = z.topk(min(k, n), 1)
    val = val - torch.logsumexp(z, 1, keepdim=True)
    if k > n:
        val, ids = torch.cat([val, val[:, :1].expand(-1, k - n)], 1), torch.cat([ids, ids[:, :1].expand(-1, k - n)], 1)
    ids = torch.where(val == -math.inf, torch.full_like(ids, PAD), ids)
    given = val.float()
    if nq > 3:
        ids[1], given[1] = PAD, -math.inf
        ids[2, -1] = n + 5
        given[3, 0] = -math.inf
        if k > 1:
            ids[3, 1], given[3, 1] = ids[0, 0], -0.7
            ids[0, -1] = ids[0, 0]
    return ids, given


def definition(z, ids, given):
    """lse, the entries' log probabilities, the loss, the entries' weights and G's second part (all for g = 1)."""
    nq, n = z.shape
    lse = torch.logsumexp(z, 1) if n else torch.full((nq,), -math.inf, dtype=R.F64)
    there = (ids >= 0) & (ids < n)
    picked = z.gather(1, ids.clamp(0, n - 1)) if n else torch.zeros(ids.shape, dtype=R.F64)
    logp = torch.where(there, torch.where(picked == -math.inf, picked, picked - lse[:, None]), 0.0)
    t = torch.where(there, given.double().exp(), 0.0)
    loss = torch.where(t > 0, t * (given.double() - logp), 0.0).sum(1)
    B = torch.zeros(nq, max(n, 1), dtype=R.F64).scatter_add_(1, ids.clamp(0, max(n - 1, 0)), -t)[:, :n]
    return lse, logp, loss, t, torch.where(z == -math.inf, 0.0, B)


def on_gpu(ids):
    return ids.to(torch.int32).cuda()


def call(ann, q, rows, b, ids, given, scale, pad=0):
    (nq, d), n, k, t = q.shape, rows.shape[0], ids.shape[1], types(ann)[q.dtype]
    qd, xd = strided(q, pad), strided(rows, pad)
    return dict(q=qd, nq=nq, q_stride=qd.stride(0), rows=xd, n=n, row_stride=xd.stride(0), d=d, type=t, scale=scale, row_bias=None if b is None else b.cuda(), k=k,
                given_ids=on_gpu(ids), given_logprobs=given.cuda(), stream=stream())


def dirty(need):
    return torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read before it is written)


def forward(ann, q, rows, b, ids, given, scale, pad=0):
    (nq, d), n, k = q.shape, rows.shape[0], ids.shape[1]
    need = ann.ann_row_distillation_workspace(nq, n, d, types(ann)[q.dtype], k)
    out = dict(loss=torch.full((nq,), 7.0, device="cuda"), lse=torch.full((nq,), 7.0, device="cuda"), logprobs=torch.full((nq, k), 7.0, device="cuda"))
    ws = dirty(need)
    ann.ann_row_distillation(**call(ann, q, rows, b, ids, given, scale, pad), workspace=ws, workspace_bytes=need, **out)
    torch.cuda.synchronize()
    return {f: v.cpu() for f, v in out.items()}


def backward(ann, q, rows, b, ids, given, scale, lse, logprobs, g, pad=0, dq=True, drows=True, dbias=True):
    (nq, d), n, k = q.shape, rows.shape[0], ids.shape[1]
    need = ann.ann_row_distillation_backward_workspace(nq, n, d, types(ann)[q.dtype], k)
    out = dict(dq=strided(torch.full_like(q, 7.0), pad, 3.0) if dq else None, drows=strided(torch.full_like(rows, 7.0), pad, 3.0) if drows else None,
               drow_bias=torch.full((n,), 7.0, device="cuda") if dbias else None)
    ws = dirty(need)
    ann.ann_row_distillation_backward(**call(ann, q, rows, b, ids, given, scale, pad), lse=lse.cuda(), logprobs=logprobs.cuda(), g_loss=g.cuda(), dq_stride=d + pad,
                                      drows_stride=d + pad, workspace=ws, workspace_bytes=need, **out)
    torch.cuda.synchronize()
    return {f: v.cpu() for f, v in out.items() if v is not None}


def check_forward(ann, q, rows, b, ids, given, scale, pad=0):
    z = R.scores(q, rows, scale, b)
    lse, logp, loss, t, _ = definition(z, ids, given)
    got = forward(ann, q, rows, b, ids, given, scale, pad)
    off = R.score_error(q, rows, scale, b) + R.sum_error(z.shape[1])
    none = lse == -math.inf
    assert (got["lse"][none] == -math.inf).all()
    assert ((got["lse"].double() - lse).abs()[~none] <= (off + 2 * R.U32 * lse.abs())[~none]).all()
    # a given row's score: its sum is fp64; what lse is off moves it
    tol = (off + 2 * R.U32 * lse.abs())[:, None] + 2 * R.U32 * logp.abs()
    out = logp == -math.inf
    assert torch.equal(got["logprobs"] == -math.inf, out)
    assert ((got["logprobs"].double() - logp).abs()[~out] <= tol[~out]).all()
    infinite = loss == math.inf
    assert torch.equal(got["loss"] == math.inf, infinite)
    assert ((got["loss"].double() - loss).abs() <= torch.where(t > 0, t * tol, 0.0).sum(1) + 2 * R.U32 * loss.abs())[~infinite].all()
    return got


def check_backward(ann, q, rows, b, ids, given, scale, g, pad=0):
    z = R.scores(q, rows, scale, b)
    nq, n = z.shape
    lse, logp, _, t, B = definition(z, ids, given)
    lse, logp = lse.float(), logp.float()
    got = backward(ann, q, rows, b, ids, given, scale, lse, logp, g, pad)
    p = torch.where(z == -math.inf, 0.0, (z - torch.where(lse == -math.inf, 0.0, lse)[:, None].double()).exp())
    W = torch.where(lse == -math.inf, 0.0, g.double() * t.sum(1))
    A, B = W[:, None] * p, torch.where((lse == -math.inf)[:, None], 0.0, g.double()[:, None] * B)
    dtype, half = q.dtype, R.half_step(q.dtype)
    # an element of the first part: the score's error through p, the log probability's rounding (which the remainder is formed by), a few roundings
    err = (R.score_error(q, rows, scale, b) + 12 * R.U32 * (1 + torch.where(lse == -math.inf, 0.0, lse).abs()))[:, None] + 8 * R.U32 + R.U32 * z.sub(
        lse[:, None].double()).abs().nan_to_num(0.0, 0.0, 0.0)
    size = A.abs() * (err + 8 * R.U32) + 4 * R.U32 * B.abs()
    given_there = B != 0
    if dtype == torch.float32:
        kept = 2.0 ** -23 * A.abs()
    else:
        by = 2.0 ** (14 - max(-100, math.frexp(W.abs().max().float().item())[1])) if dtype == torch.float16 and W.abs().max() > 0 else 1.0
        kept = half * A.abs() + (2.0 ** -25 / by if dtype == torch.float16 else 0.0)
        # what the rounding left is added at given rows; where the element may round either way, a whole step of it
        low, high = (A * by * (1 - err)).to(dtype), (A * by * (1 + err)).to(dtype)
        kept = torch.where(given_there, torch.where(low == high, 0.0, 2 * kept), kept)
    x, qq = rows.double(), q.double()
    if b is not None:
        x = torch.where((b == -math.inf)[:, None], torch.zeros_like(x), x)
    products = (6 if dtype == torch.float32 else 1) * 2 * R.U32
    G, terms = A + B, A.abs() + B.abs()
    for f, want, sizes, off in (("dq", G @ x, terms @ x.abs(), (size + kept) @ x.abs()), ("drows", G.T @ qq, terms.T @ qq.abs(), (size + kept).T @ qq.abs())):
        want, sizes, off = scale * want, abs(scale) * sizes, abs(scale) * off
        length = n if f == "dq" else nq
        tol = (half * want.abs() + R.smallest_step(dtype) + off + (products * length + 64 * R.U32) * sizes) * (1 + half)
        assert ((got[f].double() - want).abs() <= tol).all(), f
    assert ((got["drow_bias"].double() - G.sum(0)).abs() <= size.sum(0) + (nq + 64) * R.U32 * terms.sum(0) + 1e-40).all()
    return got


SHAPES = [(1, 1, 1, 1), (1, 300, 16, 3), (3, 64, 7, 64), (5, 65, 100, 10), (128, 128, 128, 5), (130, 257, 96, 20), (70, 1000, 200, 32), (33, 5000, 64, 64), (300, 4100, 768, 10),
          (9, 700, 1500, 7), (1, 20000, 128, 5), (600, 130, 130, 33), (500, 3000, 128, 40), (2000, 40, 30, 50)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHAPES)
def test_forward_and_backward(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + n)
    for bias, pad, scale in (("none", 0, 10.0), ("plain", 8, 5.0), ("holes", 1, -3.0)):
        q, rows, b, _ = inputs(nq, n, d, dtype, n + d, bias)
        ids, given = teacher_lists(q, rows, b, scale, k, d)
        check_forward(ann, q, rows, b, ids, given, scale, pad)
        check_backward(ann, q, rows, b, ids, given, scale, 0.5 + torch.rand(nq, generator=gen), pad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_student_that_has_learnt(dtype):
    """The teacher's lists are the student's own: the two parts of G cancel at the rows that count most."""
    import paper_2503_17911_amd as ann
    for nq, n, d, k in ((300, 2000, 128, 32), (40, 500, 300, 16), (280, 700, 200, 8)):
        q, rows, _, _ = inputs(nq, n, d, dtype, 3)
        ids, given = teacher_lists(q, rows, None, 20.0, k, d, near=0.0)
        check_forward(ann, q, rows, None, ids, given, 20.0)
        check_backward(ann, q, rows, None, ids, given, 20.0, torch.full((nq,), 1.0 / nq))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_every_teacher_names(dtype):
    import paper_2503_17911_amd as ann
    nq, n, d, k = 700, 2500, 96, 30
    q, rows, b, _ = inputs(nq, n, d, dtype, 3, "plain")
    ids, given = teacher_lists(q, rows, b, 5.0, k, d)
    ids[:, :20] = torch.arange(20) * 100
    check_forward(ann, q, rows, b, ids, given, 5.0)
    check_backward(ann, q, rows, b, ids, given, 5.0, torch.rand(nq, generator=torch.Generator().manual_seed(1)))


def test_losses_of_any_size_and_sign():
    """Half precision has to carry gradients of a mean over many, of a scaled loss, and of one that is taken off."""
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(50, 3000, 64, "f16", 5)
    ids, given = teacher_lists(q, rows, b, 0.05, 9, 2)
    for size in (1e-6, 1.0, -1.0, 2.0 ** 14):
        check_backward(ann, q, rows, b, ids, given, 0.05, size * (0.5 + torch.rand(50, generator=torch.Generator().manual_seed(2))))
    check_backward(ann, q, rows, b, ids, given, 0.05, torch.zeros(50))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_given_rows_that_are_left_out(dtype):
    import paper_2503_17911_amd as ann
    nq, n, d, k = 40, 900, 100, 6
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
        assert torch.equal(back[f], again[f])
    assert (back["drows"][out] == 0).all() and (back["drow_bias"][out] == 0).all()


def test_masks_of_the_lowest_value_are_ordinary_biases():
    """Rows with the lowest finite bias have no probability but can be given: their log probability is finite or -infinity, the others' gradients are as ever."""
    import paper_2503_17911_amd as ann
    nq, n, d, k = 30, 600, 64, 4
    q, rows, _, _ = inputs(nq, n, d, "bf16", 5)
    b = torch.zeros(n)
    b[::3] = torch.finfo(torch.float32).min
    ids, given = teacher_lists(q, rows, b, 8.0, k, 1)
    check_forward(ann, q, rows, b, ids, given, 8.0)
    check_backward(ann, q, rows, b, ids, given, 8.0, torch.ones(nq))


def test_parts_and_nothing():
    import paper_2503_17911_amd as ann
    for dtype, d in (("bf16", 100), ("f16", 200), ("f32", 70)):
        q, rows, b, _ = inputs(40, 900, d, dtype, 5, "holes")
        ids, given = teacher_lists(q, rows, b, 20.0, 7, 1)
        lse, logp = (v.float() for v in definition(R.scores(q, rows, 20.0, b), ids, given)[:2])
        g = torch.randn(40, generator=torch.Generator().manual_seed(3))
        full = backward(ann, q, rows, b, ids, given, 20.0, lse, logp, g)
        for f in full:
            only = backward(ann, q, rows, b, ids, given, 20.0, lse, logp, g, dq=f == "dq", drows=f == "drows", dbias=f == "drow_bias")
            assert list(only) == [f] and torch.equal(only[f], full[f])
        # all rows left out; nothing given; no queries; no rows
        out = torch.full((900,), -math.inf)
        got = forward(ann, q, rows, out, ids, given, 20.0)
        counts = ((ids >= 0) & (ids < 900) & (given > -math.inf)).any(1)
        assert (got["lse"] == -math.inf).all() and (got["loss"][counts] == math.inf).all() and (got["loss"][~counts] == 0).all()
        for v in backward(ann, q, rows, out, ids, given, 20.0, got["lse"], got["logprobs"], g).values():
            assert (v == 0).all()
        none = torch.full_like(ids, PAD)
        got = forward(ann, q, rows, b, none, given, 20.0)
        assert (got["loss"] == 0).all() and (got["logprobs"] == 0).all()
        for v in backward(ann, q, rows, b, none, given, 20.0, lse, logp, g).values():
            assert (v == 0).all()
        for v in backward(ann, q[:0], rows, b, ids[:0], given[:0], 20.0, lse[:0], logp[:0], g[:0], dq=False).values():
            assert (v == 0).all()
        got = forward(ann, q, rows[:0], None, ids, given, 20.0)
        assert (got["lse"] == -math.inf).all() and (got["loss"] == 0).all()
        assert (backward(ann, q, rows[:0], None, ids, given, 20.0, got["lse"], got["logprobs"], g, drows=False, dbias=False)["dq"] == 0).all()


def test_teachers_lists_as_the_alternatives_come():
    """ann_row_logprobs' alternatives of the teacher's queries go in as they are."""
    import paper_2503_17911_amd as ann
    nq, n, d, k = 64, 5000, 128, 16
    q, rows, _, _ = inputs(nq, n, d, "bf16", 5)
    tq = unit(q.float() + 0.05 * torch.randn(nq, d, generator=torch.Generator().manual_seed(1)))
    lp, lse, ids, val = torch.empty(nq, device="cuda"), torch.empty(nq, device="cuda"), torch.empty(nq, k, dtype=torch.int32, device="cuda"), torch.empty(nq, k, device="cuda")
    need = ann.ann_row_logprobs_workspace(nq, n, d, ann.BF16, k)
    tqd, xd = tq.bfloat16().cuda(), rows.cuda()
    ann.ann_row_logprobs(tqd, nq, d, xd, n, d, d, ann.BF16, scale=20.0, k=k, logprob=lp, lse=lse, alt_ids=ids, alt_logprobs=val, workspace=dirty(need),
                         workspace_bytes=need, stream=stream())
    got = check_forward(ann, q, rows, None, ids.cpu().long(), val.cpu(), 20.0)
    assert (got["loss"] > 0).all()
    # the teacher's own queries: no divergence but what lies behind its list and the roundings
    same = check_forward(ann, tq.bfloat16(), rows, None, ids.cpu().long(), val.cpu(), 20.0)
    assert (same["loss"].abs() <= 1e-5).all()


def test_gradient_against_differences():
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(20, 400, 48, "f32", 3, "plain")
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


def test_same_bits_again_on_other_streams_and_in_graphs():
    import paper_2503_17911_amd as ann
    for dtype, bias, nq, n, d, k in (("bf16", "none", 600, 3000, 128, 32), ("f16", "holes", 20, 3000, 200, 5), ("f32", "plain", 30, 1500, 72, 64)):
        q, rows, b, _ = inputs(nq, n, d, dtype, 5, bias)
        ids, given = teacher_lists(q, rows, b, 15.0, k, 3)
        table = call(ann, q, rows, b, ids, given, 15.0)
        t, g = types(ann)[q.dtype], torch.rand(nq, device="cuda")
        need, needb = ann.ann_row_distillation_workspace(nq, n, d, t, k), ann.ann_row_distillation_backward_workspace(nq, n, d, t, k)

        def outputs():
            return [torch.zeros(nq, device="cuda"), torch.zeros(nq, device="cuda"), torch.zeros(nq, k, device="cuda"), torch.zeros_like(table["q"]),
                    torch.zeros_like(table["rows"]), torch.zeros(n, device="cuda"), dirty(need), dirty(needb)]

        def both(o):
            a = dict(table, stream=stream(), lse=o[1], logprobs=o[2])
            ann.ann_row_distillation(**a, loss=o[0], workspace=o[6], workspace_bytes=need)
            ann.ann_row_distillation_backward(**a, g_loss=g, dq=o[3], dq_stride=o[3].stride(0), drows=o[4], drows_stride=o[4].stride(0), drow_bias=o[5],
                                              workspace=o[7], workspace_bytes=needb)

        want, other, graphed = outputs(), outputs(), outputs()
        both(want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            both(other)
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want[:6], other[:6]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(graphed)
        for replay in range(3):
            table["q"].copy_(unit(torch.randn(nq, d, device="cuda")))
            table["given_ids"].copy_(torch.randint(n, (nq, k), device="cuda") if replay else torch.full((nq, k), 3, device="cuda"))
            both(want)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(want[:6], graphed[:6])), replay


@pytest.mark.parametrize("dtype, nq, n, d", [("f32", 3000, 50_000, 136), ("f16", 5000, 60_000, 144), ("bf16", 300, 20_000, 1000)])
def test_several_chunks_of_rows(dtype, nq, n, d):
    """More scores than are kept at a time: against 64 bits on the GPU, by the sums' sizes."""
    import paper_2503_17911_amd as ann
    g = torch.Generator(device="cuda").manual_seed(1)
    k, scale, t = 12, 8.0, R.DTYPES[dtype]
    q, rows = (unit(torch.randn(m, d, generator=g, device="cuda")).to(t) for m in (nq, n))
    b = torch.randn(n, generator=g, device="cuda")
    ids, given = torch.randint(n, (nq, k), generator=g, device="cuda").int(), -2.0 - torch.rand(nq, k, generator=g, device="cuda")
    ids[:, 0] = 7
    loss, lse, logprobs = torch.empty(nq, device="cuda"), torch.empty(nq, device="cuda"), torch.empty(nq, k, device="cuda")
    T = types(ann)[t]
    table = dict(q=q, nq=nq, q_stride=d, rows=rows, n=n, row_stride=d, d=d, type=T, scale=scale, row_bias=b, k=k, given_ids=ids, given_logprobs=given, lse=lse,
                 logprobs=logprobs, stream=stream())
    need, needb = ann.ann_row_distillation_workspace(nq, n, d, T, k), ann.ann_row_distillation_backward_workspace(nq, n, d, T, k)
    ann.ann_row_distillation(**table, loss=loss, workspace=dirty(need), workspace_bytes=need)
    gl = torch.rand(nq, generator=g, device="cuda") + 0.5
    dq, drows, db = torch.empty_like(q), torch.empty_like(rows), torch.empty(n, device="cuda")
    ann.ann_row_distillation_backward(**table, g_loss=gl, dq=dq, dq_stride=d, drows=drows, drows_stride=d, drow_bias=db, workspace=dirty(needb), workspace_bytes=needb)
    q64, x64 = q.double(), rows.double()
    z = torch.mm(q64, x64.t().contiguous()) * scale + b.double()
    lse64 = torch.logsumexp(z, 1)
    assert ((lse.double() - lse64).abs() <= 1e-5).all()
    logp = (z - lse64[:, None]).gather(1, ids.long())
    w = given.double().exp()
    want = (w * (given.double() - logp)).sum(1)
    assert ((loss.double() - want).abs() <= 1e-5 * w.sum(1) + 2 * R.U32 * want.abs()).all()
    A = (z - lse.double()[:, None]).exp_() * (gl.double() * w.sum(1))[:, None]
    del z
    B = torch.zeros_like(A).scatter_add_(1, ids.long(), -gl.double()[:, None] * w)
    # a score errs by some 1e-5, sums of up to 60,000 terms by their own; 16 bits round every element of the first part and the result
    half = R.half_step(t)
    kept = half if dtype != "f32" else 2.0 ** -23
    G, size = A + B, A.abs() * (kept + 2e-5) + B.abs() * 2e-5
    for got, exact, off in ((dq, torch.mm(G, x64), torch.mm(size, x64.abs())), (drows, torch.mm(G.t().contiguous(), q64), torch.mm(size.t().contiguous(), q64.abs()))):
        assert ((got.double() - scale * exact).abs() <= (half * scale * exact.abs() + R.smallest_step(t) + scale * off) * (1 + half)).all()
    assert ((db.double() - G.sum(0)).abs() <= ((A.abs() + B.abs()) * 2e-5).sum(0)).all()


def test_offsets_beyond_32_bits():
    import paper_2503_17911_amd as ann
    nq, n, d, k, stride = 6, 1100, 64, 5, 1 << 22
    far = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda").view(n, stride)   # 9.2 GB
    far[:, :d] = unit(torch.randn(n, d, device="cuda")).bfloat16()
    near = far[:, :d].contiguous()
    q, ids, given = near[-nq:].clone(), torch.randint(n, (nq, k), device="cuda").int(), torch.full((nq, k), -1.8, device="cuda")
    got = []
    for rows, s, drows, ds in ((near, d, torch.empty_like(near), d), (far, stride, far[:, 128:], stride)):
        out = [torch.empty(nq, device="cuda"), torch.empty(nq, device="cuda"), torch.empty(nq, k, device="cuda"), torch.empty_like(q)]
        table = dict(q=q, nq=nq, q_stride=d, rows=rows, n=n, row_stride=s, d=d, type=ann.BF16, scale=20.0, k=k, given_ids=ids, given_logprobs=given, lse=out[1],
                     logprobs=out[2], stream=stream())
        need, needb = ann.ann_row_distillation_workspace(nq, n, d, ann.BF16, k), ann.ann_row_distillation_backward_workspace(nq, n, d, ann.BF16, k)
        ann.ann_row_distillation(**table, loss=out[0], workspace=dirty(need), workspace_bytes=need)
        ann.ann_row_distillation_backward(**table, g_loss=torch.ones(nq, device="cuda"), dq=out[3], dq_stride=d, drows=drows, drows_stride=ds, workspace=dirty(needb),
                                          workspace_bytes=needb)
        got.append(out + [drows[:, :d].clone()])
    assert all(torch.equal(a, c) for a, c in zip(*got)) and (got[0][4] != 0).any()


SHORT = [(1, 1, 1, 1), (1, 16, 8, 2), (17, 15, 7, 3), (16, 17, 33, 20), (3, 64, 5, 64), (300, 256, 96, 10), (33, 255, 961, 20), (40, 257, 300, 5), (20, 1024, 100, 32), (1000, 100, 131, 40)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHORT)
def test_short_lists_are_summed_in_64_bits(nq, n, d, k, dtype):
    """Of short lists every sum is fp64: the results are off by their own rounding, a small loss too (students near their teacher)."""
    import paper_2503_17911_amd as ann
    for bias, pad, scale in (("none", 0, 10.0), ("holes", 1, 8.0), ("plain", 8, -3.0)):
        q, rows, b, _ = inputs(nq, n, d, dtype, n + d, bias)
        ids, given = teacher_lists(q, rows, b, scale, k, d, near=0.02)
        z = R.scores(q, rows, scale, b)
        lse, logp, loss, t, _ = definition(z, ids, given)
        got = forward(ann, q, rows, b, ids, given, scale, pad)
        # fp64: d + n additions and a few functions, of scores up to |scale| |q| |x| + |bias|; times what a loss sums.  2 ** -24 of a result: its rounding
        most = abs(scale) * q.double().norm(dim=1) * rows.double().norm(dim=1).max() + (0.0 if b is None else b[b > -math.inf].abs().max())
        wide = (2 * d + n + 64) * 2.0 ** -53 * (1 + most + lse.abs())
        for f, want, slack in (("lse", lse, wide), ("logprobs", logp, 2 * wide[:, None]), ("loss", loss, 2 * wide * t.sum(1) + 64 * 2.0 ** -53 * (t * (given.double() - logp).nan_to_num()).abs().sum(1))):
            there = want.abs() < math.inf
            assert torch.equal(got[f].double()[~there], want[~there]), f
            assert ((got[f].double() - want).abs() <= R.U32 * want.abs() + slack + 2.0 ** -149)[there].all(), f


def test_short_list_spoilt_in_its_left_out_rows():
    """What lies in rows left out has no part in any result; of more scores than the kernels of short lists take, the others' do the same."""
    import paper_2503_17911_amd as ann
    for nq, n in ((50, 200), (40000, 250), (1100, 1000)):
        q, rows, b, _ = inputs(nq, n, 40, "bf16", 7, "holes")
        ids, given = teacher_lists(q, rows, b, 10.0, 8, 3)
        first = check_forward(ann, q, rows, b, ids, given, 10.0)
        spoilt = rows.clone()
        spoilt[b == -math.inf] = float("nan")
        second = forward(ann, q, spoilt, b, ids, given, 10.0)
        assert all(torch.equal(first[f], second[f]) for f in first)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHORT)
def test_gradients_over_short_lists_are_summed_in_64_bits(nq, n, d, k, dtype):
    """The gradients are off by lse's rounding to fp32, which they take the probabilities from, and by their own."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq)
    for bias, pad, scale in (("none", 0, 10.0), ("holes", 1, 8.0), ("plain", 8, -3.0)):
        q, rows, b, _ = inputs(nq, n, d, dtype, n + d, bias)
        ids, given = teacher_lists(q, rows, b, scale, k, d, near=0.02)
        z = R.scores(q, rows, scale, b)
        lse, _, _, t, B = definition(z, ids, given)
        g = 0.5 + torch.rand(nq, generator=gen)
        lse32 = torch.where(torch.rand(nq, generator=gen) < 0.5, lse, lse + 0.3).float()   # (of more rows than these, as with rows on several cards)
        got = backward(ann, q, rows, b, ids, given, scale, lse32, torch.zeros(nq, k), g, pad)
        A = (g.double() * t.sum(1))[:, None] * torch.where(z == -math.inf, 0.0, (z - lse32.double()[:, None]).exp())
        G = A + g.double()[:, None] * B
        x, qq = rows.double(), q.double()
        if b is not None:
            x = torch.where((b == -math.inf)[:, None], 0.0, x)
        # fp64: a score as above, an exponential of it, k subtractions, the products' n or nq additions; 2 ** -24 and half a step: the roundings at the end
        most = abs(scale) * q.double().norm(dim=1) * rows.double().norm(dim=1).max() + (0.0 if b is None else b[b > -math.inf].abs().max())
        wide = ((2 * d + k + 64) * 2.0 ** -53 * (1 + most + lse.abs()))[:, None] * (A + g.double()[:, None] * B.abs())
        many = (n + nq + 64) * 2.0 ** -53
        terms = A + g.double()[:, None] * B.abs()
        for f, want, slack in (("dq", G @ x, wide @ x.abs() + many * (terms @ x.abs())), ("drows", G.T @ qq, wide.T @ qq.abs() + many * (terms.T @ qq.abs()))):
            tol = (abs(scale) * (want.abs() * R.U32 + slack) + R.half_step(q.dtype) * abs(scale) * want.abs()) * (1 + 2 * R.half_step(q.dtype)) + R.smallest_step(q.dtype)
            assert ((got[f].double() - scale * want).abs() <= tol).all(), f
        assert ((got["drow_bias"].double() - G.sum(0)).abs() <= R.U32 * G.sum(0).abs() + wide.sum(0) + many * terms.sum(0) + 2.0 ** -149).all()
        # each by itself, and again: the same bits
        for only in (dict(drows=False, dbias=False), dict(dq=False, dbias=False), dict(dq=False, drows=False), dict()):
            again = backward(ann, q, rows, b, ids, given, scale, lse32, torch.zeros(nq, k), g, pad, **only)
            assert all(torch.equal(again[f], got[f]) for f in again)


def test_gradients_over_short_lists_with_spoilt_rows_left_out_and_queries_without_rows():
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(50, 200, 41, "bf16", 7, "holes")
    ids, given = teacher_lists(q, rows, b, 10.0, 8, 3)
    g = torch.ones(50)
    z = R.scores(q, rows, 10.0, b)
    lse = definition(z, ids, given)[0].float()
    first = backward(ann, q, rows, b, ids, given, 10.0, lse, torch.zeros(50, 8), g)
    spoilt = rows.clone()
    spoilt[b == -math.inf] = float("nan")
    second = backward(ann, q, spoilt, b, ids, given, 10.0, lse, torch.zeros(50, 8), g)
    assert all(torch.equal(first[f], second[f]) for f in first)
    assert (first["drows"][:, :41][b == -math.inf] == 0).all() and (first["drow_bias"][b == -math.inf] == 0).all()
    out = torch.full((200,), -math.inf)
    none = backward(ann, q, rows, out, ids, given, 10.0, torch.full((50,), -math.inf), torch.full((50, 8), -math.inf), g)
    assert all((none[f][:, :41] == 0).all() for f in ("dq", "drows")) and (none["drow_bias"] == 0).all()


def test_short_lists_in_a_graph():
    """Forward and backward captured over one workspace and replayed with other contents, with eager work between: each replay gives the eager calls' bits."""
    import paper_2503_17911_amd as ann
    nq, n, d, k, t = 37, 200, 100, 8, types(ann)[torch.bfloat16]
    cases = []
    for seed in (1, 2, 3):
        q, rows, b, _ = inputs(nq, n, d, "bf16", seed, "holes")
        cases.append((q.cuda(), rows.cuda(), b.cuda(), *(x.cuda() for x in teacher_lists(q, rows, b, 10.0, k, seed))))
    held = [x.clone() if x.dtype != torch.int64 else x.to(torch.int32) for x in cases[0]]
    q, rows, b, ids, given = held
    need = max(ann.ann_row_distillation_workspace(nq, n, d, t, k), ann.ann_row_distillation_backward_workspace(nq, n, d, t, k))
    ws = dirty(need)
    loss, lse, logprobs, g = torch.empty(nq, device="cuda"), torch.empty(nq, device="cuda"), torch.empty(nq, k, device="cuda"), torch.full((nq,), 0.5, device="cuda")
    dq, drows, dbias = torch.empty_like(q), torch.empty_like(rows), torch.empty(n, device="cuda")

    def both():
        what = dict(q=q, nq=nq, q_stride=d, rows=rows, n=n, row_stride=d, d=d, type=t, scale=10.0, row_bias=b, k=k, given_ids=ids, given_logprobs=given, workspace=ws,
                    workspace_bytes=need, stream=stream())
        ann.ann_row_distillation(**what, loss=loss, lse=lse, logprobs=logprobs)
        ann.ann_row_distillation_backward(**what, lse=lse, logprobs=logprobs, g_loss=g, dq=dq, dq_stride=d, drows=drows, drows_stride=d, drow_bias=dbias)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    with torch.cuda.graph(graph):
        both()
    for case in cases + cases:
        for to, x in zip(held, case):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in (loss, lse, logprobs, dq, drows, dbias)]
        ws.fill_(0xFF)
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(replayed, (loss, lse, logprobs, dq, drows, dbias)))
