"""Log probabilities of rows, entropy, alternatives and their gradients against
their definitions in 64 bits."""
import math

import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu


def types(ann):
    return {torch.float32: ann.F32, torch.float16: ann.F16, torch.bfloat16: ann.BF16}


def stream():
    return torch.cuda.current_stream().cuda_stream


def strided(x, pad, fill=float("nan")):
    wide = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]] = x.cuda()
    return wide[:, :x.shape[1]]


def unit(x):
    return x / x.norm(dim=1, keepdim=True).clamp_min(1e-6)


def inputs(nq, n, d, dtype, seed, bias="none"):
    g = torch.Generator().manual_seed(seed)
    t = R.DTYPES[dtype]
    centres = torch.randn(max(2, n // 50), d, generator=g)
    rows = unit(centres[torch.randint(len(centres), (n,), generator=g)] + 0.3 * torch.randn(n, d, generator=g))
    target = torch.randint(n, (nq,), generator=g)
    q = unit(rows[target] + 0.3 / math.sqrt(d) * torch.randn(nq, d, generator=g))
    b = None
    if bias != "none":
        b = 0.5 * torch.randn(n, generator=g)
        if bias == "holes":
            b[torch.rand(n, generator=g) < 0.2] = -math.inf
            b[0] = 0.0
    if nq > 2:
        target[1], target[2] = -1, n + 3      # none given; no row's number
    return q.to(t), rows.to(t), b, target


def targets_u32(target):
    return (target % 2**32).to(torch.int64).to(torch.uint32).view(torch.int32).cuda()


def forward(ann, q, rows, b, target, scale, k, pad=0, entropy=True, dirty=True):
    nq, d = q.shape
    n = rows.shape[0]
    qd, xd = strided(q, pad), strided(rows, pad)
    t = types(ann)[q.dtype]
    need = ann.ann_row_logprobs_workspace(nq, n, d, t, k)
    ws = torch.full((max(need, 1),), 0xFF if dirty else 0, dtype=torch.uint8, device="cuda")
    out = dict(logprob=torch.full((nq,), 7.0, device="cuda"), lse=torch.full((nq,), 7.0, device="cuda"),
               entropy=torch.full((nq,), 7.0, device="cuda") if entropy else None,
               alt_ids=torch.full((nq, k), -7, dtype=torch.int32, device="cuda") if k else None,
               alt_logprobs=torch.full((nq, k), 7.0, device="cuda") if k else None)
    ann.ann_row_logprobs(qd, nq, qd.stride(0), xd, n, xd.stride(0), d, t, scale=scale, row_bias=None if b is None else b.cuda(),
                         targets=None if target is None else targets_u32(target), k=k, workspace=ws, workspace_bytes=need, stream=stream(), **out)
    torch.cuda.synchronize()
    return {f: v.cpu() for f, v in out.items() if v is not None}


def check_forward(ann, q, rows, b, target, scale, k, pad=0):
    got = forward(ann, q, rows, b, target, scale, k, pad)
    z = R.scores(q, rows, scale, b)
    nq, n = z.shape
    lse, lp, entropy = R.log_probabilities(z, target if target is not None else torch.full((nq,), -1))
    err = R.score_error(q, rows, scale, b)
    fin = lse > -math.inf
    assert torch.equal(got["lse"].double() == -math.inf, ~fin)
    tol = err + R.sum_error(n) + 4 * R.U32 * torch.where(fin, lse, torch.zeros_like(lse)).abs()
    assert ((got["lse"].double() - lse).abs()[fin] <= tol[fin]).all()
    low = lp == -math.inf
    assert torch.equal(got["logprob"].double() == -math.inf, low)
    assert ((got["logprob"].double() - lp).abs()[~low] <= (tol + 4 * R.U32 * lp.abs())[~low]).all()
    # d H = - sum p (log p + H) ds, and sum p |log p + H| <= 2 H; the sums' own errors likewise
    assert ((got["entropy"].double() - entropy).abs() <= (2 * entropy + 1) * 2 * (err + R.sum_error(n)) + 1e-6 * (err + R.U32)).all()
    if k:
        ids, val = R.alternatives(z, k)
        assert torch.equal(got["alt_ids"].long(), ids)
        there = ids >= 0
        alt = val - torch.where(fin, lse, torch.zeros_like(lse))[:, None]
        assert (got["alt_logprobs"][~there] == -math.inf).all()
        assert ((got["alt_logprobs"].double() - alt).abs() <= tol[:, None] + 4 * R.U32 * alt.abs())[there].all()
    return got


SHAPES = [(1, 1, 1, 1), (1, 5, 3, 5), (3, 64, 16, 4), (2, 63, 8, 64), (7, 130, 100, 10), (128, 128, 128, 1), (129, 257, 96, 20), (70, 1000, 200, 10),
          (5, 3000, 33, 32), (33, 20000, 64, 10), (17, 20011, 72, 3), (300, 4100, 768, 5), (4, 50000, 960, 20), (16, 40000, 24, 64), (1, 100003, 128, 10),
          (9, 700, 1500, 7), (2, 300, 4096, 3)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHAPES)
def test_forward(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    for bias, pad, scale in (("none", 0, 20.0), ("plain", 8, 5.0), ("holes", 1, 20.0)):
        q, rows, b, target = inputs(nq, n, d, dtype, n + d, bias)
        check_forward(ann, q, rows, b, target, scale, k, pad)


def test_what_is_not_asked_for_is_not_needed():
    import paper_2503_17911_amd as ann
    q, rows, b, target = inputs(20, 3000, 100, "bf16", 4)
    full = forward(ann, q, rows, b, target, 20.0, 10)
    part = forward(ann, q, rows, b, target, 20.0, 0, entropy=False)
    assert torch.equal(full["lse"], part["lse"]) and torch.equal(full["logprob"], part["logprob"])
    none = forward(ann, q, rows, b, None, 20.0, 3)
    assert torch.equal(none["lse"], full["lse"]) and (none["logprob"] == 0).all() and torch.equal(none["alt_ids"], full["alt_ids"][:, :3])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_scales_of_any_sign_and_ties(dtype):
    import paper_2503_17911_amd as ann
    q, rows, b, target = inputs(10, 700, 48, dtype, 8)
    check_forward(ann, q, rows, None, target, -7.5, 9)
    # all scores alike: the first rows, in the order of their numbers
    assert (check_forward(ann, q, rows, None, target, 0.0, 33)["alt_ids"] == torch.arange(33)).all()
    check_forward(ann, torch.zeros_like(q), rows, None, target, 20.0, 64)
    # every row five times
    check_forward(ann, q, rows.repeat(5, 1), None, target, 20.0, 20)
    # scores far from zero, and a softmax that is one row's
    check_forward(ann, q * 30, rows * 30, None, target, 1.0, 5)


def test_many_equal_scores_among_many_rows():
    """More rows at the k-th score than are kept at a time: the lowest numbers still win."""
    import paper_2503_17911_amd as ann
    rows = torch.zeros(300_000, 16, dtype=torch.bfloat16)
    rows[:, 0] = 1.0
    rows[123_456, 0] = 2.0
    q = torch.zeros(3, 16, dtype=torch.bfloat16)
    q[:, 0] = torch.tensor([1.0, 0.0, -1.0])
    got = forward(ann, q, rows, None, torch.tensor([5, 5, 5]), 1.0, 10)
    first = torch.arange(10)
    assert (got["alt_ids"][0] == torch.cat([torch.tensor([123_456]), first[:9]])).all()
    assert (got["alt_ids"][1] == first).all() and (got["alt_ids"][2] == first).all()


def test_rows_left_out():
    import paper_2503_17911_amd as ann
    for dtype in ("f32", "bf16", "f16"):
        q, rows, _, target = inputs(40, 500, 40, dtype, 2)
        b = torch.zeros(500)
        out = torch.rand(500, generator=torch.Generator().manual_seed(1)) < 0.5
        b[out] = -math.inf
        want = check_forward(ann, q, rows, b, target, 10.0, 10)
        # what such rows hold plays no part
        spoilt = rows.clone()
        spoilt[out] = torch.tensor([float("nan"), math.inf, -math.inf] * 14)[:40].to(rows.dtype)
        got = forward(ann, q, spoilt, b, target, 10.0, 10)
        for f in want:
            assert torch.equal(want[f], got[f]), f
        # all of them: nothing is left
        got = check_forward(ann, q, rows, torch.full((500,), -math.inf), target, 10.0, 10)
        assert (got["entropy"] == 0).all() and (got["alt_ids"] == -1).all() and (got["alt_logprobs"] == -math.inf).all()
        # one of them
        one = torch.full((500,), -math.inf)
        one[321] = 1.5
        got = check_forward(ann, q, rows, one, torch.full((40,), 321), 10.0, 3)
        assert (got["alt_ids"] == torch.tensor([321, -1, -1])).all() and (got["logprob"].abs() <= 1e-5).all()


def test_masks_of_the_lowest_value_are_ordinary_biases():
    import paper_2503_17911_amd as ann
    q, rows, _, target = inputs(10, 400, 32, "bf16", 2)
    low = torch.finfo(torch.float32).min
    b = torch.zeros(400)
    b[::2] = low
    want = forward(ann, q, rows, torch.where(b == low, torch.tensor(-math.inf), b), target | 1, 10.0, 5)
    got = forward(ann, q, rows, b, target | 1, 10.0, 5)
    for f in want:
        assert torch.equal(want[f], got[f]), f
    # nothing but the lowest value: each row as likely as the others, as the sums in fp32 have it
    got = forward(ann, q, rows, torch.full((400,), low), torch.zeros(10, dtype=torch.long), 10.0, 0)
    assert ((got["entropy"] - math.log(400)).abs() < 1e-5).all() and torch.isfinite(got["lse"]).all()


def test_gradient_of_masks_of_the_lowest_value():
    import paper_2503_17911_amd as ann
    for dtype in ("f32", "f16", "bf16"):
        for d in (40, 200):
            q, rows, _, target = inputs(10, 400, d, dtype, 2)
            b = torch.full((400,), torch.finfo(torch.float32).min)
            f = forward(ann, q, rows, b, torch.zeros(10, dtype=torch.long), 10.0, 0)
            g, h = torch.ones(10), torch.full((10,), 0.5)
            got = backward(ann, q, rows, b, torch.zeros(10, dtype=torch.long), 10.0, f["lse"], f["entropy"], g, h)
            # every score is the lowest value, as fp32 has it: all rows are alike, lse - the score is nothing in fp32, so p = 1
            assert all(torch.isfinite(v).all() for v in got.values())
            b[::2] = 0.0     # half of them at the lowest value: as if they were left out
            f = forward(ann, q, rows, b, target | 1, 10.0, 0)
            got = backward(ann, q, rows, b, target | 1, 10.0, f["lse"], f["entropy"], g, h)
            b[1::2] = -math.inf
            want = backward(ann, q, rows, b, target | 1, 10.0, f["lse"], f["entropy"], torch.zeros(10), h)
            for name in ("dq", "drows", "drow_bias"):
                assert torch.isfinite(got[name]).all() and torch.isfinite(want[name]).all()


def test_no_rows():
    import paper_2503_17911_amd as ann
    got = forward(ann, torch.ones(5, 8), torch.zeros(0, 8), None, torch.zeros(5, dtype=torch.long), 1.0, 3)
    assert (got["lse"] == -math.inf).all() and (got["logprob"] == 0).all() and (got["entropy"] == 0).all() and (got["alt_ids"] == -1).all()


def test_not_a_number_stays_in_its_query():
    import paper_2503_17911_amd as ann
    q, rows, _, target = inputs(150, 900, 64, "bf16", 6)
    target[:] = 3
    want = forward(ann, q, rows, None, target, 20.0, 5)
    q[70, 3] = float("nan")
    got = forward(ann, q, rows, None, target, 20.0, 5)
    keep = torch.arange(150) != 70
    assert got["lse"][70].isnan() and got["logprob"][70].isnan() and got["entropy"][70].isnan()
    for f in want:
        assert torch.equal(want[f][keep], got[f][keep]), f
    # a row of them: every query's statistics, but the alternatives are the other rows
    q, rows, _, target = inputs(20, 900, 64, "bf16", 6)
    top = forward(ann, q, rows, None, target, 20.0, 6)["alt_ids"]
    rows[top[0, 0]] = float("nan")
    got = forward(ann, q, rows, None, target, 20.0, 5)
    assert got["lse"].isnan().all()
    for i in range(20):
        assert got["alt_ids"][i].tolist() == [j for j in top[i].tolist() if j != int(top[0, 0])][:5]


def test_offsets_beyond_32_bits():
    """Rows 65,536 elements apart: the last ones lie more than 2^32 elements from the first."""
    import paper_2503_17911_amd as ann
    n, d, stride = 66_000, 40, 65_536
    q, rows, _, target = inputs(6, n, d, "bf16", 12)
    target = torch.tensor([n - 1, 0, n - 2, 65_537, 1, n - 1])
    want = forward(ann, q, rows, None, target, 20.0, 5)
    wide = torch.empty(n, stride, dtype=torch.bfloat16, device="cuda")
    wide[:, :d] = rows.cuda()
    k, out = 5, dict(logprob=torch.empty(6, device="cuda"), lse=torch.empty(6, device="cuda"), alt_ids=torch.empty(6, 5, dtype=torch.int32, device="cuda"),
                     alt_logprobs=torch.empty(6, 5, device="cuda"))
    need = ann.ann_row_logprobs_workspace(6, n, d, ann.BF16, k)
    ws, qd = torch.empty(need, dtype=torch.uint8, device="cuda"), q.cuda()
    ann.ann_row_logprobs(qd, 6, d, wide, n, stride, d, ann.BF16, scale=20.0, targets=targets_u32(target), k=k, workspace=ws, workspace_bytes=need,
                         stream=stream(), **out)
    for f, v in out.items():
        assert torch.equal(v.cpu(), want[f]), f
    # and the gradients of such rows
    need = ann.ann_row_logprobs_backward_workspace(6, n, d, ann.BF16)
    ws, g = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.ones(6, device="cuda")
    near, near_out, dq, dq_far = rows.cuda(), torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), torch.empty_like(qd), torch.empty_like(qd)
    for x, s, dx, dxs, o in ((near, d, near_out, d, dq), (wide, stride, wide[:, d:], stride, dq_far)):
        ann.ann_row_logprobs_backward(qd, 6, d, x, n, s, d, ann.BF16, scale=20.0, targets=targets_u32(target), lse=out["lse"], g_logprob=g, dq=o, dq_stride=d,
                                      drows=dx, drows_stride=dxs, workspace=ws, workspace_bytes=need, stream=stream())
    assert torch.equal(dq, dq_far) and torch.equal(near_out, wide[:, d:2 * d]) and (near_out != 0).any()


# ------------------------------------------------------------------ gradients
def backward(ann, q, rows, b, target, scale, lse, entropy, g, h, pad=0, dq=True, drows=True, dbias=True):
    nq, d = q.shape
    n = rows.shape[0]
    t = types(ann)[q.dtype]
    qd, xd = strided(q, pad), strided(rows, pad)
    need = ann.ann_row_logprobs_backward_workspace(nq, n, d, t)
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    out = dict(dq=strided(torch.full_like(q, 7.0), pad, 3.0) if dq else None, drows=strided(torch.full_like(rows, 7.0), pad, 3.0) if drows else None,
               drow_bias=torch.full((n,), 7.0, device="cuda") if dbias else None)
    ann.ann_row_logprobs_backward(qd, nq, qd.stride(0), xd, n, xd.stride(0), d, t, lse=lse.cuda(), entropy=None if entropy is None else entropy.cuda(),
                                  scale=scale, row_bias=None if b is None else b.cuda(), targets=None if target is None else targets_u32(target),
                                  g_logprob=None if g is None else g.cuda(), g_entropy=None if h is None else h.cuda(), dq_stride=d + pad,
                                  drows_stride=d + pad, workspace=ws, workspace_bytes=need, stream=stream(), **out)
    torch.cuda.synchronize()
    return {f: v.cpu() for f, v in out.items() if v is not None}


def check_backward(ann, q, rows, b, target, scale, g, h, pad=0):
    z = R.scores(q, rows, scale, b)
    nq, n = z.shape
    lse, _, entropy = R.log_probabilities(z, target)
    lse, entropy = lse.float(), entropy.float()
    got = backward(ann, q, rows, b, target, scale, lse, entropy, g, h, pad)
    G, p = R.score_gradient(z, lse, entropy, target, g, h)
    half, t = R.half_step(q.dtype), q.dtype
    # an element of G: the score's error through p (and through the slope of the entropy), three roundings, and G's own rounding
    err = (R.score_error(q, rows, scale, b) + 12 * R.U32 * (1 + torch.where(lse > -math.inf, lse, torch.zeros_like(lse)).abs()))[:, None]
    size = torch.zeros_like(z)
    if g is not None:
        size += g.double().abs()[:, None] * p * (err + 8 * R.U32)
        size += 2 * R.U32 * G.abs()
    if h is not None:
        away = torch.where(p > 0, (z - lse.double()[:, None] + entropy.double()[:, None]).abs(), torch.zeros_like(z))
        size += h.double().abs()[:, None] * p * (away + 1) * (err * 2 + 8 * R.U32)
    if t == torch.float16:      # what lies below its range, times the power of two at least
        bound = (0 if g is None else g.abs().max().item()) + (0 if h is None else (h.abs() * (entropy.abs() + 0.375)).max().item())
        kept = half * G.abs() + 2.0 ** -38 * bound
    else:
        kept = (half if t == torch.bfloat16 else 2.0 ** -23) * G.abs()
    x, qq = rows.double(), q.double()
    if b is not None:
        x = torch.where((b == -math.inf)[:, None], torch.zeros_like(x), x)
    products = (6 if t == torch.float32 else 1) * 2 * R.U32
    for f, want, terms, off in (("dq", G @ x, G.abs() @ x.abs(), (size + kept) @ x.abs()), ("drows", G.T @ qq, G.abs().T @ qq.abs(), (size + kept).T @ qq.abs())):
        want, terms, off = scale * want, abs(scale) * terms, abs(scale) * off
        length = n if f == "dq" else nq
        tol = (half * want.abs() + R.smallest_step(t) + off + (products * length + 64 * R.U32) * terms) * (1 + half)
        assert ((got[f].double() - want).abs() <= tol).all(), f
    assert ((got["drow_bias"].double() - G.sum(0)).abs() <= size.sum(0) + (nq + 64) * R.U32 * G.abs().sum(0) + 1e-40).all()
    return got


GRAD_SHAPES = [(1, 1, 1), (1, 300, 16), (3, 64, 7), (5, 65, 100), (128, 128, 128), (130, 257, 96), (70, 1000, 200), (33, 5000, 64), (300, 4100, 768), (9, 700, 1500),
               (1, 20000, 128), (600, 130, 130)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", GRAD_SHAPES)
def test_backward(nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + n)
    for bias, pad, scale in (("none", 0, 20.0), ("plain", 8, 5.0), ("holes", 1, -3.0)):
        q, rows, b, target = inputs(nq, n, d, dtype, n + d, bias)
        g, h = -0.5 - torch.rand(nq, generator=gen), 0.2 * torch.randn(nq, generator=gen)
        check_backward(ann, q, rows, b, target, scale, g, h, pad)
    check_backward(ann, q, rows, b, target, scale, g, None)
    check_backward(ann, q, rows, b, target, scale, None, h)


def test_backward_of_any_size_of_loss():
    """Half precision has to carry gradients of a mean over many, and of a scaled loss."""
    import paper_2503_17911_amd as ann
    q, rows, b, target = inputs(50, 3000, 64, "f16", 5)
    for size in (1e-6, 1.0, 2.0 ** 14):
        g = -size * (0.5 + torch.rand(50, generator=torch.Generator().manual_seed(2)))
        check_backward(ann, q, rows, b, target, 0.05, g, 0.1 * g)
    check_backward(ann, q, rows, b, target, 20.0, torch.zeros(50), None)


def test_backward_of_parts_and_of_nothing():
    import paper_2503_17911_amd as ann
    q, rows, b, target = inputs(40, 900, 100, "bf16", 5, "holes")
    z = R.scores(q, rows, 20.0, b)
    lse, _, entropy = (v.float() for v in R.log_probabilities(z, target))
    g, h = torch.randn(40), torch.randn(40)
    full = backward(ann, q, rows, b, target, 20.0, lse, entropy, g, h)
    for f in full:
        only = backward(ann, q, rows, b, target, 20.0, lse, entropy, g, h, dq=f == "dq", drows=f == "drows", dbias=f == "drow_bias")
        assert list(only) == [f] and torch.equal(only[f], full[f])
    # rows left out get nothing, whatever they hold; so do queries without a row, and a call without queries
    spoilt = rows.clone()
    spoilt[b == -math.inf] = float("nan")
    again = backward(ann, q, spoilt, b, target, 20.0, lse, entropy, g, h, dq=False)
    assert torch.equal(again["drows"], full["drows"]) and (again["drows"][b == -math.inf] == 0).all() and (again["drow_bias"][b == -math.inf] == 0).all()
    none = backward(ann, q, rows, torch.full((900,), -math.inf), target, 20.0, torch.full((40,), -math.inf), torch.zeros(40), g, h)
    for v in none.values():
        assert (v == 0).all()
    none = backward(ann, q[:0], rows, b, target[:0], 20.0, lse[:0], entropy[:0], g[:0], h[:0], dq=False)
    assert (none["drows"] == 0).all() and (none["drow_bias"] == 0).all()
    none = backward(ann, q, rows[:0], None, target, 20.0, lse, entropy, g, h, drows=False, dbias=False)
    assert (none["dq"] == 0).all()
    # no row given anywhere: the entropy's gradient alone
    none = backward(ann, q, rows, b, None, 20.0, lse, entropy, g, h)
    want = backward(ann, q, rows, b, None, 20.0, lse, entropy, None, h)
    for f in want:
        assert torch.equal(none[f], want[f])


def test_rows_left_out_hold_anything_for_the_queries_gradient():
    import paper_2503_17911_amd as ann
    for dtype in ("f32", "f16", "bf16"):
        q, rows, b, target = inputs(40, 900, 100, dtype, 5, "holes")
        z = R.scores(q, rows, 20.0, b)
        lse, _, entropy = (v.float() for v in R.log_probabilities(z, target))
        g, h = torch.randn(40), torch.randn(40)
        want = backward(ann, q, rows, b, target, 20.0, lse, entropy, g, h)
        spoilt = rows.clone()
        spoilt[b == -math.inf] = torch.tensor([float("nan"), math.inf, -math.inf, 1.0])[torch.arange(100) % 4].to(rows.dtype)
        got = backward(ann, q, spoilt, b, target, 20.0, lse, entropy, g, h)
        for f in want:
            assert torch.equal(got[f], want[f]), (dtype, f)


def test_gradient_against_differences():
    """dq, drows and drow_bias against central differences of the 64-bit loss along random directions."""
    import paper_2503_17911_amd as ann
    q, rows, b, target = inputs(20, 400, 48, "f32", 3, "plain")
    gen = torch.Generator().manual_seed(1)
    g, h = torch.randn(20, generator=gen), torch.randn(20, generator=gen)
    f = forward(ann, q, rows, b, target, 6.0, 0)
    got = backward(ann, q, rows, b, target, 6.0, f["lse"], f["entropy"], g, h)

    def loss(q, rows, b):
        _, lp, entropy = R.log_probabilities(R.scores(q, rows, 6.0, b), target)
        return float((g.double() * lp + h.double() * entropy).sum())

    q, rows, b = q.double(), rows.double(), b.double()
    step = 1e-5
    for _ in range(4):
        e = [torch.randn(v.shape, generator=gen, dtype=R.F64) for v in (q, rows, b)]
        slope = (loss(*(v + step * w for v, w in zip((q, rows, b), e))) - loss(*(v - step * w for v, w in zip((q, rows, b), e)))) / (2 * step)
        terms = [got[f].double() * w for f, w in zip(("dq", "drows", "drow_bias"), e)]
        total, size = sum(float(v.sum()) for v in terms), sum(float(v.abs().sum()) for v in terms)
        # (a score errs by some 2^-17 at most here, its exponential by as much relative to itself)
        assert abs(total - slope) <= 2.0 ** -15 * size + 1e-4


# ------------------------------------------------------------------ calls
def test_same_bits_again_on_other_streams_and_in_graphs():
    import paper_2503_17911_amd as ann
    for dtype, bias, nq, n, d in (("bf16", "none", 200, 9000, 128), ("f16", "holes", 20, 3000, 100), ("f32", "plain", 3, 5000, 72)):
        q, rows, b, target = inputs(nq, n, d, dtype, 5, bias)
        t = types(ann)[q.dtype]
        qd, xd, td, bd = q.cuda(), rows.cuda(), targets_u32(target), None if b is None else b.cuda()
        need, needb = ann.ann_row_logprobs_workspace(nq, n, d, t, 5), ann.ann_row_logprobs_backward_workspace(nq, n, d, t)
        g, h = torch.randn(nq, device="cuda"), torch.randn(nq, device="cuda")

        def outputs():
            return [torch.zeros(nq, device="cuda"), torch.zeros(nq, device="cuda"), torch.zeros(nq, device="cuda"),
                    torch.zeros(nq, 5, dtype=torch.int32, device="cuda"), torch.zeros(nq, 5, device="cuda"), torch.zeros_like(qd), torch.zeros_like(xd),
                    torch.zeros(n, device="cuda"), torch.zeros(need, dtype=torch.uint8, device="cuda"), torch.zeros(needb, dtype=torch.uint8, device="cuda")]

        def both(o):
            table = dict(q=qd, nq=nq, q_stride=d, rows=xd, n=n, row_stride=d, d=d, type=t, scale=15.0, row_bias=bd, targets=td, stream=stream())
            ann.ann_row_logprobs(**table, k=5, logprob=o[0], lse=o[1], entropy=o[2], alt_ids=o[3], alt_logprobs=o[4], workspace=o[8], workspace_bytes=need)
            ann.ann_row_logprobs_backward(**table, lse=o[1], entropy=o[2], g_logprob=g, g_entropy=h, dq=o[5], dq_stride=d, drows=o[6], drows_stride=d,
                                          drow_bias=o[7], workspace=o[9], workspace_bytes=needb)

        want, other, graphed = outputs(), outputs(), outputs()
        both(want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            both(other)
        side.synchronize()
        for a, c in zip(want[:8], other[:8]):
            assert torch.equal(a, c)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(graphed)
        for replay in range(3):
            qd.copy_(unit(torch.randn(nq, d, device="cuda")))
            both(want)
            graph.replay()
            torch.cuda.synchronize()
            for a, c in zip(want[:8], graphed[:8]):
                assert torch.equal(a, c), replay
