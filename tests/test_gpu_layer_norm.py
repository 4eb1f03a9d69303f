"""Layer norm and its gradients against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu
# additions that follow each other in a row's sum (at most 32 pieces of a lane, 9 exchanges and wavefronts) and the roundings around them
CHAIN = 64


def types(ann):
    return {"f32": ann.F32, "f16": ann.F16, "bf16": ann.BF16}


def strided(x, pad, offset=0):
    """x on the GPU as a view with a row stride of its own (and `offset` elements from the allocation's start)."""
    n, d = x.shape
    buf = torch.full((n * (d + pad) + offset,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[offset:].view(n, d + pad)[:, :d]
    view.copy_(x)
    return view


def case(n, d, dtype, wtype, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    t, wt = R.DTYPES[dtype], R.DTYPES[wtype]
    x = (torch.randn(n, d, generator=g) * torch.exp(torch.randn(d, generator=g)) + offset).to(t)
    return x, (1 + 0.3 * torch.randn(d, generator=g)).to(wt), (0.3 * torch.randn(d, generator=g)).to(wt), torch.randn(n, d, generator=g).to(t)


SHAPES = [(1, 1), (1, 768), (3, 2), (5, 7), (64, 16), (2, 63), (33, 100), (9, 128), (17, 129), (4, 511), (3, 513), (2, 960), (3, 2048), (2, 2056),
          (3, 5000), (2, 8192), (2, 16384), (2, 16392), (1, 40001), (1000, 96), (3001, 24)]


@pytest.mark.parametrize("dtype, wtype", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, d", SHAPES)
def test_forward_and_backward(n, d, dtype, wtype):
    import paper_2503_17911_amd as ann
    for pad, shift in ((0, 0), (8, 0), (4, 2), (1, 1)):
        x, w, b, dy = case(n, d, dtype, wtype, n * 131 + d + pad)
        check(ann, x, w, b, dy, 1e-5, pad, shift)


def test_rows_far_from_zero_constant_rows_and_no_weights():
    import paper_2503_17911_amd as ann
    x, w, b, dy = case(50, 200, "f32", "f32", 1, offset=1000.0)
    check(ann, x, w, b, dy, 1e-5, 0, 0)
    x[7] = 3.25   # a row without any spread: rstd = eps^-1/2
    check(ann, x, w, b, dy, 1e-3, 0, 0)
    check(ann, x, None, b, dy, 1e-5, 0, 0)
    check(ann, x, w, None, dy, 1e-5, 0, 0)
    check(ann, x, None, None, dy, 0.5, 3, 0)


def check(ann, x, w, b, dy, eps, pad, shift):
    T = types(ann)
    name = {v: k for k, v in R.DTYPES.items()}
    n, d = x.shape
    t, wt = x.dtype, (w if w is not None else b).dtype if (w is not None or b is not None) else x.dtype
    half = R.half_step(t)
    xd, dyd = strided(x, pad, shift), strided(dy, pad, shift)
    wd, bd = (None if v is None else v.cuda() for v in (w, b))
    y, dx = strided(torch.zeros_like(x), pad, shift), strided(torch.zeros_like(x), pad, shift)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ann.ann_layer_norm(xd, n, d, xd.stride(0), T[name[t]], wd, bd, T[name[wt]], eps, y, y.stride(0), mean, rstd, torch.cuda.current_stream().cuda_stream)
    y64, mean64, rstd64 = R.layer_norm(x, w, b, eps)
    big = x.double().abs().amax(1)
    w64 = torch.ones(d, dtype=R.F64) if w is None else w.double()
    b64 = torch.zeros(d, dtype=R.F64) if b is None else b.double()
    # the mean may err by CHAIN half steps of the largest element; so may each centred value; the variance's relative error
    # follows from both (a constant row's variance is that error's square against eps)
    off = CHAIN * R.U32 * big
    assert ((mean.cpu().double() - mean64).abs() <= off + 1e-300).all()
    rel = CHAIN * R.U32 + 2 * off * rstd64 + (off * rstd64) ** 2
    assert ((rstd.cpu().double() / rstd64 - 1).abs() <= rel).all()
    tol = half * y64.abs() + R.smallest_step(t) + w64.abs() * (2 * off * rstd64)[:, None] + (rel[:, None] + 8 * R.U32) * ((y64 - b64).abs() + b64.abs())
    assert ((y.cpu().double() - y64).abs() <= tol * (1 + half)).all()

    need = ann.ann_layer_norm_backward_workspace(n, d)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read before it is written)
    dw, db = torch.empty(d, dtype=wt, device="cuda"), torch.empty(d, dtype=wt, device="cuda")
    ann.ann_layer_norm_backward(dyd, dyd.stride(0), xd, xd.stride(0), n, d, T[name[t]], wd, T[name[wt]], mean, rstd, dx, dx.stride(0), dw, db,
                                ws, need, torch.cuda.current_stream().cuda_stream)
    mean, rstd = mean.cpu(), rstd.cpu()
    dx64, dw64, db64 = R.layer_norm_grad(dy, x, w, mean, rstd)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    a = dy.double() * w64
    size = rstd.double()[:, None] * (a.abs() + a.abs().mean(1, keepdim=True) + xh.abs() * (a * xh).abs().mean(1, keepdim=True))
    assert ((dx.cpu().double() - dx64).abs() <= (half * dx64.abs() + R.smallest_step(t) + CHAIN * R.U32 * size) * (1 + half)).all()
    steps = n / 512 + 4 + CHAIN   # rows to a group, groups to a workgroup, workgroups to a column
    whalf = R.half_step(wt)
    for got, want, terms in ((dw, dw64, (dy.double() * xh).abs().sum(0)), (db, db64, dy.double().abs().sum(0))):
        assert ((got.cpu().double() - want).abs() <= (whalf * want.abs() + R.smallest_step(wt) + steps * R.U32 * terms) * (1 + whalf)).all()
    # only the weight's, only the bias', neither: the same dx, and nothing needed for neither
    again = torch.zeros_like(dx)
    for one in (dict(dweight=torch.empty_like(dw)), dict(dbias=torch.empty_like(db)), {}):
        ann.ann_layer_norm_backward(dyd, dyd.stride(0), xd, xd.stride(0), n, d, T[name[t]], wd, T[name[wt]], mean.cuda(), rstd.cuda(), again,
                                    again.stride(0), workspace=ws if one else None, workspace_bytes=need if one else 0,
                                    stream=torch.cuda.current_stream().cuda_stream, **one)
        assert torch.equal(again.cpu(), dx.cpu())
        for f, v in one.items():
            assert torch.equal(v.cpu(), {"dweight": dw, "dbias": db}[f].cpu())


def test_nothing_between_rows_is_written_and_in_place_works():
    import paper_2503_17911_amd as ann
    x, w, b, dy = case(37, 100, "bf16", "f32", 5)
    st = torch.cuda.current_stream().cuda_stream
    wide = torch.full((37, 120), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :100] = x.cuda()
    apart = torch.empty(37, 100, dtype=torch.bfloat16, device="cuda")
    ann.ann_layer_norm(wide, 37, 100, 120, ann.BF16, w.cuda(), b.cuda(), ann.F32, 1e-5, apart, 100, stream=st)
    ann.ann_layer_norm(wide, 37, 100, 120, ann.BF16, w.cuda(), b.cuda(), ann.F32, 1e-5, wide, 120, stream=st)
    assert torch.equal(wide[:, :100], apart) and (wide[:, 100:] == 7.0).all()
    # the gradient over dy
    mean, rstd = torch.randn(37, device="cuda"), torch.rand(37, device="cuda") + 0.5
    xd, d1, d2 = x.cuda(), dy.cuda(), dy.cuda()
    ann.ann_layer_norm_backward(d1, 100, xd, 100, 37, 100, ann.BF16, None, ann.BF16, mean, rstd, apart, 100, stream=st)
    ann.ann_layer_norm_backward(d2, 100, xd, 100, 37, 100, ann.BF16, None, ann.BF16, mean, rstd, d2, 100, stream=st)
    assert torch.equal(d2, apart)


def test_no_rows_give_zero_gradients_of_weights():
    import paper_2503_17911_amd as ann
    dw, db = torch.full((100,), 7.0, device="cuda"), torch.full((100,), 7.0, device="cuda")
    ann.ann_layer_norm_backward(None, 0, None, 0, 0, 100, ann.BF16, None, ann.F32, None, None, None, 0, dw, db, stream=torch.cuda.current_stream().cuda_stream)
    assert (dw == 0).all() and (db == 0).all()


def test_not_a_number_stays_in_its_row():
    import paper_2503_17911_amd as ann
    x, w, b, dy = case(40, 96, "f32", "f32", 9)
    x[3, 5], x[17, 0] = float("nan"), float("inf")
    y, xd = torch.empty(40, 96, device="cuda"), x.cuda()
    ann.ann_layer_norm(xd, 40, 96, 96, ann.F32, w.cuda(), b.cuda(), ann.F32, 1e-5, y, 96, stream=torch.cuda.current_stream().cuda_stream)
    bad = torch.zeros(40, dtype=torch.bool)
    bad[[3, 17]] = True
    assert torch.equal(y.cpu().isnan().all(1), bad) and torch.equal(y.cpu().isnan().any(1), bad)


def test_gradient_against_differences():
    """dx, dw, db against central differences of the 64-bit forward pass along random directions."""
    import paper_2503_17911_amd as ann
    n, d, eps, step = 12, 200, 1e-5, 1e-5
    x, w, b, dy = case(n, d, "f32", "f32", 21)
    st = torch.cuda.current_stream().cuda_stream
    mean, rstd, y, dx = (torch.empty(s, device="cuda") for s in ((n,), (n,), (n, d), (n, d)))
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    need = ann.ann_layer_norm_backward_workspace(n, d)
    ws, xd, dyd, wd = torch.empty(need, dtype=torch.uint8, device="cuda"), x.cuda(), dy.cuda(), w.cuda()
    ann.ann_layer_norm(xd, n, d, d, ann.F32, wd, b.cuda(), ann.F32, eps, y, d, mean, rstd, st)
    ann.ann_layer_norm_backward(dyd, d, xd, d, n, d, ann.F32, wd, ann.F32, mean, rstd, dx, d, dw, db, ws, need, st)

    def loss(x, w, b):
        return float((R.layer_norm(x, w, b, eps)[0] * dy.double()).sum())

    g = torch.Generator().manual_seed(3)
    x, w, b = x.double(), w.double(), b.double()
    for _ in range(4):
        ex, ew, eb = (torch.randn(v.shape, generator=g, dtype=R.F64) for v in (x, w, b))
        slope = (loss(x + step * ex, w + step * ew, b + step * eb) - loss(x - step * ex, w - step * ew, b - step * eb)) / (2 * step)
        terms = [(dx.cpu().double() * ex), (dw.cpu().double() * ew), (db.cpu().double() * eb)]
        got, size = sum(float(v.sum()) for v in terms), sum(float(v.abs().sum()) for v in terms)
        # every gradient errs by a few fp32 steps of its terms; the difference by its square's share and 64-bit rounding
        assert abs(got - slope) <= 4 * CHAIN * R.U32 * size + 1e-4


def test_other_stream_and_graph():
    import paper_2503_17911_amd as ann
    x, w, b, dy = case(300, 768, "bf16", "f32", 11)
    xd, wd, bd, dyd = x.cuda(), w.cuda(), b.cuda(), dy.cuda()
    need = ann.ann_layer_norm_backward_workspace(300, 768)

    def outputs():
        return [torch.zeros_like(xd), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros_like(xd),
                torch.zeros(768, device="cuda"), torch.zeros(768, device="cuda"), torch.zeros(need, dtype=torch.uint8, device="cuda")]

    def both(o):
        st = torch.cuda.current_stream().cuda_stream
        ann.ann_layer_norm(xd, 300, 768, 768, ann.BF16, wd, bd, ann.F32, 1e-5, o[0], 768, o[1], o[2], st)
        ann.ann_layer_norm_backward(dyd, 768, xd, 768, 300, 768, ann.BF16, wd, ann.F32, o[1], o[2], o[3], 768, o[4], o[5], o[6], need, st)

    want, other, graphed = outputs(), outputs(), outputs()
    both(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both(other)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(graphed)
    for replay in range(3):
        xd.copy_(torch.randn(300, 768, device="cuda"))
        both(want)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(want[:6], graphed[:6]):
            assert torch.equal(a, c), replay
    with torch.cuda.stream(side):
        both(other)
    side.synchronize()
    for a, c in zip(want[:6], other[:6]):
        assert torch.equal(a, c)
