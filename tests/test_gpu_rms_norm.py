"""Root-mean-square norm with the residual's addition, its output in 8 bits, and its
gradients, against their definitions in 64 bits."""
import pytest
import torch

import encoder_reference as E
import head_reference as R
from test_gpu_layer_norm import strided, types

pytestmark = pytest.mark.gpu
# additions that follow each other in a row's sum (40 of a lane, exchanges and wavefronts) and the roundings around them
CHAIN = 64
NAMES = {v: k for k, v in R.DTYPES.items()}


def stream():
    return torch.cuda.current_stream().cuda_stream


def case(n, d, dtype, wtype, seed):
    g = torch.Generator().manual_seed(seed)
    t = R.DTYPES[dtype]
    spread = torch.exp(0.7 * torch.randn(d, generator=g))
    w = None if wtype is None else (1 + 0.3 * torch.randn(d, generator=g)).to(R.DTYPES[wtype])
    return [(torch.randn(n, d, generator=g) * spread * s).to(t) for s in (0.5, 1.0)] + [w] + [torch.randn(n, d, generator=g).to(t) for _ in range(2)]


SHAPES = [(1, 1), (1, 768), (3, 2), (5, 7), (64, 16), (2, 63), (33, 100), (9, 128), (17, 129), (4, 511), (3, 513), (2, 960), (3, 2048), (2, 2056),
          (3, 5000), (2, 8192), (2, 16384), (2, 16392), (1, 40001), (1000, 96), (3001, 24)]
TYPES = [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", None), ("bf16", "f32")]


@pytest.mark.parametrize("dtype, wtype", TYPES)
@pytest.mark.parametrize("n, d", SHAPES)
def test_forward_and_backward(n, d, dtype, wtype):
    import paper_2503_17911_amd as ann
    for pad, shift, with_residual in ((0, 0, True), (8, 0, False), (4, 2, True), (1, 1, True)):
        x, res, w, dy, ds = case(n, d, dtype, wtype, n * 131 + d + pad)
        check(ann, x, res if with_residual else None, w, dy, ds if with_residual else None, pad, shift)


def check(ann, x, res, w, dy, ds, pad, shift, eps=1e-6):
    n, d = x.shape
    t, wt = x.dtype, torch.float32 if w is None else w.dtype
    T, WT = types(ann)[NAMES[t]], types(ann)[NAMES[wt]] if w is not None else types(ann)[NAMES[t]]
    half, tiny = R.half_step(t), R.smallest_step(t)
    on = lambda v: None if v is None else strided(v, pad, shift)  # noqa: E731
    xd, rd, dyd, dsd, wd = on(x), on(res), on(dy), on(ds), None if w is None else w.cuda()
    y, kept, rstd = on(torch.zeros_like(x)), on(torch.zeros_like(x)), torch.empty(n, device="cuda")
    more = {} if res is None else dict(residual=rd, residual_stride=rd.stride(0), sum=kept, sum_stride=kept.stride(0))
    ann.ann_rms_norm(xd, n, d, xd.stride(0), T, wd, WT, eps, y, y.stride(0), rstd=rstd, stream=stream(), **more)
    h = x
    if res is not None:
        h, h64 = kept.cpu(), x.double() + res.double()
        assert ((h.double() - h64).abs() <= (half + R.U32) * (1 + half) * h64.abs() + tiny).all()
    y64, rstd64 = E.rms_norm(h, w, eps)
    rel = CHAIN * R.U32
    assert ((rstd.cpu().double() / rstd64 - 1).abs() <= rel).all()
    assert ((y.cpu().double() - y64).abs() <= (half + (rel + 4 * R.U32) * (1 + half)) * y64.abs() + tiny).all()
    # in 8 bits: the codes' own half step (2^-4 relative, 2^-10 among the smallest), and the fp32 roundings before it
    for group in (0, 32, 64, 128):
        groups = 1 if group == 0 else -(-d // group)
        codes = torch.full((n, d + pad), 0x55, dtype=torch.uint8, device="cuda")
        sc = torch.full((n, groups + 1), -7.0, device="cuda")
        kept8, rstd8 = on(torch.zeros_like(x)), torch.empty(n, device="cuda")
        if res is not None:
            more.update(sum=kept8, sum_stride=kept8.stride(0))
        ann.ann_rms_norm_e4m3(xd, n, d, xd.stride(0), T, wd, WT, eps, codes, d + pad, group, sc, groups + 1, rstd=rstd8, stream=stream(), **more)
        # (groups may ask for another number of lanes, and so for another order of the row's sum: held to the definition like rstd)
        assert ((rstd8.cpu().double() / rstd64 - 1).abs() <= rel).all() and (res is None or torch.equal(kept8, kept))
        assert (codes[:, d:] == 0x55).all() and (sc[:, groups] == -7.0).all()
        want = E.scales(y64, group)
        got = sc[:, :groups].cpu().double()
        assert ((got - want).abs() <= (rel + 8 * R.U32) * want).all()
        v = E.e4m3_values()[codes[:, :d].cpu().long()]
        at = torch.arange(d) // (group or d)
        exact = y64 / got[:, at]
        assert ((v - exact).abs() <= (2.0 ** -4 + (rel + 8 * R.U32) * 2) * exact.abs() + 2.0 ** -10).all()

    need = ann.ann_rms_norm_backward_workspace(n, d)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read before it is written)
    dx, dw = on(torch.zeros_like(x)), None if w is None else torch.empty(d, dtype=wt, device="cuda")
    hd = xd if res is None else kept
    more = {} if ds is None else dict(dsum=dsd, dsum_stride=dsd.stride(0))
    args = (dyd, dyd.stride(0), hd, hd.stride(0), n, d, T, wd, WT, rstd)
    ann.ann_rms_norm_backward(*args, dx, dx.stride(0), dweight=dw, workspace=ws, workspace_bytes=need, stream=stream(), **more)
    dx64, dw64, size, wsize = E.rms_norm_grad(dy, h, ds, w, rstd.cpu())
    assert ((dx.cpu().double() - dx64).abs() <= (half * dx64.abs() + tiny + CHAIN * R.U32 * size) * (1 + half)).all()
    if w is not None:
        whalf = R.half_step(wt)
        steps = n / 512 + 4 + CHAIN   # rows to a group, groups to a workgroup, workgroups to a column
        assert ((dw.cpu().double() - dw64).abs() <= (whalf * dw64.abs() + R.smallest_step(wt) + steps * R.U32 * wsize) * (1 + whalf)).all()
        again = torch.zeros_like(dx)
        ann.ann_rms_norm_backward(*args, again, again.stride(0), stream=stream(), **more)
        # (another number of rows to a workgroup, the same sums of a row)
        assert torch.equal(again.cpu(), dx.cpu())


@pytest.mark.parametrize("d", [100, 768, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_nothing_between_rows_is_written(d, dtype):
    import paper_2503_17911_amd as ann
    T = types(ann)[dtype]
    x, res, w, dy, ds = (v.cuda() for v in case(37, d, dtype, "f32", 5))
    n, wide = 37, d + 20
    apart, kept, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda")
    ann.ann_rms_norm(x, n, d, d, T, w, ann.F32, 1e-6, apart, d, residual=res, residual_stride=d, sum=kept, sum_stride=d, rstd=rstd, stream=stream())
    bufs = [torch.full((n, wide), 7.0, dtype=x.dtype, device="cuda") for _ in range(2)]
    for over_x, over_res in (("sum", "y"), ("y", "sum"), ("sum", None), (None, "sum"), ("y", None)):
        for b, v in zip(bufs, (x, res)):
            b[:, :d] = v
        out = {f: torch.full((n, wide), 7.0, dtype=x.dtype, device="cuda") for f in ("sum", "y")}
        for where, b in ((over_x, bufs[0]), (over_res, bufs[1])):
            if where:
                out[where] = b
        ann.ann_rms_norm(bufs[0], n, d, wide, T, w, ann.F32, 1e-6, out["y"], wide, residual=bufs[1], residual_stride=wide, sum=out["sum"], sum_stride=wide,
                         stream=stream())
        assert torch.equal(out["y"][:, :d], apart) and torch.equal(out["sum"][:, :d], kept)
        assert all((b[:, d:] == 7.0).all() for b in (*bufs, *out.values()))
    # no sum kept: the norm is that of the rounded sum all the same
    y = torch.empty_like(x)
    ann.ann_rms_norm(x, n, d, d, T, w, ann.F32, 1e-6, y, d, residual=res, residual_stride=d, stream=stream())
    assert torch.equal(y, apart)
    # the gradient over dy, over dsum
    args = dict(dsum_stride=d, stream=stream())
    want = torch.empty_like(x)
    ann.ann_rms_norm_backward(dy, d, kept, d, n, d, T, w, ann.F32, rstd, want, d, dsum=ds, **args)
    d1, d2 = dy.clone(), ds.clone()
    ann.ann_rms_norm_backward(d1, d, kept, d, n, d, T, w, ann.F32, rstd, d1, d, dsum=ds, **args)
    ann.ann_rms_norm_backward(dy, d, kept, d, n, d, T, w, ann.F32, rstd, d2, d, dsum=d2, **args)
    assert torch.equal(d1, want) and torch.equal(d2, want)


@pytest.mark.parametrize("group", [0, 32, 128])
def test_rows_of_zeros_tiny_rows_and_rows_that_are_not_numbers(group):
    import paper_2503_17911_amd as ann
    n, d = 6, 300
    x = torch.randn(n, d, generator=torch.Generator().manual_seed(4))
    x[1] = 0.0
    x[2] = 1e-30                    # with eps: the values stay that small
    x[3, 5] = float("nan")
    x[4] *= 1e18                    # (the squares' sum is at the end of fp32's range)
    xd = x.cuda()
    codes, rstd = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
    groups = 1 if group == 0 else -(-d // group)
    sc = torch.empty(n, groups, device="cuda")
    ann.ann_rms_norm_e4m3(xd, n, d, d, ann.F32, None, ann.F32, 1e-6, codes, d, group, sc, groups, rstd=rstd, stream=stream())
    v = E.e4m3_values()[codes.cpu().long()] * sc.cpu().double()[:, torch.arange(d) // (group or d)]
    assert (v[1] == 0).all() and torch.isfinite(sc).all() and (sc > 0).all()
    assert v[3].isnan().all() and rstd[3].isnan()
    want, _ = E.rms_norm(x, None, 1e-6)
    for row in (0, 2, 4, 5):
        # (the group's largest has the code 448: its step is 32 scales)
        assert ((v[row] - want[row]).abs() <= 2.0 ** -4 * (1 + 1e-5) * want[row].abs() + 2.0 ** -10 * sc[row].max().item()).all()
        assert (v[row].abs().max() - want[row].abs().max()).abs() <= 1e-5 * want[row].abs().max()


@pytest.mark.parametrize("d", [100, 5000, 20_000])
def test_rows_whose_squares_leave_the_range(d):
    import paper_2503_17911_amd as ann
    x = torch.randn(4, d, generator=torch.Generator().manual_seed(4))
    x[1] *= 1e25
    x[2] *= 5e37
    x[3, 7] = float("inf")
    for t, T in ((torch.float32, ann.F32), (torch.bfloat16, ann.BF16)):
        xt = x.to(t)
        y, rstd = torch.empty(4, d, dtype=t, device="cuda"), torch.empty(4, device="cuda")
        ann.ann_rms_norm(xt.cuda(), 4, d, d, T, None, T, 1e-6, y, d, rstd=rstd, stream=stream())
        want, rstd64 = E.rms_norm(xt, None, 1e-6)
        # (1 / 5e37 is below fp32's normal numbers: 2^-150 of rounding)
        assert ((rstd[:3].cpu().double() - rstd64[:3]).abs() <= CHAIN * R.U32 * rstd64[:3] + 2.0 ** -150).all()
        off = (CHAIN * R.U32 + 2.0 ** -150 / rstd64[:3, None]) * 2 + R.half_step(t)
        assert ((y[:3].cpu().double() - want[:3]).abs() <= off * want[:3].abs()).all()
        # a row with an infinite element: nothing of the others is left
        got = y[3].cpu()
        assert got[7].isnan() and (got[:7] == 0).all() and (got[8:] == 0).all() and rstd[3] == 0


def test_every_code_is_the_nearest():
    """Rows of one group whose largest value is 448 after the norm: codes as torch rounds fp32 to e4m3, ties to even."""
    import paper_2503_17911_amd as ann
    n, d = 512, 128
    g = torch.Generator().manual_seed(3)
    w = torch.cat([torch.tensor([448.0]), torch.exp2(torch.randint(-12, 9, (d - 1,), generator=g).float()) * (1 + torch.randint(0, 16, (d - 1,), generator=g) / 16)])
    w = w.clamp_max(448.0)
    x = torch.where(torch.rand(n, d, generator=g) < 0.5, -1.0, 1.0)   # h * rstd = h exactly: mean(h^2) = 1, eps = 0
    codes, sc = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, 1, device="cuda")
    ann.ann_rms_norm_e4m3(x.cuda(), n, d, d, ann.F32, w.cuda(), ann.F32, 0.0, codes, d, 128, sc, 1, stream=stream())
    assert (sc == 1.0).all()
    assert torch.equal(codes.cpu(), (x * w).to(torch.float8_e4m3fn).view(torch.uint8))


def test_same_bits_again_on_other_streams_and_in_graphs():
    import paper_2503_17911_amd as ann
    for n, d, dtype in ((300, 768, "bf16"), (37, 100, "f16"), (5, 9000, "f32")):
        T = types(ann)[dtype]
        x, res, w, dy, ds = (v.cuda() for v in case(n, d, dtype, "f32", 7))
        need = ann.ann_rms_norm_backward_workspace(n, d)

        def outputs():
            return [torch.zeros_like(x), torch.zeros_like(x), torch.zeros(n, device="cuda"), torch.zeros_like(x), torch.zeros(d, device="cuda"),
                    torch.zeros(n, d, dtype=torch.uint8, device="cuda"), torch.zeros(n, -(-d // 128), device="cuda"),
                    torch.zeros(need, dtype=torch.uint8, device="cuda")]

        def all_of(o):
            more = dict(residual=res, residual_stride=d, sum=o[0], sum_stride=d, rstd=o[2], stream=stream())
            ann.ann_rms_norm(x, n, d, d, T, w, ann.F32, 1e-6, o[1], d, **more)
            ann.ann_rms_norm_e4m3(x, n, d, d, T, w, ann.F32, 1e-6, o[5], d, 128, o[6], -(-d // 128), **more)
            ann.ann_rms_norm_backward(dy, d, o[0], d, n, d, T, w, ann.F32, o[2], o[3], d, dsum=ds, dsum_stride=d, dweight=o[4], workspace=o[7],
                                      workspace_bytes=need, stream=stream())

        want, other, graphed = outputs(), outputs(), outputs()
        all_of(want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            all_of(other)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[:7], other[:7]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            all_of(graphed)
        for _ in range(3):
            x.copy_(torch.randn(n, d, device="cuda"))
            all_of(want)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want[:7], graphed[:7]))


def test_gradient_against_differences():
    """dx and dweight against central differences of the 64-bit loss sum(dy y) + sum(dsum h) along random directions."""
    import paper_2503_17911_amd as ann
    n, d = 12, 50
    x, res, w, dy, ds = case(n, d, "f32", "f32", 9)
    y, kept, dx, dw, rstd = *(torch.empty(n, d, device="cuda") for _ in range(3)), torch.empty(d, device="cuda"), torch.empty(n, device="cuda")
    ann.ann_rms_norm(x.cuda(), n, d, d, ann.F32, w.cuda(), ann.F32, 1e-3, y, d, residual=res.cuda(), residual_stride=d, sum=kept, sum_stride=d, rstd=rstd,
                     stream=stream())
    need = ann.ann_rms_norm_backward_workspace(n, d)
    ann.ann_rms_norm_backward(dy.cuda(), d, kept, d, n, d, ann.F32, w.cuda(), ann.F32, rstd, dx, d, dsum=ds.cuda(), dsum_stride=d, dweight=dw,
                              workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need, stream=stream())

    def loss(h, w):
        return float((dy.double() * E.rms_norm(h, w, 1e-3)[0] + ds.double() * h).sum())

    h, w, step = kept.cpu().double(), w.double(), 1e-5
    g = torch.Generator().manual_seed(1)
    for _ in range(4):
        e = [torch.randn(v.shape, generator=g, dtype=E.F64) for v in (h, w)]
        slope = (loss(h + step * e[0], w + step * e[1]) - loss(h - step * e[0], w - step * e[1])) / (2 * step)
        terms = [dx.cpu().double() * e[0], dw.cpu().double() * e[1]]
        assert abs(sum(float(v.sum()) for v in terms) - slope) <= 2 * CHAIN * R.U32 * sum(float(v.abs().sum()) for v in terms) + 1e-4
