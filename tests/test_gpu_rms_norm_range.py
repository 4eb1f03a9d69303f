"""Root-mean-square norm of rows whose squares lie below fp32's range, where eps does not hide them."""
import math

import pytest
import torch

import encoder_reference as E
import head_reference as R
from test_gpu_layer_norm import types
from test_gpu_rms_norm import CHAIN, case, check, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, wtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("d", [1, 60, 129, 768, 5000, 20_001])
def test_tiny_rows_without_eps(d, dtype, wtype):
    import paper_2503_17911_amd as ann
    n = 10
    x, res, w, dy, ds = case(n, d, dtype, wtype, d)
    # ordinary rows among them; what lies lowest is a normal number still, so that sums with the residual round as ever
    size = torch.tensor([1.0, 1e-17, 1e-19, 1e-20, 1e-21, 1e-22, 1e-23, 1e-25, 1e-30, 1e3])[:, None]
    x, res = (x.float().clamp(-4, 4).sign() * x.float().abs().clamp(0.05, 4) * size).to(x.dtype), (0.25 * size * res.float().sign()).to(x.dtype)
    # (as the call gets them: 1e-43 is 71 of fp32's smallest numbers, 0.5 % less)
    for eps in torch.tensor([0.0, 1e-43, 1e-40]).double().tolist():
        check(ann, x, None, w, dy, ds, 0, 0, eps)
        check(ann, x, res, w, dy, None, 1, 1, eps)


@pytest.mark.parametrize("d", [60, 5000, 20_001])
def test_rows_below_the_normal_numbers(d):
    """1 / rms leaves fp32's range below 2^-128: rstd is +infinity there, y is right all the same."""
    import paper_2503_17911_amd as ann
    for dtype in ("f32", "bf16"):
        t, T = R.DTYPES[dtype], types(ann)[dtype]
        x = torch.randint(-3, 4, (5, d), generator=torch.Generator().manual_seed(d)).double()
        x[:, 0] = 2.0
        # (whole multiples of the type's smallest numbers, 2^-149 and 2^-133)
        x = (x * torch.tensor([2.0 ** -120, 2.0 ** -126, 2.0 ** -131, 2.0 ** -133, 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149], dtype=E.F64)[:, None]).to(t)
        y, rstd = torch.empty(5, d, dtype=t, device="cuda"), torch.empty(5, device="cuda")
        ann.ann_rms_norm(x.cuda(), 5, d, d, T, None, T, 0.0, y, d, rstd=rstd, stream=stream())
        want, rstd64 = E.rms_norm(x, None, 0.0)
        assert ((y.cpu().double() - want).abs() <= ((CHAIN + 4) * R.U32 + R.half_step(t)) * want.abs()).all()
        held = rstd64 <= torch.finfo(torch.float32).max
        assert held[0] and not held[4]
        assert ((rstd.cpu().double() / rstd64 - 1).abs() <= CHAIN * R.U32)[held].all() and (rstd.cpu()[~held] == math.inf).all()
        # the values in 8 bits
        for group in (0, 64):
            groups = 1 if group == 0 else -(-d // group)
            codes, sc = torch.empty(5, d, dtype=torch.uint8, device="cuda"), torch.empty(5, groups, device="cuda")
            ann.ann_rms_norm_e4m3(x.cuda(), 5, d, d, T, None, T, 0.0, codes, d, group, sc, groups, stream=stream())
            v = E.e4m3_values()[codes.cpu().long()] * sc.cpu().double()[:, torch.arange(d) // (group or d)]
            off = 2.0 ** -10 * sc.cpu().double()[:, torch.arange(d) // (group or d)]
            assert ((v - want).abs() <= (2.0 ** -4 + 4 * CHAIN * R.U32) * want.abs() + off).all()


def test_rows_of_zeros():
    import paper_2503_17911_amd as ann
    for dtype, d in (("f32", 100), ("f16", 100), ("bf16", 20_000)):
        t, T = R.DTYPES[dtype], types(ann)[dtype]
        x = torch.zeros(2, d, dtype=t, device="cuda")
        y, rstd = torch.full_like(x, 7.0), torch.empty(2, device="cuda")
        ann.ann_rms_norm(x, 2, d, d, T, None, T, 1e-6, y, d, rstd=rstd, stream=stream())
        assert (y == 0).all() and ((rstd - 1e3).abs() <= 1e3 * 4 * R.U32).all()
        # without eps there is no norm: 0 / 0
        ann.ann_rms_norm(x, 2, d, d, T, None, T, 0.0, y, d, rstd=rstd, stream=stream())
        assert y.isnan().all() and (rstd == math.inf).all()
