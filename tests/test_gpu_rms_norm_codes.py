"""e4m3 codes of the root-mean-square norm for scales that are no power of two: v / scale is a division, and what lies halfway between two codes goes to the even one."""
import pytest
import torch

import encoder_reference as E
import head_reference as R
from test_gpu_layer_norm import types
from test_gpu_rms_norm import stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [128, 256, 2048, 16_512])   # (16,512: longer than a workgroup's registers in any type)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_values_halfway_between_codes(d, dtype, group):
    import paper_2503_17911_amd as ann
    values = E.e4m3_values()[:127]                       # 0 .. 448
    halfway = (values[1:] + values[:-1]) / 2             # five bits each at most
    g = torch.Generator().manual_seed(d + group)
    for scale in (1.0, 3.0, 7.0, 49.0, 127.0, 199.0, 7.0 / 512, 113.0 * 2 ** 20):
        # exact in fp32: eight bits times five.  The group's largest gives the scale: 448 times it, over 448
        v = halfway[torch.randint(len(halfway), (d,), generator=g)]
        v[::(group or d)] = 448.0
        w = (v * scale).float()
        assert torch.equal(w.double(), v * scale)
        x = torch.where(torch.rand(3, d, generator=g) < 0.5, -1.0, 1.0)   # h * rstd = h exactly: mean(h^2) = 1, eps = 0
        groups = 1 if group == 0 else d // group
        codes, sc = torch.empty(3, d, dtype=torch.uint8, device="cuda"), torch.empty(3, groups, device="cuda")
        ann.ann_rms_norm_e4m3(x.to(R.DTYPES[dtype]).cuda(), 3, d, d, types(ann)[dtype], w.cuda(), ann.F32, 0.0, codes, d, group, sc, groups, stream=stream())
        assert (sc == scale).all()
        want = (x * w / scale).to(torch.float8_e4m3fn)
        assert torch.equal(want.double().abs(), (x * v).float().to(torch.float8_e4m3fn).double().abs())   # (the quotients are exact)
        assert torch.equal(codes.cpu(), want.view(torch.uint8)), scale


@pytest.mark.parametrize("group", [0, 64])
def test_any_scale(group):
    """Values of all kinds: the code is that of fp32's quotient."""
    import paper_2503_17911_amd as ann
    n, d = 200, 384
    g = torch.Generator().manual_seed(group)
    w = torch.exp2(14 * torch.rand(d, generator=g) - 8) * (1 + torch.rand(d, generator=g))
    x = torch.where(torch.rand(n, d, generator=g) < 0.5, -1.0, 1.0)
    groups = 1 if group == 0 else d // group
    codes, sc = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(n, groups, device="cuda")
    ann.ann_rms_norm_e4m3(x.cuda(), n, d, d, ann.F32, w.cuda(), ann.F32, 0.0, codes, d, group, sc, groups, stream=stream())
    at = torch.arange(d) // (group or d)
    assert torch.equal(sc.cpu(), torch.stack([p.abs().amax(1) / 448 for p in torch.split(x * w, group or d, dim=1)], 1))
    assert torch.equal(codes.cpu(), (x * w / sc.cpu()[:, at]).to(torch.float8_e4m3fn).view(torch.uint8))
