"""Gradients where rows are masked with finite biases: such rows have no
probability, so everything is as if they were left out, whatever the weights."""
import math

import pytest
import torch

import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("mask, weight", [(LOWEST, 0.5), (LOWEST, 2.0), (LOWEST, -1000.0), (-2e38, 2.0), (-1e36, 4096.0)])
@pytest.mark.parametrize("nq, d", [(30, 40), (300, 40), (30, 200), (300, 200)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masked_rows_are_as_if_left_out(dtype, nq, d, mask, weight):
    import paper_2503_17911_amd as ann
    n, scale = 700, 10.0
    q, rows, _, target = L.inputs(nq, n, d, dtype, 2)
    target = target | 1     # (odd rows are kept)
    gen = torch.Generator().manual_seed(nq + d)
    g, h = -0.5 - torch.rand(nq, generator=gen), weight * (0.5 + 0.5 * torch.rand(nq, generator=gen))
    b = torch.zeros(n)
    b[::2] = mask
    left_out = torch.where(b == mask, torch.tensor(-math.inf), b)
    f = L.forward(ann, q, rows, b, target, scale, 0)
    same = L.forward(ann, q, rows, left_out, target, scale, 0)
    for name in f:
        assert torch.equal(f[name], same[name]), name
    for weights in ((g, h), (None, h)):
        want = L.backward(ann, q, rows, left_out, target, scale, f["lse"], f["entropy"], *weights)
        got = L.backward(ann, q, rows, b, target, scale, f["lse"], f["entropy"], *weights)
        for name in want:
            assert torch.isfinite(want[name]).all() and (want[name] != 0).any()
            assert torch.equal(got[name], want[name]), name
