"""Alternatives among scores that are all alike or below fp32's normal numbers,
at sizes that reach every kernel which bounds them."""
import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu
SHAPES = [(5, 3000, 40, 20), (70, 3000, 40, 20), (70, 3000, 200, 20), (600, 4100, 16, 1), (1100, 15_001, 192, 10)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHAPES)
def test_a_scale_of_zero(nq, n, d, k, dtype):
    """All scores are the bias: equal ones in the order of their numbers."""
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(nq, n, d, dtype, 4)
    first = torch.arange(k).expand(nq, k)
    for bias in (None, torch.zeros(n)):
        got = L.forward(ann, q, rows, bias, target, 0.0, k)
        assert torch.equal(got["alt_ids"].long(), first)
    bias[::3] = 1.0
    got = L.forward(ann, q, rows, bias, target, 0.0, k)
    assert torch.equal(got["alt_ids"].long(), 3 * first)


@pytest.mark.parametrize("scale", [2.0 ** -130, -2.0 ** -130, 2.0 ** -140])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", SHAPES)
def test_scores_below_the_normal_numbers(nq, n, d, k, dtype, scale):
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(nq, n, d, dtype, 4)
    got = L.forward(ann, q, rows, None, target, scale, k)
    ids, _ = R.alternatives(R.scores(q, rows, scale, None), k)
    assert torch.equal(got["alt_ids"].long(), ids)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -130, 2.0 ** -30])
@pytest.mark.parametrize("nq, n, d", [(5, 3000, 40), (5, 31, 16), (70, 3000, 40), (70, 3001, 200), (70, 20, 200), (1100, 15_001, 192)])
def test_statistics_of_small_scales(nq, n, d, scale, dtype):
    import paper_2503_17911_amd as ann
    for bias in ("none", "holes"):
        q, rows, b, target = L.inputs(nq, n, d, dtype, 4, bias)
        L.check_forward(ann, q, rows, b, target, scale, 0)
