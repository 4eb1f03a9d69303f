"""Gradients beside queries that take no part with their weights, and beside
weights that are not finite: the other queries' are what they are without them."""
import math

import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


def problem(nq, d, dtype):
    """Weights of a scaled loss.  Queries 1 and 2 have no given row, query 7 (by its lse) no row at all."""
    n, scale = 900, 10.0
    q, rows, _, target = L.inputs(nq, n, d, dtype, 3)
    gen = torch.Generator().manual_seed(nq + d)
    g, h = -256.0 * (0.5 + torch.rand(nq, generator=gen)), 25.0 * torch.randn(nq, generator=gen)
    g[[1, 2, 7]], h[7] = 0.0, 0.0
    lse, _, entropy = (v.float() for v in R.log_probabilities(R.scores(q, rows, scale, None), target))
    lse[7] = -math.inf
    return (q, rows, None, target, scale, lse, entropy), g, h


SHAPES = [(50, 40), (300, 40), (50, 200), (300, 200)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, d", SHAPES)
@pytest.mark.parametrize("value", [1e6, 1e30, math.inf, math.nan])
def test_queries_that_take_no_part(value, nq, d, dtype):
    import paper_2503_17911_amd as ann
    args, g, h = problem(nq, d, dtype)
    want = L.backward(ann, *args, g, h)
    g[[1, 2, 7]], h[7] = value, value
    got = L.backward(ann, *args, g, h)
    for name in want:
        assert torch.isfinite(want[name]).all() and torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, d", SHAPES)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_weights_that_are_not_finite(value, nq, d, dtype):
    import paper_2503_17911_amd as ann
    args, g, h = problem(nq, d, dtype)
    others = torch.arange(nq) != 9
    g[9], h[9] = 0.0, 0.0
    want = L.backward(ann, *args, g, h)["dq"]
    for which in (g, h):
        which[9] = value
        got = L.backward(ann, *args, g, h)["dq"]
        assert torch.isfinite(want[others]).all() and torch.equal(got[others], want[others])
        which[9] = 0.0


@pytest.mark.parametrize("d", [40, 200])
def test_weights_near_the_end_of_fp32(d):
    """Half precision: the largest weights that there are, brought down by the scale of the scores."""
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(50, 900, d, "f16", 3)
    scale = 2.0 ** -100
    lse, _, entropy = (v.float() for v in R.log_probabilities(R.scores(q, rows, scale, None), target))
    g = -1.0 - torch.rand(50, generator=torch.Generator().manual_seed(1))
    want = L.backward(ann, q, rows, None, target, scale, lse, entropy, g * 2.0 ** 90, None, dbias=False)
    got = L.backward(ann, q, rows, None, target, scale, lse, entropy, g * 2.0 ** 110, None, dbias=False)
    for name in want:   # (a power of two apart, up to what fp16 keeps of its smallest values)
        a, b = want[name].double() * 2.0 ** 20, got[name].double()
        assert (a != 0).any() and ((a - b).abs() <= R.half_step(torch.float16) * 2 * b.abs() + 2.0 ** -25 * 2.0 ** 20).all()
