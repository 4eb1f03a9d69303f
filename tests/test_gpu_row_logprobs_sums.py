"""What the sums of the log probabilities may lose, where the scores themselves are exact."""
import math

import numpy as np
import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


def scale_near(value):
    """A scale whose product with log2 e is rounded by next to nothing, and how much that is."""
    for step in range(10_000):
        scale = np.float32(value + step * 2.0 ** -18)
        c = scale * np.float32(math.log2(math.e))
        off = abs(float(c) / (float(scale) * math.log2(math.e)) - 1)
        if off < 1e-9:
            return float(scale), off
    raise AssertionError


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(3, 3000, 16), (70, 3000, 16), (70, 3000, 160), (1100, 15_001, 192), (600, 9001, 128)])
def test_large_scores(nq, n, d, dtype):
    """Scores of some 4,000 and more whose products are whole numbers: nothing of their size may go to the log probabilities, which are small."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + n)
    q, rows = torch.zeros(nq, d), torch.zeros(n, d)
    rows[:, 0], rows[:, 1:16] = 64.0, torch.randint(2, (n, 15), generator=gen).float()
    q[:, 0], q[:, 1:16] = 64.0 + torch.arange(nq) % 16, 1.0
    scale, off = scale_near(1.0)
    target = torch.randint(n, (nq,), generator=gen)
    t = R.DTYPES[dtype]
    got = L.forward(ann, q.to(t), rows.to(t), None, target, scale, 0)
    z = R.scores(q, rows, scale, None)
    _, lp, entropy = R.log_probabilities(z, target)
    assert z.min() > 4000 and z.max() < 5200
    # an exponent (at most 15 * 1.45 + 29 in size) is rounded once; an exponential is off by two steps at most; sums of 16
    # and what follows; the scale's rounding
    err = (51 * math.log(2) + 4 + 24) * R.U32 + 5200 * off
    assert ((got["logprob"].double() - lp).abs() <= err + R.U32 * lp.abs()).all()
    assert ((got["entropy"].double() - entropy).abs() <= (2 * entropy + 1) * 2 * err + R.U32 * entropy).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.7, 1.3])
@pytest.mark.parametrize("nq, n, d", [(3, 3001, 16), (70, 3001, 16), (70, 3001, 160), (1100, 15_001, 192)])
def test_large_scores_at_a_scale_that_is_rounded(nq, n, d, scale, dtype):
    """Likewise where scale log2 e is not an fp32 number."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + n)
    q, rows = torch.zeros(nq, d), torch.zeros(n, d)
    rows[:, 0], rows[:, 1:16] = 64.0, torch.randint(2, (n, 15), generator=gen).float()
    q[:, 0], q[:, 1:16] = 64.0 + torch.arange(nq) % 16, 1.0
    scale = float(np.float32(scale))
    target = torch.randint(n, (nq,), generator=gen)
    t = R.DTYPES[dtype]
    got = L.forward(ann, q.to(t), rows.to(t), None, target, scale, 0)
    _, lp, entropy = R.log_probabilities(R.scores(q, rows, scale, None), target)
    # as above; the scale's rounding counts by its square, and for the entropy by the scores' variance (at most (15 * 1.3 / 2)^2)
    err = (15 * 1.3 * 1.45 + 29) * math.log(2) * R.U32 + (4 + 24) * R.U32
    assert ((got["logprob"].double() - lp).abs() <= err + R.U32 * lp.abs()).all()
    assert ((got["entropy"].double() - entropy).abs() <= (2 * entropy + 1) * 2 * err + R.U32 * entropy + 4 * 96 * R.U32).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(1, 1, 1), (5, 1, 1), (33, 1, 3), (70, 1, 1), (70, 1, 4)])
def test_one_row_and_few_columns(nq, n, d, dtype):
    """lse is the only score: fp32 elements keep all their bits."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + d)
    t = R.DTYPES[dtype]
    q, rows = torch.randn(nq, d, generator=gen).to(t), torch.randn(n, d, generator=gen).to(t)
    got = L.forward(ann, q, rows, None, None, 1.0, 0)
    want = (q.double() @ rows.double().T)[:, 0]
    # six products of parts (or one) to an element, each rounding the sum by 2^-23 of the terms at most; parts left out; three roundings;
    # and an exponential near one that is off by two steps
    terms = (q.double().abs() @ rows.double().abs().T)[:, 0]
    steps = 6 * d + 1 if dtype == "f32" else d
    assert ((got["lse"].double() - want).abs() <= (2 * steps + 3) * R.U32 * terms + 4 * R.U32).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [8, 200])
def test_gradients_keep_the_bits_of_their_factors(d, dtype):
    """Two rows, one query.  Queries of zeros: both probabilities are 1/2, dq = scale g (x_t - x_o) / 2; rows of zeros: drows = +-scale g q / 2."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(d)
    t, scale, g = R.DTYPES[dtype], 3.0, torch.tensor([-1.7])
    rows, target = torch.randn(2, d, generator=gen).to(t), torch.tensor([1])
    lse, entropy = torch.full((1,), math.log(2)), torch.full((1,), math.log(2))
    # G is g / 2: its probability's three roundings, its own to 16 bits (fp32: what three parts leave), six products of two terms; the result
    kept = 2.0 ** -23 if dtype == "f32" else R.half_step(t)
    off = kept + (8 + 2 * 6 * 2 + 4) * R.U32
    got = L.backward(ann, torch.zeros(1, d).to(t), rows, None, target, scale, lse, entropy, g, None)
    x, half = rows.double(), R.half_step(t)
    size = scale * 0.85 * (x[0].abs() + x[1].abs())
    want = -scale * 0.85 * (x[1] - x[0])
    assert ((got["dq"][0].double() - want).abs() <= half * want.abs() + R.smallest_step(t) + off * size).all()
    q = torch.randn(1, d, generator=gen).to(t)
    got = L.backward(ann, q, torch.zeros(2, d).to(t), None, target, scale, lse, entropy, g, None)
    want = torch.stack([q[0], -q[0]]).double() * scale * 0.85
    assert ((got["drows"].double() - want).abs() <= (half + off) * want.abs() + R.smallest_step(t)).all()
