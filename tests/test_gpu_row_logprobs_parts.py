"""Few fp32 queries: how far the product of three parts may lie from the scores."""
import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq, d", [(1, 960), (8, 960), (16, 1024), (20, 512), (32, 100)])
def test_scores_of_one_row(nq, d):
    """lse is the only score.  All products are of one sign and size, so that what the additions lose adds up."""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(d)
    q, rows = 1 + torch.rand(nq, d, generator=gen), 1 + torch.rand(1, d, generator=gen)
    got = L.forward(ann, q, rows, None, None, 1.0, 0)
    want = (q.double() @ rows.double().T)[:, 0]
    # one addition to 32 columns, off by a step of the sum so far at most, whose mean is half of the last one (and as much again for the order inside
    # the instruction); the smaller products' by 2^-8 of that; parts left out; the last roundings
    steps = (d + 31) // 32
    err = (steps / 2 * 2 * 2 * (1 + 5 / 256) + 2 + 4) * R.U32
    assert ((got["lse"].double() - want).abs() <= err * want).all()


@pytest.mark.parametrize("d", [512, 960, 1024])
def test_scores_round_as_often_as_those_of_16_bits(d):
    """Whatever the matrix instruction loses, three parts lose it once: the errors of 40 tables of one row spread like those of 16-bit
    elements of the same sizes.  (Six products into one sum: sqrt(6) times as far.)"""
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(d)
    spread = {}
    for dtype in ("f32", "bf16"):
        off = []
        for _ in range(40):
            q, rows = (1 + torch.rand(n, d, generator=gen).to(R.DTYPES[dtype]) for n in (16, 1))
            want = (q.double() @ rows.double().T)[:, 0]
            off.append(L.forward(ann, q, rows, None, None, 1.0, 0)["lse"].double() / want - 1)
        spread[dtype] = float(torch.cat(off).square().mean().sqrt())
    # (640 samples each: 3 % off at one standard deviation; the smaller products add 2 % of a rounding)
    assert spread["f32"] <= 1.5 * spread["bf16"]
