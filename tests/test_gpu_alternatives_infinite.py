"""Rows whose score is infinite are the first alternatives; rows whose score is
not a number are none."""
import math

import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu
SHAPES = [(5, 3000, 40), (70, 3000, 40), (70, 3000, 200), (1100, 15_001, 192)]


def wanted(q, rows, b, k):
    z = R.scores(q, rows, 20.0, b)
    ids, _ = R.alternatives(torch.where(z.isnan(), torch.full_like(z, -math.inf), z), k)
    return ids


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", SHAPES)
@pytest.mark.parametrize("k", [1, 10])
def test_biases_of_infinity(k, nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    q, rows, b, target = L.inputs(nq, n, d, dtype, 6, "holes")
    for at in ([5], [n - 2], [39, 17, 1031]):
        some = b.clone()
        some[at] = math.inf
        got = L.forward(ann, q, rows, some, target, 20.0, k)
        assert torch.equal(got["alt_ids"].long(), wanted(q, rows, some, k)), at


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", SHAPES)
def test_rows_of_infinity_beside_rows_that_are_not_numbers(nq, n, d, dtype):
    """A group of 16 rows whose first holds NaN and whose others are infinite."""
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(nq, n, d, dtype, 6)
    q = q.abs() + 0.01
    group = torch.tensor([r + 64 for r in range(32) if r // 4 % 2 == 0])
    rows[group] = math.inf
    rows[group[0]] = math.nan
    got = L.forward(ann, q, rows, None, target, 20.0, 20)
    assert torch.equal(got["alt_ids"].long(), wanted(q, rows, None, 20))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bias", ["none", "plain", "holes"])
@pytest.mark.parametrize("nq, n, d", SHAPES)
def test_rows_that_are_not_numbers(nq, n, d, bias, dtype):
    """They are no alternatives, and hide none: among them the likeliest rows, the last row and a whole group."""
    import paper_2503_17911_amd as ann
    q, rows, b, target = L.inputs(nq, n, d, dtype, 6, bias)
    rows[target[3:].clamp(0, n - 1)[:4]] = math.nan
    rows[128:160], rows[n - 1] = math.nan, math.nan
    got = L.forward(ann, q, rows, b, target, 20.0, 10)
    assert torch.equal(got["alt_ids"].long(), wanted(q, rows, b, 10))
    assert got["lse"].isnan().all()
