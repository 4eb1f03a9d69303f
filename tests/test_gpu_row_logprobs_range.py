"""Scores below fp32's range: such rows have no probability."""
import math

import pytest
import torch

import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(5, 300, 16), (70, 300, 16), (70, 300, 160), (1100, 15_002, 192)])
def test_scores_of_minus_infinity(nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    scale, k = 2.0 ** 100, 5
    q, rows, target = torch.zeros(nq, d), torch.zeros(n, d), torch.full((nq,), 7)
    q[:, 0], rows[::2, 0] = 2.0 ** 15, -2.0 ** 15     # even rows: -2^130; the others: 0, like each other
    q, rows = q.to(L.R.DTYPES[dtype]), rows.to(L.R.DTYPES[dtype])
    want = math.log(n // 2)
    near = 64 * L.R.U32 * (1 + want)      # sums of 16 and what follows, three roundings of numbers of that size
    for b in (None, torch.zeros(n)):
        got = L.forward(ann, q, rows, b, target, scale, k)
        assert ((got["lse"] - want).abs() <= near).all() and ((got["logprob"] + want).abs() <= near).all()
        assert (got["alt_ids"] == 2 * torch.arange(k) + 1).all()
        if b is None:
            assert got["entropy"].isnan().all()
        else:
            assert ((got["entropy"] - want).abs() <= 2 * near).all()
        g, h, entropy = torch.full((nq,), -0.5), torch.full((nq,), 0.25), torch.full((nq,), want)
        one = L.backward(ann, q, rows, b, target, scale, got["lse"], entropy, g, h, drows=False)
        assert (one["dq"] == 0).all()     # (rows with probability hold zeros)
        sums = torch.full((n,), 0.5 * nq / (n // 2), dtype=L.R.F64)
        sums[::2], sums[7] = 0.0, 0.5 * nq / (n // 2) - 0.5 * nq
        # the entropy's part is p times what lse and entropy are off (each by `near`); p by as much
        assert ((one["drow_bias"].double() - sums).abs() <= (2 * 0.25 + 2 * 0.5) * near * nq / (n // 2) + 2 * near * sums.abs()).all()
