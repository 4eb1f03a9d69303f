"""The entropy where a few rows stand far above all others."""
import math

import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("nq, n, d", [(3, 6016, 16), (70, 6016, 16), (600, 6016, 128), (70, 6016, 160), (1100, 15_040, 192)])
def test_few_rows_far_above_the_others(nq, n, d, bias, dtype):
    """Every other block of 32 rows holds two with a score of 18; all others' is 0, and each lane sees some of these before.  Beside one of the
    large terms the small ones are less than half a step: their share of the entropy (18 times their probability) must not go with them."""
    import paper_2503_17911_amd as ann
    q, rows = torch.zeros(nq, d), torch.zeros(n, d)
    q[:, 0] = 1.0
    rows[32::64, 0], rows[36::64, 0] = 18.0, 18.0
    t = R.DTYPES[dtype]
    got = L.forward(ann, q.to(t), rows.to(t), torch.zeros(n) if bias else None, torch.full((nq,), 32), 1.0, 0)
    lse, lp, entropy = R.log_probabilities(R.scores(q, rows, 1.0, None), torch.full((nq,), 32))
    # 15 additions to a term of one, each off by half a step; two exponentials; what joins the lanes; the result
    err = (15 + 8) * R.U32
    assert ((got["lse"].double() - lse).abs() <= err + R.U32 * lse).all()
    assert ((got["logprob"].double() - lp).abs() <= err + R.U32 * lp.abs()).all()
    assert ((got["entropy"].double() - entropy).abs() <= err + R.U32 * entropy).all()
