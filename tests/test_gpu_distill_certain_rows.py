"""Log probabilities of given rows are not above zero, also of a row that has all probability but for what lse is off."""
import pytest
import torch

import head_reference as R
from test_gpu_row_distillation import check_forward
from test_gpu_row_logprobs import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(300, 1, 64), (300, 200, 96), (300, 1500, 100), (7, 5000, 64), (300, 3000, 200)])
def test_certain_rows(nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    q, rows, _, target = inputs(nq, n, d, dtype, n)
    rows = rows.float()
    rows[:, -1] = 0.0
    q = (4 * rows[target.clamp(0, n - 1)]).to(R.DTYPES[dtype])
    # a row of its own for every query: others are far
    keep = target.clamp(0, n - 1).unique()
    far = torch.ones(n, dtype=torch.bool)
    far[keep[:1]] = False
    rows[far] = -rows[keep[0]] * 0.5
    q[:] = (rows[keep[0]] * (3 + torch.arange(nq) / 64.0)[:, None]).to(q.dtype)
    rows = rows.to(q.dtype)
    ids, given = keep[:1].expand(nq).clone()[:, None], torch.full((nq, 1), -0.01)
    got = check_forward(ann, q, rows, None, ids, given, 30.0)
    assert (got["logprobs"] <= 0).all()
    assert (got["loss"] >= (given.double().exp() * given.double())[:, 0].float()).all()
