"""Given rows whose weight, exp of the teacher's log probability, is zero in 64 bits do not count, also where the student leaves them out."""
import math

import pytest
import torch

from test_gpu_row_distillation import check_forward, forward, teacher_lists
from test_gpu_row_logprobs import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n", [(40, 900), (40, 1500), (5, 200)])   # (900 and 200: a short list)
def test_rows_left_out_that_the_teacher_gives_nothing(nq, n, dtype):
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(nq, n, 64, dtype, 5, "holes")
    ids, given = teacher_lists(q, rows, b, 20.0, 6, 1)
    out = torch.nonzero(b == -math.inf)[:, 0]
    plain = forward(ann, q, rows, b, ids, given, 20.0)
    ids, given = ids.clone(), given.clone()
    # teachers that mask a row by a low number, by the lowest, by what exp just has no number for; entry 2 of a list of six
    for i, low in ((0, -1e4), (1, torch.finfo(torch.float32).min), (3, -746.0), (4, -1000.0)):
        ids[i, 2], given[i, 2] = out[i], low
    got = check_forward(ann, q, rows, b, ids, given, 20.0)
    assert torch.isfinite(got["loss"]).all()
    assert (got["logprobs"][[0, 1, 3, 4], 2] == -math.inf).all()
    assert torch.equal(got["loss"][5:], plain["loss"][5:])
    # a weight that is a number, however small, counts
    given[4, 2] = -700.0
    got = check_forward(ann, q, rows, b, ids, given, 20.0)
    assert got["loss"][4] == math.inf and torch.isfinite(got["loss"][:4]).all()


@pytest.mark.parametrize("n", [900, 1500])
def test_a_teacher_that_is_not_a_number_is_not_hidden(n):
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(40, n, 64, "f32", 5)
    ids, given = teacher_lists(q, rows, b, 20.0, 6, 1)
    given[5, 2] = math.nan
    got = forward(ann, q, rows, b, ids, given, 20.0)
    assert got["loss"][5].isnan() and torch.isfinite(got["loss"][:5]).all() and torch.isfinite(got["loss"][6:]).all()
