"""The gradient of the rows' biases over many queries."""
import math

import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, d", [("bf16", 16), ("f16", 64), ("bf16", 136), ("f32", 16)])
def test_a_million_like_queries(d, dtype):
    """Every query adds the same to a row: what each addition loses has one sign."""
    import paper_2503_17911_amd as ann
    nq, n = 1_000_003, 48
    t = R.DTYPES[dtype]
    q, rows = torch.zeros(nq, d, dtype=t, device="cuda"), torch.ones(n, d, dtype=t, device="cuda")
    lse, g = torch.full((nq,), math.log(n), device="cuda"), torch.full((nq,), -0.7, device="cuda")
    target = torch.full((nq,), 5, dtype=torch.int32, device="cuda")
    dbias = torch.full((n,), 7.0, device="cuda")
    ty = L.types(ann)[t]
    need = ann.ann_row_logprobs_backward_workspace(nq, n, d, ty)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ann.ann_row_logprobs_backward(q, nq, d, rows, n, d, d, ty, lse=lse, scale=1.0, targets=target, g_logprob=g, drow_bias=dbias, workspace=ws,
                                  workspace_bytes=need, stream=L.stream())
    torch.cuda.synchronize()
    want = torch.full((n,), 0.7 / n, dtype=R.F64)
    want[5] -= 0.7
    want *= nq
    # an element: lse and the exponent (each off by half a step of some 6), the exponential, two products; sums of up to 64 of them, and a
    # last one; what is carried from sum to sum leaves less than a step
    element = 2 * 6 * R.U32 + 6 * R.U32
    assert ((dbias.cpu().double() / want - 1).abs() <= element + (64 + 4) * R.U32).all()
