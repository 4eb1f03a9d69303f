"""Distillation over long lists captured over one workspace: G in two parts goes by the probabilities of each replay, not of the capture."""
import pytest
import torch

from test_gpu_row_distillation import dirty, teacher_lists
from test_gpu_row_logprobs import inputs, stream, types

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq, n, d", [(300, 1500, 96), (300, 3000, 200), (1200, 20_000, 136), (40, 1500, 200)])
def test_replays_with_other_contents(nq, n, d):
    import paper_2503_17911_amd as ann
    k, t = 8, types(ann)[torch.bfloat16]
    cases = []
    # soft and sharp scores: queries of a tenth of the length have no probability above 2^-10
    for seed, size in ((1, 1.0), (2, 0.1), (3, 3.0), (4, 0.0)):
        q, rows, _, _ = inputs(nq, n, d, "bf16", seed)
        q = (size * q.float()).to(q.dtype)
        ids, given = teacher_lists(q, rows, None, 10.0, k, seed)
        cases.append((q.cuda(), rows.cuda(), ids.to(torch.int32).cuda(), given.cuda()))
    q, rows, ids, given = (x.clone() for x in cases[0])
    need = max(ann.ann_row_distillation_workspace(nq, n, d, t, k), ann.ann_row_distillation_backward_workspace(nq, n, d, t, k))
    ws, g = dirty(need), torch.full((nq,), 0.5, device="cuda")
    out = [torch.empty(nq, device="cuda"), torch.empty(nq, device="cuda"), torch.empty(nq, k, device="cuda"), torch.empty_like(q), torch.empty_like(rows), torch.empty(n, device="cuda")]

    def both():
        what = dict(q=q, nq=nq, q_stride=d, rows=rows, n=n, row_stride=d, d=d, type=t, scale=10.0, k=k, given_ids=ids, given_logprobs=given, workspace=ws,
                    workspace_bytes=need, stream=stream(), lse=out[1], logprobs=out[2])
        ann.ann_row_distillation(**what, loss=out[0])
        ann.ann_row_distillation_backward(**what, g_loss=g, dq=out[3], dq_stride=d, drows=out[4], drows_stride=d, drow_bias=out[5])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for case in cases + cases:
        for to, x in zip((q, rows, ids, given), case):
            to.copy_(x)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in out]
        ws.fill_(0x3C)
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(replayed, out))
        assert all(torch.isfinite(x).all() for x in out)
