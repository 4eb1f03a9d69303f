"""Workspaces and outputs of exactly the bytes that are asked for: nothing behind them is written, and what they held before does not matter."""
import pytest
import torch

import head_reference as R
from test_gpu_embedding import on_gpu, tokens
from test_gpu_row_distillation import teacher_lists
from test_gpu_row_logprobs import inputs, stream, types

pytestmark = pytest.mark.gpu
GUARD = 8192


class Guarded:
    """`need` bytes of a workspace with a pattern behind them."""

    def __init__(self, need, fill):
        self.need = need
        self.all = torch.full((need + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        self.all[:need] = fill

    def intact(self):
        return bool((self.all[self.need:] == 0xA5).all())


def guarded_output(rows, d, dtype):
    """A contiguous output with a pattern behind its last row."""
    buf = torch.full((rows * d + GUARD,), 7.0, dtype=dtype, device="cuda")
    return buf[:rows * d].view(rows, d), buf[rows * d:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, rows, d", [(1, 1, 1), (7, 3, 5), (5000, 70, 33), (12_289, 3001, 20), (40_000, 1 << 15, 12), (20_000, 1000, 100), (270_000, 50_001, 8)])
def test_embedding_backward(n, rows, d, dtype):
    import paper_2503_17911_amd as ann
    t = R.DTYPES[dtype]
    ids, dy = on_gpu(tokens(n, rows, "zipf", n)), torch.randn(n, d, device="cuda").to(t)
    need, got = ann.ann_embedding_backward_workspace(n, rows, d), []
    for fill in (0x00, 0xFF, 0x3C):
        ws, (out, behind) = Guarded(need, fill), guarded_output(rows, d, t)
        ann.ann_embedding_backward(dy, d, types(ann)[t], ids, n, 1.0, rows, d, out, d, types(ann)[t], workspace=ws.all, workspace_bytes=need, stream=stream())
        assert ws.intact() and (behind == 7.0).all()
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n, d", [(1, 1), (5, 33), (100, 768), (37, 1030), (3, 20_000)])
def test_rms_norm(n, d, dtype):
    import paper_2503_17911_amd as ann
    t = R.DTYPES[dtype]
    T = types(ann)[t]
    x, dy = (torch.randn(n, d, device="cuda").to(t) for _ in range(2))
    w, rstd = torch.rand(d, device="cuda") + 0.5, torch.empty(n, device="cuda")
    y, behind = guarded_output(n, d, t)
    s, s_behind = guarded_output(n, d, t)
    ann.ann_rms_norm(x, n, d, d, T, w, ann.F32, 1e-6, y, d, residual=dy, residual_stride=d, sum=s, sum_stride=d, rstd=rstd, stream=stream())
    assert (behind == 7.0).all() and (s_behind == 7.0).all()
    for group in (0, 32, 128):
        groups = -(-d // group) if group else 1
        codes = torch.full((n * d + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        scales, sc_behind = guarded_output(n, groups, torch.float32)
        ann.ann_rms_norm_e4m3(x, n, d, d, T, w, ann.F32, 1e-6, codes, d, group, scales, groups, rstd=rstd, stream=stream())
        assert (codes[n * d:] == 0xA5).all() and (sc_behind == 7.0).all()
    need, got = ann.ann_rms_norm_backward_workspace(n, d), []
    for fill in (0x00, 0xFF):
        ws, (dx, dx_behind), (dw, dw_behind) = Guarded(need, fill), guarded_output(n, d, t), guarded_output(1, d, torch.float32)
        ann.ann_rms_norm_backward(dy, d, s, d, n, d, T, w, ann.F32, rstd, dx, d, dweight=dw, workspace=ws.all, workspace_bytes=need, stream=stream())
        assert ws.intact() and (dx_behind == 7.0).all() and (dw_behind == 7.0).all()
        got += [dx, dw]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nq, n, d, k", [(1, 1, 1, 1), (3, 50, 7, 64), (130, 257, 96, 20), (300, 4100, 200, 10), (600, 300, 130, 33), (500, 5000, 64, 40), (260, 1029, 300, 64)])
def test_row_distillation(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    q, rows, b, _ = inputs(nq, n, d, dtype, 5, "plain")
    ids, given = teacher_lists(q, rows, b, 9.0, k, 3)
    T = types(ann)[q.dtype]
    q, rows = q.cuda(), rows.cuda()
    table = dict(q=q, nq=nq, q_stride=d, rows=rows, n=n, row_stride=d, d=d, type=T, scale=9.0, row_bias=b.cuda(), k=k, given_ids=on_gpu(ids),
                 given_logprobs=given.cuda(), stream=stream())
    need, needb, got = ann.ann_row_distillation_workspace(nq, n, d, T, k), ann.ann_row_distillation_backward_workspace(nq, n, d, T, k), []
    for fill in (0x00, 0xFF, 0x3C):
        ws, wsb = Guarded(need, fill), Guarded(needb, fill)
        outs = [guarded_output(*shape) for shape in ((1, nq, torch.float32), (1, nq, torch.float32), (nq, k, torch.float32), (nq, d, q.dtype), (n, d, q.dtype),
                                                     (1, n, torch.float32))]
        loss, lse, logprobs, dq, drows, db = (o for o, _ in outs)
        ann.ann_row_distillation(**table, loss=loss, lse=lse, logprobs=logprobs, workspace=ws.all, workspace_bytes=need)
        ann.ann_row_distillation_backward(**table, lse=lse, logprobs=logprobs, g_loss=torch.ones(nq, device="cuda"), dq=dq, dq_stride=d, drows=drows, drows_stride=d,
                                          drow_bias=db, workspace=wsb.all, workspace_bytes=needb)
        assert ws.intact() and wsb.intact() and all((behind == 7.0).all() for _, behind in outs)
        got.append([o for o, _ in outs])
    for other in got[1:]:
        assert all(torch.equal(a, c) for a, c in zip(got[0], other))
