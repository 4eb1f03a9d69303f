"""Arguments that token embeddings and the root-mean-square norm refuse on the host, and the sizes of their workspaces (no GPU)."""
import math

import pytest

import paper_2503_17911_amd as ann
from test_head_arguments import refused

EMBED = dict(table=16, rows=4, dim=8, table_stride=8, table_type=ann.BF16, ids=16, n=2, scale=1.0, y=16, y_stride=8, type=ann.BF16)


@pytest.mark.parametrize("change, status, words", [
    (dict(table=None), ann.EINVAL, "NULL"), (dict(ids=None), ann.EINVAL, "NULL"), (dict(y=None), ann.EINVAL, "NULL"), (dict(dim=0), ann.EINVAL, "dim"),
    (dict(type=3, table_type=3), ann.EINVAL, "type"), (dict(table_type=ann.F16), ann.EINVAL, "tables"), (dict(table_stride=7), ann.EINVAL, "stride"),
    (dict(type=ann.F32), ann.EINVAL, "tables"), (dict(y_stride=7), ann.EINVAL, "stride"), (dict(n=1 << 31), ann.ECAPACITY, "2^31"),
    (dict(rows=(1 << 31) + 1), ann.ECAPACITY, "2^31"), (dict(dim=ann.MAX_NORM_DIM + 1), ann.ECAPACITY, "ANN_MAX_NORM_DIM"),
])
def test_embedding_refuses(change, status, words):
    refused(status, words, ann.ann_embedding, **{**EMBED, **change})


GRAD = dict(dy=16, dy_stride=8, type=ann.F16, ids=16, n=2, scale=1.0, rows=4, dim=8, dtable=16, dtable_stride=8, table_type=ann.F32, workspace=256,
            workspace_bytes=1 << 20)


@pytest.mark.parametrize("change, status, words", [
    (dict(dy=None), ann.EINVAL, "NULL"), (dict(ids=None), ann.EINVAL, "NULL"), (dict(dtable=None), ann.EINVAL, "NULL"), (dict(dim=0), ann.EINVAL, "dim"),
    (dict(type=7), ann.EINVAL, "type"), (dict(table_type=ann.BF16), ann.EINVAL, "tables"), (dict(dy_stride=7), ann.EINVAL, "stride"),
    (dict(dtable_stride=7), ann.EINVAL, "stride"), (dict(n=1 << 31), ann.ECAPACITY, "2^31"), (dict(workspace=None), ann.EINVAL, "workspace"),
    (dict(workspace_bytes=8), ann.EINVAL, "needed"), (dict(workspace=264), ann.EINVAL, "aligned"),
])
def test_embedding_backward_refuses(change, status, words):
    refused(status, words, ann.ann_embedding_backward, **{**GRAD, **change})


NORM = dict(x=16, n=2, dim=8, x_stride=8, type=ann.BF16, weight=None, weight_type=ann.BF16, eps=1e-6, y=32, y_stride=8, residual=48, residual_stride=8,
            sum=64, sum_stride=8)
NORM8 = dict(NORM, group=32, scales=80, scale_stride=1)
COMMON = [
    (dict(x=None), ann.EINVAL, "NULL"), (dict(y=None), ann.EINVAL, "NULL"), (dict(dim=0), ann.EINVAL, "dim"), (dict(type=3), ann.EINVAL, "type"),
    (dict(weight=16, weight_type=ann.F16), ann.EINVAL, "weights"), (dict(x_stride=7), ann.EINVAL, "stride"), (dict(y_stride=7), ann.EINVAL, "stride"),
    (dict(residual_stride=7), ann.EINVAL, "stride"), (dict(sum_stride=7), ann.EINVAL, "stride"), (dict(residual=None), ann.EINVAL, "sum without"),
    (dict(sum=32), ann.EINVAL, "same rows"), (dict(eps=-1.0), ann.EINVAL, "eps"), (dict(eps=math.nan), ann.EINVAL, "eps"),
    (dict(dim=ann.MAX_NORM_DIM + 1), ann.ECAPACITY, "ANN_MAX_NORM_DIM"), (dict(n=1 << 40), ann.ECAPACITY, "n ="),
]


@pytest.mark.parametrize("change, status, words", COMMON)
def test_rms_norm_refuses(change, status, words):
    refused(status, words, ann.ann_rms_norm, **{**NORM, **change})


@pytest.mark.parametrize("change, status, words", COMMON + [
    (dict(group=16), ann.EINVAL, "group"), (dict(group=256), ann.EINVAL, "group"), (dict(scales=None), ann.EINVAL, "scales"),
    (dict(scale_stride=0), ann.EINVAL, "scale_stride"), (dict(dim=33, x_stride=33, y_stride=33, residual_stride=33, sum_stride=33), ann.EINVAL, "scale_stride"),
    (dict(y=16), ann.EINVAL, "place"), (dict(y=48), ann.EINVAL, "place"),
])
def test_rms_norm_e4m3_refuses(change, status, words):
    refused(status, words, ann.ann_rms_norm_e4m3, **{**NORM8, **change})


BACK = dict(dy=16, dy_stride=8, h=16, h_stride=8, n=2, dim=8, type=ann.F16, weight=16, weight_type=ann.F32, rstd=16, dx=16, dx_stride=8, dsum=16,
            dsum_stride=8, dweight=16, workspace=256, workspace_bytes=1 << 20)


@pytest.mark.parametrize("change, status, words", [
    (dict(dy=None), ann.EINVAL, "NULL"), (dict(h=None), ann.EINVAL, "NULL"), (dict(rstd=None), ann.EINVAL, "NULL"), (dict(dx=None), ann.EINVAL, "NULL"),
    (dict(dy_stride=7), ann.EINVAL, "stride"), (dict(h_stride=7), ann.EINVAL, "stride"), (dict(dx_stride=7), ann.EINVAL, "stride"),
    (dict(dsum_stride=7), ann.EINVAL, "stride"), (dict(workspace=None), ann.EINVAL, "workspace"), (dict(workspace_bytes=31), ann.EINVAL, "needed"),
    (dict(workspace=264), ann.EINVAL, "aligned"), (dict(weight=None, weight_type=ann.BF16), ann.EINVAL, "weights"), (dict(dim=0), ann.EINVAL, "dim"),
])
def test_rms_norm_backward_refuses(change, status, words):
    refused(status, words, ann.ann_rms_norm_backward, **{**BACK, **change})


def test_nothing_is_no_work():
    ann.ann_embedding(**{**EMBED, "n": 0, "ids": None, "y": None})
    ann.ann_embedding_backward(**{**GRAD, "n": 0, "rows": 0, "dy": None, "ids": None, "dtable": None, "workspace": None, "workspace_bytes": 0})
    ann.ann_rms_norm(**{**NORM, "n": 0, "x": None, "y": None})
    ann.ann_rms_norm_e4m3(**{**NORM8, "n": 0, "x": None, "y": None, "scales": None})
    ann.ann_rms_norm_backward(**{**BACK, "n": 0, "dy": None, "h": None, "dx": None, "rstd": None, "dweight": None, "workspace": None, "workspace_bytes": 0})


def test_workspaces():
    assert ann.ann_rms_norm_backward_workspace(0, 100) == ann.ann_embedding_backward_workspace(0, 10, 100) == 0
    assert 0 < ann.ann_rms_norm_backward_workspace(1, 100) <= ann.ann_rms_norm_backward_workspace(1 << 30, 100) < 1 << 20
    # 16 bytes of order to an id, and parts whose number has an end
    assert ann.ann_embedding_backward_workspace(100_000_000, 50_000, 1000) < 16 * 100_000_000 + (1 << 29)


SCORES = dict(q=16, nq=2, q_stride=8, rows=16, n=4, row_stride=8, d=8, type=ann.BF16, k=2, given_ids=16, given_logprobs=16, workspace=256, workspace_bytes=1 << 30)
DISTILL = dict(SCORES, loss=16, lse=16, logprobs=16)
DISTILL_BACK = dict(SCORES, lse=16, logprobs=16, g_loss=16, dq=16, dq_stride=8, drows=16, drows_stride=8)
DISTILL_COMMON = [
    (dict(q=None), ann.EINVAL, "q is NULL"), (dict(rows=None), ann.EINVAL, "rows is NULL"), (dict(d=0), ann.EINVAL, "d == 0"), (dict(type=3), ann.EINVAL, "type"),
    (dict(q_stride=7), ann.EINVAL, "stride"), (dict(scale=math.inf), ann.EINVAL, "scale"), (dict(k=0), ann.EINVAL, "k == 0"),
    (dict(k=ann.MAX_ALTERNATIVES + 1), ann.ECAPACITY, "ANN_MAX_ALTERNATIVES"), (dict(given_ids=None), ann.EINVAL, "given_ids"),
    (dict(given_logprobs=None), ann.EINVAL, "given_ids"), (dict(lse=None), ann.EINVAL, "lse"), (dict(logprobs=None), ann.EINVAL, "lse"),
    (dict(n=1 << 31), ann.ECAPACITY, "2^31"), (dict(nq=1 << 24), ann.ECAPACITY, "2^24"), (dict(workspace=None), ann.EINVAL, "workspace"),
    (dict(workspace_bytes=7), ann.EINVAL, "needed"), (dict(workspace=264), ann.EINVAL, "aligned"),
]


@pytest.mark.parametrize("change, status, words", DISTILL_COMMON + [(dict(loss=None), ann.EINVAL, "loss")])
def test_row_distillation_refuses(change, status, words):
    refused(status, words, ann.ann_row_distillation, **{**DISTILL, **change})


@pytest.mark.parametrize("change, status, words", DISTILL_COMMON + [
    (dict(g_loss=None), ann.EINVAL, "g_loss"), (dict(dq_stride=7), ann.EINVAL, "dq_stride"), (dict(drows_stride=7), ann.EINVAL, "drows_stride"),
])
def test_row_distillation_backward_refuses(change, status, words):
    refused(status, words, ann.ann_row_distillation_backward, **{**DISTILL_BACK, **change})


def test_targets_are_refused():
    import ctypes
    scores = ann.RowScores(q=16, rows=16, n=4, q_stride=8, row_stride=8, nq=2, d=8, type=ann.BF16, scale=1.0, row_bias=None, targets=16)
    assert ann._lib.ann_row_distillation(ctypes.byref(scores), 2, 16, 16, 16, 16, 16, 256, 1 << 30, None) == ann.EINVAL
    assert ann._lib.ann_row_distillation_backward(ctypes.byref(scores), 2, 16, 16, 16, 16, 16, 16, 8, 16, 8, None, 256, 1 << 30, None) == ann.EINVAL


def test_distillation_of_no_queries_is_no_work():
    ann.ann_row_distillation(**{**DISTILL, "nq": 0, "q": None, "loss": None, "lse": None, "logprobs": None, "workspace": None, "workspace_bytes": 0})
    for t in (ann.F32, ann.F16, ann.BF16):
        assert ann.ann_row_distillation_workspace(0, 100, 8, t, 1) == ann.ann_row_distillation_backward_workspace(0, 100, 8, t, 1) == 0
        # sums for the smaller of the rows and the entries
        few, many = (ann.ann_row_distillation_backward_workspace(nq, 1_000_000, 128, t, 8) for nq in (100, 10_000))
        assert few < 1 << 29 and many < 1 << 31
