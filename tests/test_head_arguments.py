"""Arguments that the operators of a model's head refuse on the host, and the
sizes of their workspaces (no GPU)."""
import math

import pytest

import paper_2503_17911_amd as ann


def refused(status, words, call, *args, **kw):
    with pytest.raises(ann.AnnError) as e:
        call(*args, **kw)
    assert e.value.status == status and words in str(e.value)


NORM = dict(x=16, n=2, dim=8, x_stride=8, type=ann.BF16, weight=None, bias=None, weight_type=ann.BF16, eps=1e-5, y=16, y_stride=8)


@pytest.mark.parametrize("change, status, words", [
    (dict(x=None), ann.EINVAL, "NULL"), (dict(y=None), ann.EINVAL, "NULL"), (dict(dim=0), ann.EINVAL, "dim"),
    (dict(type=3), ann.EINVAL, "type"), (dict(weight=16, weight_type=ann.F16), ann.EINVAL, "weights"),
    (dict(bias=16, weight_type=7), ann.EINVAL, "weights"), (dict(x_stride=7), ann.EINVAL, "stride"), (dict(y_stride=7), ann.EINVAL, "stride"),
    (dict(eps=-1.0), ann.EINVAL, "eps"), (dict(eps=math.nan), ann.EINVAL, "eps"),
    (dict(dim=ann.MAX_NORM_DIM + 1, x_stride=1 << 21, y_stride=1 << 21), ann.ECAPACITY, "ANN_MAX_NORM_DIM"),
    (dict(n=1 << 40), ann.ECAPACITY, "n ="),
])
def test_layer_norm_refuses(change, status, words):
    refused(status, words, ann.ann_layer_norm, **{**NORM, **change})


def test_layer_norm_of_nothing_is_no_work():
    ann.ann_layer_norm(**{**NORM, "n": 0, "x": None, "y": None})


GRAD = dict(dy=16, dy_stride=8, x=16, x_stride=8, n=2, dim=8, type=ann.F16, weight=16, weight_type=ann.F32, mean=16, rstd=16, dx=16,
            dx_stride=8, dweight=16, dbias=16, workspace=16, workspace_bytes=1 << 20)


@pytest.mark.parametrize("change, status, words", [
    (dict(dy=None), ann.EINVAL, "NULL"), (dict(x=None), ann.EINVAL, "NULL"), (dict(mean=None), ann.EINVAL, "NULL"),
    (dict(rstd=None), ann.EINVAL, "NULL"), (dict(dx=None), ann.EINVAL, "NULL"), (dict(workspace=None), ann.EINVAL, "workspace"),
    (dict(workspace_bytes=2 * 8 * 4 - 1), ann.EINVAL, "workspace"), (dict(workspace=18), ann.EINVAL, "aligned"),
    (dict(dy_stride=7), ann.EINVAL, "stride"), (dict(x_stride=7), ann.EINVAL, "stride"), (dict(dx_stride=7), ann.EINVAL, "stride"),
    (dict(weight=None, dbias=None, weight_type=ann.BF16), ann.EINVAL, "weights"), (dict(dim=0), ann.EINVAL, "dim"),
])
def test_layer_norm_backward_refuses(change, status, words):
    refused(status, words, ann.ann_layer_norm_backward, **{**GRAD, **change})


SCORES = dict(q=16, nq=2, q_stride=8, rows=16, n=4, row_stride=8, d=8, type=ann.BF16)
FORWARD = dict(SCORES, logprob=16, lse=16, k=2, alt_ids=16, alt_logprobs=16, workspace=256, workspace_bytes=1 << 30)
BACKWARD = dict(SCORES, lse=16, dq=16, dq_stride=8, drows=16, drows_stride=8, workspace=256, workspace_bytes=1 << 30)
COMMON = [
    (dict(q=None), ann.EINVAL, "q is NULL"), (dict(rows=None), ann.EINVAL, "rows is NULL"), (dict(d=0), ann.EINVAL, "d == 0"),
    (dict(type=3), ann.EINVAL, "type"), (dict(q_stride=7), ann.EINVAL, "stride"), (dict(row_stride=7), ann.EINVAL, "stride"),
    (dict(scale=math.inf), ann.EINVAL, "scale"), (dict(scale=math.nan), ann.EINVAL, "scale"), (dict(n=1 << 31), ann.ECAPACITY, "2^31"),
    (dict(nq=1 << 31), ann.ECAPACITY, "2^31"),
    (dict(d=ann.MAX_SCORE_DIM + 1, q_stride=1 << 14, row_stride=1 << 14), ann.ECAPACITY, "ANN_MAX_SCORE_DIM"),
    (dict(workspace=None), ann.EINVAL, "workspace"), (dict(workspace_bytes=8), ann.EINVAL, "needed"), (dict(workspace=264), ann.EINVAL, "aligned"),
]


@pytest.mark.parametrize("change, status, words", COMMON + [
    (dict(logprob=None), ann.EINVAL, "logprob"), (dict(lse=None), ann.EINVAL, "lse"), (dict(k=0), ann.EINVAL, "k = 0"),
    (dict(alt_ids=None), ann.EINVAL, "alt_ids"), (dict(alt_logprobs=None), ann.EINVAL, "alt_ids"),
    (dict(k=ann.MAX_ALTERNATIVES + 1), ann.ECAPACITY, "ANN_MAX_ALTERNATIVES"),
])
def test_row_logprobs_refuses(change, status, words):
    refused(status, words, ann.ann_row_logprobs, **{**FORWARD, **change})


@pytest.mark.parametrize("change, status, words", COMMON + [
    (dict(lse=None), ann.EINVAL, "lse"), (dict(g_entropy=16), ann.EINVAL, "entropy"), (dict(dq_stride=7), ann.EINVAL, "dq_stride"),
    (dict(drows_stride=7), ann.EINVAL, "drows_stride"),
])
def test_row_logprobs_backward_refuses(change, status, words):
    refused(status, words, ann.ann_row_logprobs_backward, **{**BACKWARD, **change})


def test_no_queries_are_no_work():
    ann.ann_row_logprobs(**{**FORWARD, "nq": 0, "q": None, "workspace": None, "workspace_bytes": 0})


def test_workspaces():
    assert ann.ann_layer_norm_backward_workspace(0, 100) == 0
    assert 0 < ann.ann_layer_norm_backward_workspace(1, 100) <= ann.ann_layer_norm_backward_workspace(1 << 30, 100) < 1 << 20
    for t in (ann.F32, ann.F16, ann.BF16):
        assert ann.ann_row_logprobs_workspace(0, 100, 8, t, 1) == ann.ann_row_logprobs_workspace(10, 0, 8, t, 1) == 0
        assert ann.ann_row_logprobs_workspace(10, 1000, 8, t, 0) < ann.ann_row_logprobs_workspace(10, 1000, 8, t, 5)
        # the gradient's does not grow with the rows without end
        assert ann.ann_row_logprobs_backward_workspace(10_000, 100_000_000, 128, t) < 2 << 30
