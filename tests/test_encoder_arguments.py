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
