"""Sizes whose launches would have more lanes than there may be are refused."""
import pytest

import paper_2503_17911_amd as ann


@pytest.mark.parametrize("nq, n", [(1 << 24, 10), (10, (1 << 31) - 255)])
def test_too_many_queries_or_rows(nq, n):
    one = 1 << 12  # an address: nothing is read
    with pytest.raises(ann.AnnError, match="2\\^24"):
        ann.ann_row_logprobs(one, nq, 8, one, n, 8, 8, ann.F32, logprob=one, lse=one)
    with pytest.raises(ann.AnnError, match="2\\^24"):
        ann.ann_row_logprobs_backward(one, nq, 8, one, n, 8, 8, ann.F32, lse=one)
    assert ann.ann_row_logprobs_workspace(nq, n, 8, ann.F32, 1) == 0 and ann.ann_row_logprobs_backward_workspace(nq, n, 8, ann.F32) == 0
