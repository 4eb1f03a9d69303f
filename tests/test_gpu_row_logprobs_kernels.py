"""Sizes at which the remaining kernels and ways through them are taken."""
import pytest
import torch

import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


# rows of at most 128 columns, many queries: groups of 64 rows (n >= 256 k d) and of 16, at least 512 queries (256 lanes each at the end)
@pytest.mark.parametrize("nq, n, d, k", [(70, 4100, 16, 1), (600, 4100, 16, 1), (600, 9001, 30, 1), (513, 25_000, 96, 1), (600, 3000, 128, 20), (700, 2908, 30, 32),
                                         (900, 333, 92, 64), (65, 33_000, 128, 1)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_short_rows(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    for bias, pad, scale in (("none", 0, 20.0), ("none", 8, -7.0), ("plain", 1, 5.0), ("holes", 8, 20.0)):
        q, rows, b, target = L.inputs(nq, n, d, dtype, n + d, bias)
        L.check_forward(ann, q, rows, b, target, scale, k, pad)


@pytest.mark.parametrize("nq, n, d, k", [(40, 900, 2000, 40), (130, 600, 4096, 64), (600, 1500, 1025, 33), (600, 3001, 130, 50)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_long_rows_and_many_alternatives(nq, n, d, k, dtype):
    import paper_2503_17911_amd as ann
    for bias, pad, scale in (("none", 0, -20.0), ("holes", 3, 20.0)):
        q, rows, b, target = L.inputs(nq, n, d, dtype, n + d, bias)
        L.check_forward(ann, q, rows, b, target, scale, k, pad)


@pytest.mark.parametrize("dtype, n, d", [("f32", 66_000, 40), ("bf16", 130_000, 136)])
def test_backward_in_several_chunks_with_biases_and_entropy(dtype, n, d):
    import paper_2503_17911_amd as ann
    nq = 2100
    q, rows, b, target = L.inputs(nq, n, d, dtype, 7, "holes")
    gen = torch.Generator().manual_seed(5)
    L.check_backward(ann, q, rows, b, target, 20.0, -0.5 - torch.rand(nq, generator=gen), 0.2 * torch.randn(nq, generator=gen))
