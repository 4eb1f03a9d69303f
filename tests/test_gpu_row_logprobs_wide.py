"""Log probabilities of rows where the tables are large enough for the kernels
that take 256 rows at a time, and alternatives among scores of large size."""
import math

import pytest
import torch

import head_reference as R
import test_gpu_row_logprobs as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bias", ["none", "plain", "holes"])
@pytest.mark.parametrize("nq, n, d, k", [(1100, 15_001, 192, 10), (300, 50_003, 160, 1), (1153, 14_080, 224, 0), (129, 66_000, 256, 64), (1100, 15_001, 136, 2)])
def test_forward(nq, n, d, k, bias, dtype):
    import paper_2503_17911_amd as ann
    q, rows, b, target = L.inputs(nq, n, d, dtype, n + d, bias)
    # (pad 8: rows of whole 16-byte pieces)
    L.check_forward(ann, q, rows, b, target, 20.0 if bias != "plain" else -5.0, k, 8)


def test_rows_left_out_and_not_numbers():
    """Runs of rows left out, among them whole groups and tiles; rows left out hold NaN."""
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(700, 24_000, 192, "bf16", 5)
    b = torch.zeros(24_000)
    b[512:1024] = -math.inf
    b[4096:4112] = -math.inf
    b[8000:8031] = -math.inf
    b[23_990:] = -math.inf
    held = rows.clone()
    held[b == -math.inf] = 0.0
    want = L.check_forward(ann, q, held, b, target, 20.0, 20)
    held[b == -math.inf] = float("nan")
    got = L.forward(ann, q, held, b, target, 20.0, 20)
    for f in want:
        assert torch.equal(want[f], got[f]), f


@pytest.mark.parametrize("nq, n, d", [(5, 3000, 40), (70, 3000, 40), (70, 3000, 200), (700, 24_000, 192)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_behind_a_large_mask(nq, n, d, dtype):
    """All rows but three carry -1e6: the other alternatives differ by less than fp32 keeps of their scores."""
    import paper_2503_17911_amd as ann
    q, rows, _, target = L.inputs(nq, n, d, dtype, 21)
    b = torch.full((n,), -1e6)
    b[[7, n // 2, n - 1]] = 0.0
    L.check_forward(ann, q, rows, b, target, 20.0, 20)


def test_strides_that_the_wide_tiles_do_not_take():
    import paper_2503_17911_amd as ann
    q, rows, b, target = L.inputs(1100, 15_001, 192, "bf16", 8)
    want = L.forward(ann, q, rows, b, target, 20.0, 10)
    got = L.forward(ann, q, rows, b, target, 20.0, 10, pad=3)
    err = R.score_error(q, rows, 20.0, b).float() + 1e-5
    assert torch.equal(want["alt_ids"], got["alt_ids"])
    for f in ("lse", "logprob"):
        assert ((want[f] - got[f]).abs() <= 2 * err).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nq, n, d", [(1100, 15_001, 160), (300, 50_003, 192), (257, 47_000, 224), (1100, 15_001, 136)])
def test_backward(nq, n, d, dtype):
    import paper_2503_17911_amd as ann
    gen = torch.Generator().manual_seed(nq + n)
    q, rows, b, target = L.inputs(nq, n, d, dtype, n + d)
    g, h = -0.5 - torch.rand(nq, generator=gen), 0.2 * torch.randn(nq, generator=gen)
    L.check_backward(ann, q, rows, b, target, 20.0, g, h)
    L.check_backward(ann, q, rows, b, target, -3.0, g, None, 8)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_backward_in_several_chunks(dtype):
    """G of more than 512 MiB: rows are taken in parts, the queries' gradient is carried from part to part."""
    import paper_2503_17911_amd as ann
    nq, n, d, scale = 2100, 150_100, 160, 20.0
    t, gen = R.DTYPES[dtype], torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(n, d, generator=gen, device="cuda")
    rows = (rows / rows.norm(dim=1, keepdim=True)).to(t)
    target = torch.randint(n, (nq,), generator=gen, device="cuda")
    q = rows[target].float() + 0.05 * torch.randn(nq, d, generator=gen, device="cuda")
    q = (q / q.norm(dim=1, keepdim=True)).to(t)
    q64, x64 = q.double(), rows.double()
    logp = scale * torch.mm(q64, x64.t().contiguous())
    lse = torch.logsumexp(logp, 1).float()
    logp -= lse.double()[:, None]
    p = logp.exp()
    g = -0.5 - torch.rand(nq, generator=gen, device="cuda")
    G = -g.double()[:, None] * p
    G[torch.arange(nq, device="cuda"), target] += g.double()
    dq, drows, dbias = torch.empty_like(q), torch.empty_like(rows), torch.empty(n, device="cuda")
    ty = L.types(ann)[t]
    need = ann.ann_row_logprobs_backward_workspace(nq, n, d, ty)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ann.ann_row_logprobs_backward(q, nq, d, rows, n, d, d, ty, lse=lse, scale=scale, targets=target.int(), g_logprob=g, dq=dq, dq_stride=d,
                                  drows=drows, drows_stride=d, drow_bias=dbias, workspace=ws, workspace_bytes=need, stream=L.stream())
    # the score's error (d additions of at most the norms' product, twice; four roundings), G's rounding to 16 bits, the result's
    half = R.half_step(t)
    norms = scale * q64.norm(dim=1) * x64.norm(dim=1).max()
    err = ((d + 64) * 2 * R.U32 * norms + 4 * R.U32 * norms + 12 * R.U32 * (1 + lse.double().abs()))[:, None]
    off = g.double().abs()[:, None] * p * (err + 8 * R.U32) + (half + 2 * R.U32) * G.abs() + (2.0 ** -38 * g.abs().max().item() if t == torch.float16 else 0.0)
    for got, want, bound, terms, length in (
            (dq, torch.mm(G, x64), torch.mm(off, x64.abs()), torch.mm(G.abs(), x64.abs()), n),
            (drows, torch.mm(G.t().contiguous(), q64), torch.mm(off.t().contiguous(), q64.abs()), torch.mm(G.abs().t().contiguous(), q64.abs()), nq)):
        tol = scale * (half * want.abs() + bound + (2 * length + 64) * R.U32 * terms) * (1 + half) + R.smallest_step(t)
        assert ((got.double() - scale * want).abs() <= tol).all()
    assert ((dbias.double() - G.sum(0)).abs() <= off.sum(0) + (nq + 64) * R.U32 * G.abs().sum(0)).all()
