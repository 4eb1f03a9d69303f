"""Token embeddings and the table's gradient by sorted tokens, against their definitions in 64 bits."""
import math

import pytest
import torch

import encoder_reference as E
import head_reference as R
from test_gpu_layer_norm import strided, types

pytestmark = pytest.mark.gpu
PAD = -1
TYPES = [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")]


def stream():
    return torch.cuda.current_stream().cuda_stream


def tokens(n, rows, law, seed):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    if law == "zipf":
        ids = (torch.exp(u * math.log(rows + 1.0)) - 1).long()
    elif law == "one":
        ids = torch.full((n,), rows // 2)
    elif law == "each":
        ids = torch.arange(n) % rows
    elif law == "pads":
        ids = torch.full((n,), PAD)
    else:
        ids = (u * rows).long()
    ids = ids.clamp(-1, rows - 1)
    if law not in ("one", "pads"):
        ids[torch.rand(n, generator=g) < 0.1] = PAD
        ids[torch.rand(n, generator=g) < 0.02] = rows        # just behind the last row
        ids[torch.rand(n, generator=g) < 0.02] = 2 ** 31 - 1
    return ids


def on_gpu(ids):
    return ids.to(torch.int32).cuda()


@pytest.mark.parametrize("dtype, ttype", TYPES)
@pytest.mark.parametrize("n, rows, d", [(1, 1, 1), (1, 50_000, 768), (2, 3, 7), (37, 100, 100), (500, 40, 129), (33, 7, 1030), (9, 1000, 5000), (3, 0, 16),
                                        (70_000, 5000, 24)])
def test_forward(n, rows, d, dtype, ttype):
    import paper_2503_17911_amd as ann
    t, tt = R.DTYPES[dtype], R.DTYPES[ttype]
    g = torch.Generator().manual_seed(n + rows + d)
    table, ids = torch.randn(rows, d, generator=g).to(tt), tokens(n, max(rows, 1), "even", n)
    want = E.embedding(table, ids, 3.7)
    for pad, shift in ((0, 0), (8, 0), (1, 1)):
        td, y = strided(table, pad, shift) if rows else None, strided(torch.zeros(n, d, dtype=t), pad, shift)
        before = torch.as_strided(y, (n, d + pad), (d + pad, 1)) if shift == 0 else None
        if before is not None:
            before.fill_(7.0)
        ann.ann_embedding(td, rows, d, d + pad, types(ann)[ttype], on_gpu(ids), n, 3.7, y, y.stride(0), types(ann)[dtype], stream())
        half = R.half_step(t)
        assert ((y.cpu().double() - want).abs() <= (half + R.U32 * 2) * (1 + half) * want.abs() + R.smallest_step(t)).all()
        assert before is None or (before[:, d:] == 7.0).all()


SIZES = [(12_288, 3000, 40), (12_289, 3000, 40), (8192, 3000, 40), (8193, 3000, 40), (16_384, 3000, 8), (16_385, 3000, 8), (16_383, 40_000, 24), (40_001, 2047, 12), (40_001, 2048, 12), (1, 1, 8), (1, 200, 768), (2, 2, 1), (31, 5, 3), (32, 9, 100), (33, 1000, 129), (64, 64, 16), (65, 3, 260), (1000, 77, 100), (4096, 3000, 40),
         (4097, 3000, 40), (4097, 1, 8), (20_000, 70_000, 24), (9000, 100, 1030), (20_000, 900, 768), (150_000, 3000, 8), (300_000, 3, 20), (280_000, 1 << 22, 3), (300_000, 3_000_000, 2)]


@pytest.mark.parametrize("law", ["zipf", "one", "each", "pads", "even"])
@pytest.mark.parametrize("n, rows, d", SIZES)
def test_gradient(n, rows, d, law):
    import paper_2503_17911_amd as ann
    for i, (dtype, ttype) in enumerate(TYPES):
        if n * d > 200_000 and i not in (2, 3):
            continue
        check(ann, n, rows, d, law, dtype, ttype, *((0, 0), (8, 0), (1, 1))[(i + n) % 3])


def check(ann, n, rows, d, law, dtype, ttype, pad, shift):
    t, tt = R.DTYPES[dtype], R.DTYPES[ttype]
    g = torch.Generator().manual_seed(n + rows + d)
    ids, dy, old = tokens(n, rows, law, n), torch.randn(n, d, generator=g).to(t), torch.randn(rows, d, generator=g).to(tt)
    want, size, count = E.embedding_grad(dy, ids, 0.7, rows)
    dyd = strided(dy, pad, shift)
    need = ann.ann_embedding_backward_workspace(n, rows, d)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read before it is written)
    half, tiny = R.half_step(tt), R.smallest_step(tt)
    # as many additions as the row has terms, and at most sixteen to join its parts
    off = ((count + 16) * R.U32)[:, None] * size
    for accumulate in (False, True):
        out = torch.full((rows, d + pad), 7.0, dtype=tt, device="cuda")
        if accumulate:
            out[:, :d] = old.cuda()
        ann.ann_embedding_backward(dyd, dyd.stride(0), types(ann)[dtype], on_gpu(ids), n, 0.7, rows, d, out, d + pad, types(ann)[ttype], accumulate, ws, need,
                                   stream())
        got = out[:, :d].cpu()
        exact = want + old.double() if accumulate else want
        assert ((got.double() - exact).abs() <= (half * exact.abs() + tiny + off + 2 * R.U32 * (want.abs() + exact.abs())) * (1 + half)).all()
        none = count == 0
        assert torch.equal(got[none], old[none] if accumulate else torch.zeros_like(old)[none])
        assert (out[:, d:] == 7.0).all()


def test_nothing_to_sum():
    import paper_2503_17911_amd as ann
    out = torch.ones(5, 12, device="cuda")
    ann.ann_embedding_backward(None, 0, ann.F32, None, 0, 1.0, 5, 12, out, 12, ann.F32, accumulate=True, stream=stream())
    assert (out == 1).all()
    ann.ann_embedding_backward(None, 0, ann.F32, None, 0, 1.0, 5, 12, out, 12, ann.F32, stream=stream())
    assert (out == 0).all()


def test_rows_of_padding_do_not_count():
    import paper_2503_17911_amd as ann
    for n in (100, 6000):
        ids = tokens(n, 50, "even", 3)
        dy = torch.randn(n, 64)
        dy[(ids < 0) | (ids >= 50)] = float("nan")
        out = torch.empty(50, 64, device="cuda")
        need = ann.ann_embedding_backward_workspace(n, 50, 64)
        ann.ann_embedding_backward(dy.cuda(), 64, ann.F32, on_gpu(ids), n, 1.0, 50, 64, out, 64, ann.F32,
                                   workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need, stream=stream())
        assert torch.isfinite(out).all()


def test_same_bits_again_on_other_streams_and_in_graphs():
    import paper_2503_17911_amd as ann
    for n, rows, d, dtype in ((300, 40, 100, "f16"), (9000, 700, 96, "bf16"), (280_000, 2000, 16, "f32")):
        T = types(ann)[dtype]
        ids, dy = on_gpu(tokens(n, rows, "zipf", 5)), torch.randn(n, d, device="cuda").to(R.DTYPES[dtype])
        table = torch.randn(rows, d, device="cuda").to(dy.dtype)
        need = ann.ann_embedding_backward_workspace(n, rows, d)

        def outputs():
            return [torch.zeros_like(dy), torch.zeros_like(table), torch.zeros(need, dtype=torch.uint8, device="cuda")]

        def both(o):
            ann.ann_embedding(table, rows, d, d, T, ids, n, 2.0, o[0], d, T, stream())
            ann.ann_embedding_backward(dy, d, T, ids, n, 2.0, rows, d, o[1], d, T, workspace=o[2], workspace_bytes=need, stream=stream())

        want, other, graphed = outputs(), outputs(), outputs()
        both(want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            both(other)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[:2], other[:2]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(graphed)
        for replay in range(3):
            ids.copy_(on_gpu(tokens(n, rows, ("even", "one", "zipf")[replay], replay)))
            both(want)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want[:2], graphed[:2])), replay


def test_many_tokens():
    """More than the sort's blocks take in their usual rounds, and more chunks than there may be of the shortest; ones are summed exactly."""
    import paper_2503_17911_amd as ann
    n, rows = 17_500_000, 5000
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = (torch.exp(torch.rand(n, generator=g, device="cuda") * math.log(rows + 1.0)) - 1).int()
    out = torch.empty(rows, 1, device="cuda")
    need = ann.ann_embedding_backward_workspace(n, rows, 1)
    ann.ann_embedding_backward(torch.ones(n, 1, device="cuda", dtype=torch.bfloat16), 1, ann.BF16, ids, n, 1.0, rows, 1, out, 1, ann.F32,
                               workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need, stream=stream())
    count = torch.bincount(ids[ids < rows], minlength=rows)
    assert count.max() > 1 << 20 and torch.equal(out[:, 0].double(), count.double())


def test_offsets_beyond_32_bits():
    """Rows of the table, of y and of dy that lie more than 2^32 elements from the first."""
    import paper_2503_17911_amd as ann
    d, stride, rows = 8, 1 << 22, 1100
    far = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")   # 9.2 GB, of which every row's first elements are used
    table = far.view(rows, stride)
    table[:, :d] = torch.randn(rows, d, device="cuda").bfloat16()
    near = table[:, :d].contiguous()
    ids = torch.randperm(rows, device="cuda").int()
    y, y_far = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda"), table[:, 64:]
    ann.ann_embedding(near, rows, d, d, ann.BF16, ids, rows, 2.0, y, d, ann.BF16, stream())
    ann.ann_embedding(table, rows, d, stride, ann.BF16, ids, rows, 2.0, y_far, stride, ann.BF16, stream())
    assert torch.equal(y, y_far[:, :d]) and torch.equal(y, (2 * near.float())[ids.long()].bfloat16())
    need = ann.ann_embedding_backward_workspace(rows, rows, d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    grad, grad_far = torch.empty_like(y), table[:, 128:]
    ann.ann_embedding_backward(y, d, ann.BF16, ids, rows, 0.5, rows, d, grad, d, ann.BF16, workspace=ws, workspace_bytes=need, stream=stream())
    ann.ann_embedding_backward(y_far, stride, ann.BF16, ids, rows, 0.5, rows, d, grad_far, stride, ann.BF16, workspace=ws, workspace_bytes=need, stream=stream())
    assert torch.equal(grad, near) and torch.equal(grad_far[:, :d], near)


def test_rows_without_a_token_stay_as_they_are_between_batches():
    """Several batches into one gradient, the table's rows among them that it is also scored against: each is rounded into the table's type once."""
    import paper_2503_17911_amd as ann
    rows, d = 64, 40
    out = torch.randn(rows, d, device="cuda").bfloat16()
    want = out.clone()
    for n in (0, 5, 300):
        ids, dy = on_gpu(tokens(n, rows, "even", n)), torch.randint(-4, 5, (n, d), device="cuda").bfloat16()
        need = ann.ann_embedding_backward_workspace(n, rows, d)
        ann.ann_embedding_backward(dy, d, ann.BF16, ids, n, 1.0, rows, d, out, d, ann.BF16, accumulate=True,
                                   workspace=torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), workspace_bytes=need, stream=stream())
        there = (ids >= 0) & (ids < rows)
        add = torch.zeros(rows, d, device="cuda").index_add_(0, ids[there].long(), dy[there].float())   # (whole numbers: exact)
        hit = torch.bincount(ids[there].long(), minlength=rows) > 0
        want = torch.where(hit[:, None], (want.float() + add).bfloat16(), want)
        assert torch.equal(out, want)
