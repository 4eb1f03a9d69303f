"""The example that teaches an encoder of tokens: embedding, norms and loss together, as they are used."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "distill_query_encoder.py"
    spec = importlib.util.spec_from_file_location("distill_query_encoder", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_runs():
    got = example().train(n=3000, d=64, hidden=96, tokens=500, length=7, batch=64, steps=6, report=lambda _: None)
    assert len(got["losses"]) == 6 and all(0 < v < 100 for v in got["losses"])
    assert ((got["mine"] >= 0) & (got["mine"] < 3000)).all()


def plain_loss(p, ids, rows, rows_given, given, scale, eps):
    """The same encoder and loss by torch's operations in 64 bits."""
    table, *layers, last, project = p
    hidden = table.shape[1]
    flat = ids.reshape(-1).long()
    x = table[flat.clamp_min(0)] * hidden ** 0.5 * (flat >= 0)[:, None]
    h = torch.zeros_like(x)

    def norm(h, w):
        return h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w

    for weight, up, down in zip(*(layers[i::3] for i in range(3))):
        h = h + x
        x = torch.mm(torch.tanh(torch.mm(norm(h, weight), up)), down)
    y = norm(h + x, last)
    there = (ids >= 0).double()
    q = torch.mm((y.view(*ids.shape, hidden) * there[:, :, None]).sum(1) / there.sum(1, keepdim=True), project)
    logp = torch.log_softmax(scale * torch.mm(q, rows.t().contiguous()), 1)
    return (given.exp() * (given - logp.gather(1, rows_given.long()))).sum(1)


def test_the_gradients_are_those_of_torch():
    """All parameters' gradients, from the tokens' table to the projection, and the rows', fp32 against 64 bits."""
    m = example()
    g = torch.Generator(device="cuda").manual_seed(2)
    p = m.parameters(300, 80, 2, 48, g)
    ids = torch.randint(300, (40, 9), generator=g, device="cuda", dtype=torch.int32)
    ids[:, 5:][torch.rand(40, 4, generator=g, device="cuda") < 0.5] = -1
    rows = torch.randn(700, 48, generator=g, device="cuda", requires_grad=True)
    rows_given, given = m.teacher_answers(torch.randn(40, 48, generator=g, device="cuda"), rows.detach(), 0.4, 8)
    loss = m.RowDistillation.apply(m.queries(p, ids, torch.float32), rows, rows_given, given, 0.4)
    loss.mean().backward()
    p64 = [v.detach().double().requires_grad_() for v in p]
    rows64 = rows.detach().double().requires_grad_()
    want = plain_loss(p64, ids, rows64, rows_given, given.double(), 0.4, m.EPS)
    want.mean().backward()
    assert ((loss.double() - want).abs() <= 1e-4 * (1 + want.abs())).all()
    # relative to each gradient's largest element: chains of a dozen sums of at most 700 fp32 terms (and torch's fp32 products between), each off by at
    # most some 700 x 2^-24 = 4e-5 of its terms' sizes
    for got, exact in zip((*p, rows), (*p64, rows64)):
        assert ((got.grad.double() - exact.grad).abs().max() <= 1e-3 * exact.grad.abs().max()).all()
    assert (p[0].grad[torch.bincount(ids[ids >= 0].long(), minlength=300) == 0] == 0).all()


def test_states_in_8_bits_are_the_norms():
    """The norm's output in 8 bits stands for the output in 16: a product with either differs by the codes' rounding."""
    import paper_2503_17911_amd as ann
    m = example()
    n, d = 33, 256
    g = torch.Generator(device="cuda").manual_seed(3)
    x, h = (torch.randn(n, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(d, generator=g, device="cuda") + 0.5
    y, kept = m.AddRmsNorm.apply(x, h, w)
    codes, scales = torch.empty(n, d, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(n, d // 128, device="cuda")
    kept8 = torch.empty_like(x)
    ann.ann_rms_norm_e4m3(x, n, d, d, ann.BF16, w, ann.F32, m.EPS, codes, d, 128, scales, d // 128, residual=h, residual_stride=d, sum=kept8, sum_stride=d,
                          stream=m.stream())
    assert torch.equal(kept, kept8)
    v = codes.float() * scales.repeat_interleave(128, 1)
    # a code is off by half a step of e4m3 (2^-4, or 2^-10 of the scale), y by half a step of bf16
    assert ((v - y.float()).abs() <= (2.0 ** -4 + 2.0 ** -8) * y.float().abs() * 1.01 + 2.0 ** -10 * scales.repeat_interleave(128, 1)).all()


def test_the_package_may_be_imported_before_torch():
    """In a process of its own: the library and torch share one HIP runtime whichever is asked for first."""
    import subprocess
    import sys
    code = ("import paper_2503_17911_amd as ann, torch\n"
            "x = torch.ones(4, 64, device='cuda'); y = torch.empty_like(x)\n"
            "ann.ann_rms_norm(x, 4, 64, 64, ann.F32, None, ann.F32, 0.0, y, 64, stream=torch.cuda.current_stream().cuda_stream)\n"
            "assert (y == 1).all()\n")
    root = Path(__file__).resolve().parent.parent
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]
