"""The example that trains an encoder's last layers with the library's calls, small."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "train_query_encoder.py"
    spec = importlib.util.spec_from_file_location("train_query_encoder", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_and_answers():
    got = example().train(n=3000, d=64, hidden=192, batch=128, steps=60, report=lambda _: None)
    assert got["losses"][0] > 1.0 and got["losses"][-1] < 0.1 * got["losses"][0]
    assert got["hit"] > 0.9
    # the likeliest rows are the search's nearest by inner product (the same order: equal scores by their number in both)
    assert (got["ids"] == got["near"]).float().mean() > 0.99
    p = got["values"].double().exp()
    assert (p.sum(1) <= 1 + 1e-5).all() and (got["values"][:, 1:] <= got["values"][:, :-1]).all()


def test_the_loss_gradients_are_those_of_torch():
    m = example()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(40, 96, generator=g, device="cuda", requires_grad=True)
    weight = torch.randn(96, generator=g, device="cuda", requires_grad=True)
    bias = torch.randn(96, generator=g, device="cuda", requires_grad=True)
    rows = torch.randn(500, 96, generator=g, device="cuda", requires_grad=True)
    target = torch.randint(500, (40,), generator=g, device="cuda").int()
    logprob, entropy = m.RowLogProbs.apply(m.LayerNorm.apply(x, weight, bias, 1e-5), rows, target, 0.3)
    (-(logprob + 0.1 * entropy).mean()).backward()
    x64, w64, b64, r64 = (v.detach().double().requires_grad_() for v in (x, weight, bias, rows))
    mean = x64.mean(1, keepdim=True)
    y = (x64 - mean) / torch.sqrt(((x64 - mean) ** 2).mean(1, keepdim=True) + 1e-5) * w64 + b64
    logp = torch.log_softmax(0.3 * torch.mm(y, r64.t().contiguous()), 1)
    (-(logp.gather(1, target.long()[:, None])[:, 0] - 0.1 * (logp.exp() * logp).sum(1)).mean()).backward()
    # relative to each gradient's largest element: sums of 500 (or 40) terms with fp32 roundings of scores of size 30, 6 x 96 products each
    for got, want in ((x, x64), (weight, w64), (bias, b64), (rows, r64)):
        assert ((got.grad.double() - want.grad).abs().max() <= 1e-3 * want.grad.abs().max()).all()
