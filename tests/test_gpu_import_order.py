"""Tensors of torch reach the library whichever of the two a program imports first."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent
CODE = """
import {first}
import {second}
import torch
import paper_2503_17911_amd as ann
ann.ann_default_expansions_per_step(64, 32)
x = torch.arange(12.0, device="cuda").view(3, 4)
y = torch.empty(2, 4, device="cuda")
ann.ann_embedding(x, 3, 4, 4, ann.F32, torch.tensor([2, 0], dtype=torch.int32, device="cuda"), 2, 2.0, y, 4, ann.F32, torch.cuda.current_stream().cuda_stream)
print(y.tolist() == (2 * x[[2, 0]]).tolist())
"""


@pytest.mark.parametrize("first, second", [("paper_2503_17911_amd", "torch"), ("torch", "paper_2503_17911_amd")])
def test_both_orders(first, second):
    r = subprocess.run([sys.executable, "-c", CODE.format(first=first, second=second)], capture_output=True, text=True, timeout=100,
                       env=dict(os.environ, PYTHONPATH=str(ROOT)))
    assert r.returncode == 0 and r.stdout.split() == ["True"], r.stderr
