"""Importing the binding loads neither torch nor a second HIP runtime, whatever is imported first, and does not need a torch that works (no GPU)."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
RUNTIMES = "sorted({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l})"


def run(code, *paths):
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([*map(str, paths), str(ROOT)]))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, env=env, cwd="/", timeout=300)
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


def test_torch_is_not_imported():
    assert run("import sys, paper_2503_17911_amd as a; print('torch' in sys.modules, a.ann_default_expansions_per_step(64, 32))") == ["False", "4"]


@pytest.mark.parametrize("first, second", [("paper_2503_17911_amd", "torch"), ("torch", "paper_2503_17911_amd")])
def test_one_runtime(first, second):
    assert run(f"import {first}, {second}; print(len({RUNTIMES}))") == ["1"]


@pytest.mark.parametrize("torch", [None, "raise OSError('libtorch_cpu.so: cannot open shared object file')", "raise ImportError('no')", "raise RuntimeError('broken')"])
def test_a_torch_that_does_not_work(tmp_path, torch):
    """An installation that fails, and one without the runtime, before the real one on the path."""
    (tmp_path / "torch" / "lib").mkdir(parents=True)
    (tmp_path / "torch" / "__init__.py").write_text(torch or "")
    if torch and "OSError" in torch:
        (tmp_path / "torch" / "lib" / "libamdhip64.so").write_text("not a library")
    assert run(f"import paper_2503_17911_amd as a; print(a.ann_default_expansions_per_step(64, 32), len({RUNTIMES}))", tmp_path) == ["4", "1"]
