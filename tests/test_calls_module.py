"""The extension module that marshals the paged-cache operations (_calls.so): when it is built, and what works without it."""
import os
import subprocess
import sys

import pytest


@pytest.fixture
def compiler(tmp_path, monkeypatch):
    """build_calls with a compiler that only leaves a file, in a folder of its own; the commands that it was given."""
    from paper_2512_21571_b200 import build
    runs = []

    def run(cmd, **kw):
        runs.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built %d" % len(runs))
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(build.subprocess, "run", run)
    return build, runs


def test_the_module_is_built_once_for_a_torch_and_again_for_another(compiler, monkeypatch):
    import torch
    build, runs = compiler
    assert build.build_calls() == build.CALLS and len(runs) == 1
    build.build_calls()
    assert len(runs) == 1                                              # nothing changed
    monkeypatch.setattr(torch, "__version__", "99.0")
    build.build_calls()
    assert len(runs) == 2 and open(build.CALLS).read() == "built 2"    # another torch: its headers are others
    build.build_calls()
    assert len(runs) == 2
    monkeypatch.setenv("CUDA_HOME", "/elsewhere")
    build.build_calls()
    assert len(runs) == 3                                              # another command
    os.utime(build.CALLS, (1, 1))
    build.build_calls()
    assert len(runs) == 4                                              # sources newer than the module
    build.build_calls(force=True)
    assert len(runs) == 5


def test_a_module_without_a_stamp_is_built_again(compiler):
    build, runs = compiler
    with open(build.CALLS, "w") as f:
        f.write("of unknown origin")
    build.build_calls()
    assert len(runs) == 1 and open(build.CALLS).read() == "built 1"


def test_the_rest_of_the_binding_does_without_the_module():
    from paper_2512_21571_b200 import build
    build.build()
    prog = """
import sys
sys.path.insert(0, %r)
sys.modules["paper_2512_21571_b200._calls"] = None          # as if it were missing
from paper_2512_21571_b200 import binding as nnc
import torch
assert nnc.Model and nnc.bounds_check_report() == (-1, 0)
freq, amplitude = nnc.rope_frequencies(64, device="cpu")
assert freq[0] == 1.0
x = torch.zeros(2, 2, 64)
pos = torch.zeros(2, dtype=torch.int32)
for call in (lambda: nnc.op_rope(x, pos, freq), lambda: nnc.op_rope(x, pos, freq, out=x)):
    try:
        call()
    except ImportError as e:
        assert "paper_2512_21571_b200.build" in str(e) and e.__cause__ is not None
    else:
        raise AssertionError("no error")
print("done")
""" % os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", prog], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stdout + r.stderr
