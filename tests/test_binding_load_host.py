"""The compiled binding is loaded by the first feed-forward call: the package imports without it, and one that was built for something
else is never loaded.  Needs no GPU: copies of the package are imported by processes that find no compiler."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2605_26660_b200 as wq

PACKAGE = os.path.dirname(os.path.abspath(wq.__file__))
ROOT = os.path.dirname(PACKAGE)

CALL = """
import types, torch
import paper_2605_26660_b200 as wq
print("imported", wq.windq_scratch_bytes_gated_forward(4, 64, 64) > 0)
ctx = types.SimpleNamespace(device=0, _h=types.SimpleNamespace(value=None), _check=None)
for _ in range(2):
    try:
        wq.windq_quantize_rows(ctx, torch.zeros(2, 8), stream=types.SimpleNamespace(cuda_stream=0))
    except Exception as e:
        print(type(e).__name__, e)
"""


def run(tmp_path, binding, stamp, program=CALL):
    """`program` in a copy of the package with that binding and stamp, where no compiler is on the path."""
    copy = tmp_path / "paper_2605_26660_b200"
    copy.mkdir()
    os.symlink(os.path.join(ROOT, "include"), tmp_path / "include")
    for name in os.listdir(PACKAGE):
        if not name.startswith(("_binding", "__pycache__")):
            os.symlink(os.path.join(PACKAGE, name), copy / name)
    for name in ("__init__.py", "_build.py"):          # python takes a package's place from where its file is
        os.unlink(copy / name)
        (copy / name).write_bytes(open(os.path.join(PACKAGE, name), "rb").read())
    if binding:
        os.symlink(os.path.join(PACKAGE, "_binding.so"), copy / "_binding.so")
    if stamp:
        (copy / "_binding.so.srchash").write_text(stamp)
    env = {k: v for k, v in os.environ.items() if k != "PYTHONPATH"} | {"PATH": str(tmp_path), "PYTHONPATH": str(tmp_path)}
    done = subprocess.run([sys.executable, "-c", program], cwd=tmp_path, env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    return done.stdout.splitlines()


def test_the_package_imports_without_a_binding(tmp_path):
    lines = run(tmp_path, False, None)
    assert lines[0] == "imported True" and all(line.startswith("ImportError the compiled binding") for line in lines[1:]) and len(lines) == 3


def test_a_binding_for_something_else_is_not_loaded(tmp_path):
    lines = run(tmp_path, True, "0" * 64)
    assert lines[0] == "imported True" and all(line.startswith("ImportError the compiled binding") for line in lines[1:]) and len(lines) == 3


def test_a_current_binding_needs_no_compiler(tmp_path):
    wq._build.build_binding()
    program = CALL + """
assert wq._binding.__name__ == "paper_2605_26660_b200._binding" and wq._binding.__file__.startswith(%r)
""" % str(tmp_path)
    gone = "import paper_2605_26660_b200._build as b\ndef none(): raise RuntimeError('no nvcc')\nb.nvcc_path = none\n"
    lines = run(tmp_path, True, wq._build.binding_hash(), gone + program)
    assert lines[0] == "imported True" and all(line.startswith("TypeError X must be") for line in lines[1:]) and len(lines) == 3


@pytest.mark.parametrize("owner,name", [(torch, "__version__"), (sys, "version")])
def test_what_a_binding_is_built_for_counts(monkeypatch, owner, name):
    before = wq._build.binding_hash()
    monkeypatch.setattr(owner, name, "another")
    assert wq._build.binding_hash() != before
