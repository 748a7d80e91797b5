"""Callers that use the step alone do without the operators: without the extension that marshals their arguments, and with a
build of the library from before them.  No compute call is made here (no GPU needed)."""
import os
import subprocess
import sys

import pytest

from paper_2103_07454_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ASKS = """
import torch
from paper_2103_07454_b200 import binding as B
lib = B.load_library()
assert lib.eg_step.argtypes is not None and B._lib is lib
try:
    B.residual_norm(torch.zeros(1, 2, 8), torch.zeros(1, 2, 8))
except B.EventGradError as e:
    assert "build" in str(e), e
else:
    raise AssertionError("an operator was called")
print("done")
"""


def run(code, **env):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT, **env), capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr


def test_without_the_extension():
    run("import sys\nsys.modules['paper_2103_07454_b200._marshal'] = None\n" + ASKS)


def test_with_a_library_from_before_the_operators(tmp_path):
    operators = set(B._OPERATORS) | {"eg_operator_status", "eg_selftest_operator_wait"}
    assert operators <= set(B.EXPORTS)
    src = tmp_path / "older.c"
    src.write_text("\n".join(f"int {name}(void) {{ return 0; }}" for name in B.EXPORTS if name not in operators))
    lib = tmp_path / "older.so"
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    run(ASKS, EG_LIBRARY=str(lib))


def test_operators_are_there_in_this_build():
    assert B._operators() is B._operators()
    with pytest.raises(TypeError):
        B._operators().residual_norm()


def test_the_extension_is_built_again_for_another_torch_or_interpreter(tmp_path, monkeypatch):
    """It is compiled against both; its source's time says nothing about them."""
    from paper_2103_07454_b200 import build
    calls = []

    def compiler(cmd, check):
        calls.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build, "MARSHAL_STAMP", str(tmp_path / "deep" / "_marshal.txt"))
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build.build_marshal()
    build.build_marshal()
    assert len(calls) == 1
    monkeypatch.setattr(build.sys, "version", "another interpreter")
    build.build_marshal()
    build.build_marshal()
    assert len(calls) == 2
    here = build._stamp()
    monkeypatch.setattr(build, "_stamp", lambda: here + "another torch")
    build.build_marshal()
    build.build_marshal()
    assert len(calls) == 3
    build.build_marshal(force=True)
    assert len(calls) == 4
    os.remove(tmp_path / "_marshal.so")
    build.build_marshal()
    assert len(calls) == 5
