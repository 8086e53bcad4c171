"""The package where the attention calls' native binding is missing or cannot be built (CPU)."""
import importlib.util
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2606_10493_amd")


def test_the_other_calls_work_without_the_binding(tmp_path):
    """An import, a host call of the FFN's and of the attention's C ABI; the attention calls say what is missing."""
    copy = tmp_path / "paper_2606_10493_amd"
    copy.mkdir()
    for name in os.listdir(PKG):
        if name.endswith(".py") or name == "libmoe.so":
            shutil.copy(os.path.join(PKG, name), copy / name)
    code = """
import paper_2606_10493_amd as moe
assert moe.__file__.startswith(%r), moe.__file__
assert moe.moe_router_workspace(1, 7168, 256) >= 0
d = moe.MoeAttnDims(8, 2, 128)
assert moe.moe_attn_prefill_workspace(d, 1, 509, 8701) > 0
for call, n in ((moe.moe_rope, 8), (moe.moe_attn_prefill, 9)):
    try:
        call(d, *[None] * (n - 1))
    except ImportError as e:
        assert "_binding.so" in str(e) and "build.py" in str(e), e
    else:
        raise AssertionError("no ImportError")
print("fine")
""" % str(tmp_path)
    res = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert res.returncode == 0 and "fine" in res.stdout, res.stdout + res.stderr


@pytest.fixture()
def build(tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("_build_under_test", os.path.join(PKG, "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    monkeypatch.setattr(mod, "BINDING", str(tmp_path / "_binding.so"))
    return mod


def test_a_missing_compiler_leaves_the_library_built(build, monkeypatch, capsys):
    """No C++ compiler or no Python headers: a warning, and no binding of an earlier build that might not fit."""
    for name, value in (("CXX", None), ("CXX", "/nowhere/g++"), ("PYTHON_INCLUDE", "/nowhere/include")):
        open(build.BINDING, "w").close()
        with monkeypatch.context() as m:
            m.setattr(build, name, value)
            assert build.build_binding() is False
        assert not os.path.exists(build.BINDING)
        assert "_binding.so is not built" in capsys.readouterr().err


def test_a_source_that_does_not_compile_is_an_error(build, monkeypatch, tmp_path):
    (tmp_path / "binding.cpp").write_text("#error broken\n")
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    with pytest.raises(RuntimeError, match="binding.cpp failed"):
        build.build_binding()
    assert not os.path.exists(build.BINDING)
