"""The C++ module of the calls on real-valued tensors: what works without it."""
import os
import shutil
import subprocess
import sys

import pytest

import paper_2202_05239_b200 as package

HERE = os.path.dirname(os.path.abspath(package.__file__))


@pytest.mark.parametrize("module", [None, b"no shared object"])
def test_fixed_point_path_without_the_module(tmp_path, module):
    """Without the module, or with one that does not load, the package imports, and the calls that need the module say so."""
    copy = tmp_path / "copied"
    copy.mkdir()
    os.symlink(os.path.join(HERE, "libf8net.so"), copy / "libf8net.so")
    for name in ("__init__.py", "api.py", "synth.py"):
        shutil.copy(os.path.join(HERE, name), copy / name)
    if module is not None:
        (copy / "_f8torch.so").write_bytes(module)
    code = (
        "import torch\n"
        "from copied import api\n"
        "assert api._lib.f8_linear_fixed and api.Net\n"
        "for call in (api.f8_linear_scaled, api.f8_quantize_rows, api.f8_norm_quantize, api.f8_token_logprobs):\n"
        "    try:\n"
        "        call(*[torch.zeros(1, 1)] * (5 if call is api.f8_linear_scaled else 1))\n"
        "    except ImportError as e:\n"
        "        assert 'copied.build' in str(e), e\n"
        "    else:\n"
        "        raise AssertionError(call)\n")
    run = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env={**os.environ, "PYTHONPATH": str(tmp_path)}, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


def test_module_is_built_again_for_another_torch_or_python(monkeypatch):
    """A module made for another torch or another Python does not load, however new its file is."""
    from paper_2202_05239_b200 import api, build
    assert build.binding_is_current()
    assert build.binding_made_for() in api._f8torch.__doc__
    import torch
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", torch.__version__ + "1")
        assert not build.binding_is_current()
    with monkeypatch.context() as m:
        m.setattr(build.sysconfig, "get_config_var", lambda name: "cpython-399-none")
        assert not build.binding_is_current()
    with monkeypatch.context() as m:
        m.setattr(build, "BINDING", build.BINDING + ".none")
        assert not build.binding_is_current()
    assert build.binding_is_current()
