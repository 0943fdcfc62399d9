"""The dense operators' short binding in C is optional: without a C compiler, Python's headers or a torch whose
DLPack header has the table of C functions, the library is built all the same, and the package imports and
takes the long way through Python and ctypes."""
import importlib.util
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def build(tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("_emb_build", os.path.join(ROOT, "paper_2110_09132_amd", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    monkeypatch.setattr(mod, "NATIVE_PATH", str(tmp_path / "_native.so"))
    return mod


def test_it_is_built_here(build):
    assert build.build_native() == build.NATIVE_PATH
    assert os.path.exists(build.NATIVE_PATH)


def test_without_a_compiler(build, monkeypatch, capsys):
    monkeypatch.setenv("CC", "/nonexistent/cc")
    open(build.NATIVE_PATH, "w").close()  # of an earlier build: it goes
    assert build.build_native() is None
    assert not os.path.exists(build.NATIVE_PATH)
    assert "not built" in capsys.readouterr().out


def test_with_a_torch_of_an_older_dlpack(build, monkeypatch, tmp_path, capsys):
    (tmp_path / "ATen").mkdir()
    (tmp_path / "ATen" / "dlpack.h").write_text("#define DLPACK_MAJOR_VERSION 1\n#define DLPACK_MINOR_VERSION 0\n"
                                                "typedef struct { void *data; } DLTensor;\n")
    monkeypatch.setattr(build, "torch_include", lambda: str(tmp_path))
    assert build.build_native() is None
    assert not os.path.exists(build.NATIVE_PATH)
    assert "not built" in capsys.readouterr().out


def test_an_error_in_the_source_is_one(build, monkeypatch, tmp_path):
    (tmp_path / "native.c").write_text("#error mistake\n")
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    with pytest.raises(subprocess.CalledProcessError):
        build.build_native()


def test_the_package_imports_without_it():
    code = ("import sys\n"
            "sys.modules['paper_2110_09132_amd._native'] = None\n"
            "import torch, paper_2110_09132_amd as emb\n"
            "from paper_2110_09132_amd import dense\n"
            "dense._stream = lambda stream: 0\n"
            "assert not dense._native.use(None, torch.Tensor, torch.nn.Parameter)\n"
            "for call in (lambda: emb.layer_norm(torch.ones(2, 3)),\n"
            "             lambda: emb.relative_bias(torch.ones(2, 3), torch.zeros(3, dtype=torch.int32), 1, 1),\n"
            "             lambda: emb.adamw_step([torch.ones(2)], [], [], [], 1e-3, 0.9, 0.999, 1e-8, 0.0, 1)):\n"
            "    try:\n"
            "        call()\n"
            "    except emb.EmbError as e:\n"
            "        assert 'CUDA' in str(e)\n"
            "    else:\n"
            "        raise AssertionError\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
