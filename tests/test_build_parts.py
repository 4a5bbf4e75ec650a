"""What the build needs torch for, and what not.  No GPU is needed."""
import glob
import os
import shutil
import subprocess
import sys
import sysconfig

from paper_2210_03858_b200 import build as bcq_build

ROOT = os.path.dirname(bcq_build.HERE)


def test_the_library_is_built_without_torch(tmp_path):
    # a compiler that only leaves the files it is asked for: what counts is that everything but the torch binding is built
    package = tmp_path / "paper_2210_03858_b200"
    package.mkdir()
    for name in ("__init__.py", "build.py", "synth.py"):
        shutil.copy(os.path.join(bcq_build.HERE, name), package)
    shutil.copytree(bcq_build.CSRC, package / "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    nvcc = tmp_path / "nvcc"
    nvcc.write_text('#!/bin/sh\nwhile [ $# -gt 0 ]; do if [ "$1" = -o ]; then : > "$2"; fi; shift; done\n')
    nvcc.chmod(0o755)
    code = """if True:
        import sys
        sys.modules["torch"] = None    # no such module
        from paper_2210_03858_b200 import build
        assert build.tensor_call_path() is None
        print(build.build_library())
        assert not build.is_stale()
    """
    r = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env=dict(os.environ, NVCC=str(nvcc), PYTHONPATH=str(tmp_path)), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert sorted(os.path.basename(p) for p in glob.glob(str(package / "*.so"))) == \
        ["_bcq_call" + sysconfig.get_config_var("EXT_SUFFIX"), "libbcq_b200.so"]


def test_the_torch_binding_belongs_to_one_version_of_torch(monkeypatch):
    bcq_build.build_library()
    path = bcq_build.tensor_call_path()
    root, version, cuda = bcq_build._torch()
    assert version in os.path.basename(path) and os.path.exists(path) and not bcq_build.is_stale()
    assert glob.glob(os.path.join(bcq_build.HERE, "_tensor_call*.so")) == [path]
    monkeypatch.setattr(bcq_build, "_torch", lambda: (root, version + ".1", cuda))
    assert bcq_build.is_stale() and not os.path.exists(bcq_build.tensor_call_path())
    monkeypatch.setattr(bcq_build, "_torch", lambda: (root, version, None))  # without CUDA there is nothing to bind
    assert bcq_build.tensor_call_path() is None and not bcq_build.is_stale()


def test_the_version_is_that_of_the_torch_that_is_imported():
    import pytest
    torch = pytest.importorskip("torch")
    root, version, cuda = bcq_build._torch()
    assert os.path.samefile(root, os.path.dirname(torch.__file__)) and version == str(torch.__version__) and cuda == torch.version.cuda
