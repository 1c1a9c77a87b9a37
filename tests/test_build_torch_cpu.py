"""The module of Python entry points is built against one torch: what the build and the binding do without torch, without its CUDA part, and
with another one than it is built for.  No GPU needed."""
import os
import subprocess
import types

import pytest

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build


@pytest.fixture()
def elsewhere(monkeypatch, tmp_path):
    """build() into a folder of its own, with compilers replaced by something that leaves a file, and the commands as they run."""
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libditango.so"))
    monkeypatch.setattr(build, "OPS_LIB", str(tmp_path / "ops.so"))
    return ran


def other_torch(monkeypatch, tmp_path, version="2.12.0a0+git1234567", without=""):
    """A folder that looks like a torch of that version."""
    folder = tmp_path / "torch"
    files = ["include/torch/csrc/autograd/python_variable.h", "include/c10/cuda/CUDAStream.h"] + [f"lib/lib{n}.so" for n in build.OPS_LIBS]
    for f in files:
        if f != without:
            (folder / f).parent.mkdir(parents=True, exist_ok=True)
            (folder / f).touch()
    (folder / "version.py").write_text(f"__all__ = []\n__version__ = '{version}'\ndebug = False\n")
    spec = types.SimpleNamespace(submodule_search_locations=[str(folder)])
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: spec)


def test_without_torch_the_library_is_built_alone(elsewhere, monkeypatch):
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    with pytest.warns(UserWarning, match="entry points.*torch"):
        assert build.build(force=True) == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.OPS_LIB) and len(elsewhere) == 1


@pytest.mark.parametrize("without", ["include/c10/cuda/CUDAStream.h", "lib/libc10_cuda.so", "include/torch/csrc/autograd/python_variable.h"])
def test_without_a_part_of_torch_the_library_is_built_alone(elsewhere, monkeypatch, tmp_path, without):
    other_torch(monkeypatch, tmp_path, without=without)
    with pytest.warns(UserWarning, match="entry points.*" + os.path.basename(without)):
        build.build(force=True)
    assert os.path.exists(build.LIB) and not os.path.exists(build.OPS_LIB) and len(elsewhere) == 1


def test_another_torch_is_built_for_anew(elsewhere, monkeypatch, tmp_path):
    build.build()
    build.build()
    assert len(elsewhere) == 2
    for n, version in enumerate(("2.12.0a0+git1234567", "2.12.0.dev20270101+cu130", "2.12.0")):
        other_torch(monkeypatch, tmp_path, version)
        build.build()
        assert len(elsewhere) == 3 + n and f'-DBUILT_FOR_TORCH="{version}"' in elsewhere[-1]
        build.build()
        assert len(elsewhere) == 3 + n


def test_a_module_that_says_nothing_of_its_torch_is_built_anew(elsewhere):
    build.build()
    os.remove(build.OPS_LIB + ".torch")
    build.build()
    assert len(elsewhere) == 3


def test_the_binding_goes_by_the_whole_version(monkeypatch):
    build.build()
    import torch
    dt._load_ops()
    for version in ("2.11.0a0+git70d99e9", torch.__version__.split("+")[0] + "+of_another_build"):
        monkeypatch.setattr(torch, "__version__", version)
        with pytest.raises(ImportError, match="built for torch"):
            dt._load_ops()


@pytest.mark.parametrize("version", ["2.11.0a0+git70d99e9", "2.12.0.dev20270101+cu130"])
def test_a_torch_of_any_version_is_served_once_built_for(monkeypatch, tmp_path, version):
    """Pre-releases and builds from source, whose headers know the release alone."""
    import torch
    folder = tmp_path / "torch"
    folder.mkdir()
    real = os.path.dirname(torch.__file__)
    for part in ("include", "lib"):
        os.symlink(os.path.join(real, part), folder / part)
    (folder / "version.py").write_text(f"__version__ = '{version}'\n")
    build.build()
    monkeypatch.setattr(build, "OPS_LIB", str(tmp_path / "_ditango_ops.so"))
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: types.SimpleNamespace(submodule_search_locations=[str(folder)]))
    build._build_ops(False)
    monkeypatch.undo()
    # (in a process of its own: a module of C is loaded once)
    code = ("import torch\nfrom paper_2607_15650_b200 import binding as dt\n"
            f"torch.__version__, dt.OPS_PATH = {version!r}, {str(tmp_path / '_ditango_ops.so')!r}\n"
            "assert dt._norm_rows([torch.zeros(4, 8)]) is not None and dt.dt_rope\n")
    subprocess.run([os.sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(build.__file__))))
