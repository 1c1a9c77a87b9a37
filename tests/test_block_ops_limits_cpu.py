"""Host side of the operators around the self-attention: calls that the documentation rules out, and what the library and its
Python entry points need to be built and loaded.  No GPU needed."""
import ctypes
import os
import subprocess
import sysconfig

import pytest

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build
from tests.test_block_ops_cpu import norm_call


@pytest.fixture(scope="module")
def lib():
    build.build()
    return dt.lib()


def test_selftest_refuses_long_limits(lib):
    assert lib.dt_selftest_ops_timeout(1000001, None) == dt.DT_ERR_INVALID_ARG and lib.dt_last_error(None)


@pytest.mark.parametrize("kw", [
    dict(y_strides=(512, 512)), dict(y_strides=(1024, 512)), dict(y_strides=(512, 520)), dict(y_strides=(1528, 512)),
    dict(residual_out_strides=(512, 512)), dict(residual_out_strides=(1024, 512)), dict(residual_out_strides=(512, 1016)),
    dict(n0=3, n1=2, y_strides=(512, 1024)), dict(n0=2 ** 15, n1=2 ** 15, y_strides=(2 ** 24 - 8, 512)),
    # in the residual's place, with the residual's own (overlapping) strides
    dict(ro=2 ** 24, r=2 ** 24, residual_strides=(1024, 512), residual_out_strides=(1024, 512)),
])
def test_norm_refuses_outputs_whose_rows_meet_across_the_two_strides(lib, kw):
    assert norm_call(lib, **kw) == dt.DT_ERR_INVALID_ARG
    assert b"overlap" in lib.dt_last_error(None)


def test_rotation_and_norm_stand_without_the_attention_kernels(lib, tmp_path):
    """Nothing of dt_rope and dt_add_rmsnorm, their first call included, goes through the cross attention's files."""
    out = str(tmp_path / "part.so")
    subprocess.run([build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xptxas", "-O1", "-shared", "-Xcompiler", "-fPIC",
                    "-Xlinker", "-zdefs", "--threads", "3", "-o", out] + [os.path.join(build.CSRC, f) for f in ("ops_api.cu", "rope.cu", "add_rmsnorm.cu")],
                   check=True)
    part = ctypes.CDLL(out)
    assert part.dt_rope(None, *[None] * 12) == dt.DT_ERR_INVALID_ARG and part.dt_add_rmsnorm(None, *[None] * 7) == dt.DT_ERR_INVALID_ARG


@pytest.fixture()
def elsewhere(monkeypatch, tmp_path):
    """build() into a folder of its own, with nvcc replaced by something that leaves a file, and the commands as they run."""
    ran, real = [], subprocess.run

    def run(cmd, **kw):
        ran.append(cmd[0])
        if cmd[0] == build.NVCC:
            open(cmd[cmd.index("-o") + 1], "w").close()
            return None
        return real(cmd, stderr=subprocess.DEVNULL, **kw)
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libditango.so"))
    monkeypatch.setattr(build, "OPS_LIB", str(tmp_path / "ops.so"))
    return ran


@pytest.mark.parametrize("without", ["headers", "compiler"])
def test_the_library_is_built_without_what_the_python_entry_points_need(elsewhere, monkeypatch, tmp_path, without):
    if without == "headers":
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda *a, **k: {"include": str(tmp_path)})
    else:
        monkeypatch.setenv("CC", "no-such-compiler")
    with pytest.warns(UserWarning, match="entry points"):
        assert build.build(force=True) == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.OPS_LIB) and elsewhere == [build.NVCC]


def test_entry_points_that_do_not_compile_are_an_error_behind_the_library(elsewhere, monkeypatch, tmp_path):
    (tmp_path / "broken.c").write_text("#error\n")
    monkeypatch.setattr(build, "OPS_SOURCE", str(tmp_path / "broken.c"))
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert os.path.exists(build.LIB) and not os.path.exists(build.OPS_LIB)


def test_the_whole_build_and_nothing_twice(elsewhere):
    build.build()
    assert os.path.exists(build.LIB) and os.path.exists(build.OPS_LIB) and len(elsewhere) == 2
    build.build()
    assert len(elsewhere) == 2


def test_the_module_of_entry_points_is_named_for_its_interpreter(lib):
    """Two Python versions on one tree build and load a module each."""
    suffix = sysconfig.get_config_var("EXT_SUFFIX")
    assert suffix and build.OPS_LIB.endswith("_ditango_ops" + suffix) and dt.OPS_PATH == build.OPS_LIB and os.path.exists(build.OPS_LIB)
    assert dt.dt_rope.__module__ == "_ditango_ops"
