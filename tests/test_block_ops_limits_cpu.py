"""Host side of the operators around the self-attention: calls that the documentation rules out, and what the library and its
Python entry points need to be built and loaded.  No GPU needed."""
import ctypes
import os
import subprocess

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
