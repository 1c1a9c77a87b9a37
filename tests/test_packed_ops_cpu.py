"""Host side of the operators for packed requests: every refusal comes before any CUDA call, calls without rows are fine without a
device, the entry points look at their tensors.  No GPU needed."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return dt.lib()


P = 2 ** 24       # stands for a device pointer; a refused call never reads it
INV, UNS = dt.DT_ERR_INVALID_ARG, dt.DT_ERR_UNSUPPORTED


def s4(b=4096, l=128, h=64, d=1):
    return (C.c_int64 * 4)(b, l, h, d)


def adapter_call(lib, x=P, w=2 * P, bias=None, a=3 * P, b=4 * P, scales=None, starts=5 * P, which=6 * P, y=7 * P, ws=8 * P, ws_bytes=2 ** 20, **kw):
    c = dict(dtype=0, bias_dtype=0, rows=20, K=64, N=72, rank=16, adapters=3, segments=2, x_stride=64, w_stride=64, y_stride=72)
    c.update(kw)
    cfg = dt.dt_adapter_config(*[c[n] for n, _ in dt.dt_adapter_config._fields_])
    return lib.dt_adapter_linear(C.byref(cfg), x, w, bias, a, b, scales, starts, which, y, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNS), (dict(dtype=1), UNS), (dict(bias_dtype=1), UNS), (dict(rows=-1), INV), (dict(K=0), INV), (dict(N=0), INV), (dict(rank=-8), INV),
    (dict(adapters=-1), INV), (dict(segments=-1), INV), (dict(rows=2 ** 30 + 1), UNS), (dict(K=2 ** 20 + 8), UNS), (dict(N=2 ** 20 + 8), UNS),
    (dict(adapters=65536), UNS), (dict(segments=2 ** 20 + 1), UNS), (dict(K=60), UNS), (dict(N=70), UNS), (dict(rank=0), UNS), (dict(rank=12), UNS),
    (dict(rank=136), UNS), (dict(x=None), INV), (dict(w=None), INV), (dict(y=None), INV), (dict(x=P + 8), INV), (dict(w=P + 2), INV), (dict(y=P + 8), INV),
    (dict(x_stride=56), INV), (dict(x_stride=68), INV), (dict(w_stride=56), INV), (dict(w_stride=68), INV), (dict(y_stride=64), INV), (dict(y_stride=76), INV),
    (dict(y=P), INV), (dict(y=2 * P), INV), (dict(bias=P + 1), INV), (dict(bias=P + 2, bias_dtype=2), INV), (dict(a=None), INV), (dict(b=None), INV),
    (dict(a=P + 8), INV), (dict(starts=None), INV), (dict(which=None), INV), (dict(starts=P + 2), INV), (dict(scales=P + 2), INV), (dict(ws=None), INV),
    (dict(ws=P + 8), INV), (dict(ws_bytes=20 * 16 * 2 - 1), INV), (dict(rows=16, ws_bytes=16 * 16 * 4 - 1), INV),
])
def test_adapter_refusals(lib, kw, status):
    assert adapter_call(lib, **kw) == status
    assert lib.dt_last_error(None)


def packed_call(lib, q=P, qs=None, k=2 * P, ks=None, v=3 * P, vs=None, q_starts=None, k_starts=None, q_lens=None, key_lens=None, prefix=None, table=None,
                slopes=None, o=4 * P, os=None, lse=None, **kw):
    c = dict(dtype=0, B=2, Lq=3, Lk=5, H=2, H_kv=2, D=64, docs=0, causal=0, bias_far=0, softmax_scale=0.1, softcap=0.0)
    c.update(kw)
    cfg = dt.dt_packed_config(*[c[n] for n, _ in dt.dt_packed_config._fields_])
    z = lambda s: s4() if s is None else s  # noqa: E731
    return lib.dt_packed_attn(C.byref(cfg), q, z(qs), k, z(ks), v, z(vs), q_starts, k_starts, q_lens, key_lens, prefix, table, slopes, o, z(os), lse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNS), (dict(D=96), UNS), (dict(B=-1), INV), (dict(Lq=-1), INV), (dict(Lk=-1), INV), (dict(H=0), INV), (dict(H_kv=0), INV), (dict(docs=-1), INV),
    (dict(H=3), INV), (dict(B=40000), UNS), (dict(Lk=2 ** 24 + 1), UNS), (dict(Lq=2 ** 30), UNS), (dict(docs=65537, q_starts=P, k_starts=P), UNS),
    (dict(softmax_scale=0.0), INV), (dict(softmax_scale=math.nan), INV), (dict(softmax_scale=math.inf), INV), (dict(softcap=-1.0), INV),
    (dict(softcap=math.nan), INV), (dict(softcap=math.inf), INV), (dict(softcap=1e-39, softmax_scale=1e-39), INV), (dict(softcap=1e30, softmax_scale=1e-20), INV),
    (dict(softcap=1e-30, softmax_scale=1e20), INV), (dict(table=P, slopes=P), INV), (dict(table=P, bias_far=-1), INV), (dict(table=P, bias_far=513), UNS),
    (dict(docs=2), INV), (dict(docs=2, q_starts=P), INV), (dict(q_starts=P, k_starts=P), INV), (dict(docs=2, q_starts=P, k_starts=P, q_lens=P), INV),
    (dict(docs=2, q_starts=P, k_starts=P, key_lens=P), INV), (dict(q=None), INV), (dict(o=None), INV), (dict(k=None), INV), (dict(v=None), INV),
    (dict(q=P + 8), INV), (dict(k=P + 2), INV), (dict(qs=s4(d=2)), INV), (dict(ks=s4(h=60)), INV), (dict(vs=s4(l=-128)), INV), (dict(os=s4(b=0)), INV),
    (dict(os=s4(l=0)), INV), (dict(os=s4(h=32)), INV), (dict(o=2 * P), INV), (dict(o=3 * P), INV), (dict(o=P, os=s4(l=256)), INV),
    (dict(key_lens=P + 2), INV), (dict(prefix=P + 1), INV), (dict(lse=P + 2), INV), (dict(slopes=P + 2), INV),
])
def test_packed_refusals(lib, kw, status):
    assert packed_call(lib, **kw) == status
    assert lib.dt_last_error(None)


def test_calls_without_rows_are_fine_without_a_device(lib):
    assert adapter_call(lib, rows=0) == dt.DT_OK and adapter_call(lib, rows=0, x=None, y=None, ws=None, ws_bytes=0) == dt.DT_OK
    assert packed_call(lib, B=0) == dt.DT_OK and packed_call(lib, Lq=0, q=None, o=None) == dt.DT_OK
    assert lib.dt_adapter_linear(None, *[None] * 10, 0, None) == INV and lib.dt_packed_attn(None, *[None] * 17) == INV


@pytest.mark.parametrize("rows,rank,want", [(0, 0, 0), (16, 8, 16 * 16 * 4), (17, 8, 17 * 16 * 2), (1000, 72, 1000 * 80 * 2), (3, 128, 3 * 128 * 4)])
def test_workspace(lib, rows, rank, want):
    assert dt.dt_adapter_workspace_bytes(rows, rank) == want


@pytest.mark.parametrize("rows,rank", [(-1, 8), (2 ** 30 + 1, 8), (5, -1), (5, 129)])
def test_workspace_refusals(lib, rows, rank):
    with pytest.raises(dt.DitangoError):
        dt.dt_adapter_workspace_bytes(rows, rank)
    assert lib.dt_adapter_workspace_bytes(5, 8, None) == INV


def test_entry_points_look_at_their_tensors(lib):
    """Host tensors, and what is no tensor of torch's."""
    x, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(72, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        dt.dt_adapter_linear(x, w, torch.zeros(3, 72, dtype=torch.bfloat16), None, None, None, None, None)
    q = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        dt.dt_packed_attn(q, q, q, q.clone(), 0.1)
    with pytest.raises(AssertionError):
        dt.dt_packed_attn(q.to_sparse(), q, q, q, 0.1)
    with pytest.raises(AssertionError):
        dt.dt_packed_attn(torch.zeros([1] * 9), q, q, q, 0.1)
    with pytest.raises(AttributeError):
        dt.dt_packed_attn([q], q, q, q, 0.1)
    with pytest.raises(TypeError):
        dt.dt_packed_attn(q, q, q, q)
    with pytest.raises(TypeError):
        dt.dt_packed_attn(q, q, q, q, 0.1, window=3)
    with pytest.raises(TypeError):
        dt.dt_adapter_linear(x, w, x, None, None, None, None, None, x=x)


def test_tensors_of_other_classes_are_seen_alike(lib):
    """Parameters and subclasses go by their Python attributes, torch's own by its headers: the same shapes and strides."""
    class Sub(torch.Tensor):
        pass
    base = torch.zeros(4, 6, 40)[:, 1:5, 8:32]
    want = dt._norm_rows([base])
    assert want == (4, 4, [(240, 40)])
    assert dt._norm_rows([base.as_subclass(Sub)]) == want and dt._norm_rows([torch.nn.Parameter(base)]) == want


def test_kernels_that_begin_early_promise_nothing_about_what_they_read():
    """A kernel that is resident while the launch before may still write reads nothing by ld.global.nc (__ldg), and by no cached-load
    intrinsic that the compiler may move ahead of the wait."""
    csrc = os.path.join(os.path.dirname(build.__file__), "csrc")
    early = set()
    for f in sorted(os.listdir(csrc)):
        if f.endswith((".cu", ".cuh", ".h")):
            text = re.sub(r"//.*", "", open(os.path.join(csrc, f)).read())
            if re.search(r"wait_for_previous\(\)|AdapterParams|PackedParams", text):
                early.add(f)
                assert not re.search(r"\b__ld(g|cg|cs|ca|lu|cv)\s*\(|ld\.global\.nc|__restrict__", text), f
    assert early >= {"adapter_linear.cu", "adapter_linear.h", "adapter_tiles.cu", "packed_attn.cu", "packed_attn.h", "packed_tiles.cu", "tile_wait.cuh"}


@pytest.mark.parametrize("kw", [dict(softmax_scale=3e38), dict(softmax_scale=3.4e38, softcap=3.4e38), dict(softmax_scale=100.0, softcap=3e38)])
def test_scales_and_caps_that_base_2_does_not_hold_are_refused(lib, kw):
    """Logits are kept in base 2, where a factor beyond 2^127.5 is infinite and every row would be NaN."""
    assert packed_call(lib, **kw) == INV
    assert b"base 2" in lib.dt_last_error(None)
    ok = {k: 2.0 ** 127 for k in kw}
    ok["Lq"] = 0
    assert packed_call(lib, **ok) == dt.DT_OK
