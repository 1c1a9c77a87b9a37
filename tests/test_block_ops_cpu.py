"""Host side of the operators around the self-attention: every refusal comes before any CUDA call, the frequencies follow
their published formulas, and row strides collapse as the binding says.  No GPU needed."""
import ctypes as C
import math

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return dt.lib()


P = 4096          # stands for a device pointer; a refused call never reads it
INV, UNS = dt.DT_ERR_INVALID_ARG, dt.DT_ERR_UNSUPPORTED


def s4(b=4096, l=128, h=64, d=1):
    return (C.c_int64 * 4)(b, l, h, d)


def rope_call(lib, q=P, qs=None, qo=P, qos=None, k=P + 2 ** 20, ks=None, ko=P + 2 ** 20, kos=None, f=P, pos=P, ps=(0, 1, 0), **kw):
    c = dict(dtype=0, B=2, L=3, H=2, H_k=2, D=64, rotary_dim=64, layout=0, axes=1, transpose=0, attn_factor=1.0)
    c.update(kw)
    cfg = dt.dt_rope_config(*[c[n] for n, _ in dt.dt_rope_config._fields_])
    z = lambda s: s4() if s is None else s  # noqa: E731
    return lib.dt_rope(C.byref(cfg), q, z(qs), qo, z(qos), k, z(ks), ko, z(kos), f, pos, (C.c_int64 * 3)(*ps) if ps else None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNS), (dict(layout=2), UNS), (dict(B=-1), INV), (dict(L=-1), INV), (dict(H=0), INV), (dict(H_k=-1), INV),
    (dict(D=60, rotary_dim=60), UNS), (dict(D=264), UNS), (dict(D=0), INV), (dict(rotary_dim=63), INV), (dict(rotary_dim=0), INV),
    (dict(rotary_dim=66), INV), (dict(axes=0), UNS), (dict(axes=5), UNS), (dict(attn_factor=math.inf), INV), (dict(attn_factor=math.nan), INV),
    (dict(H=65536), UNS), (dict(B=65536, L=65536), UNS),
    (dict(q=None), INV), (dict(qo=None), INV), (dict(k=None), INV), (dict(ko=None), INV), (dict(f=None), INV), (dict(f=P + 4), INV),
    (dict(q=P + 8), INV), (dict(ko=P + 2), INV), (dict(qs=s4(d=2)), INV), (dict(qs=s4(l=-128)), INV), (dict(qs=s4(h=60)), INV),
    (dict(qos=s4(b=0)), INV), (dict(kos=s4(l=0)), INV), (dict(ks=s4(l=0)), INV), (dict(qos=s4(l=256)), INV), (dict(kos=s4(b=8192)), INV),
    (dict(pos=None, axes=2), INV), (dict(ps=None), INV), (dict(pos=P + 2), INV),
    (dict(qo=P + 2 ** 20, q=P + 2 ** 21), INV), (dict(ko=P, q=P + 2 ** 21), INV), (dict(ko=P), INV),
    (dict(qo=P + 64, qos=s4(h=32)), INV), (dict(qo=P + 64, qos=s4(l=64)), INV), (dict(qo=P + 64, qos=s4(b=320)), INV),
])
def test_rope_refusals(lib, kw, status):
    assert rope_call(lib, **kw) == status
    assert lib.dt_last_error(None)


def test_empty_calls_are_fine_without_a_device(lib):
    assert rope_call(lib, B=0) == dt.DT_OK and rope_call(lib, L=0, q=None) == dt.DT_OK
    assert norm_call(lib, n0=0) == dt.DT_OK and norm_call(lib, n1=0, x=None, y=None) == dt.DT_OK
    assert cross_call(lib, B=0) == dt.DT_OK and cross_call(lib, Lq=0, q=None, o=None) == dt.DT_OK
    assert lib.dt_rope(None, *[None] * 12) == INV
    assert lib.dt_add_rmsnorm(None, *[None] * 7) == INV
    assert lib.dt_cross_attn(None, None, None, None, None, None, None, None, None, 0, None, None, None, None) == INV


def norm_call(lib, x=P, w=P, r=P + 2 ** 20, ro=P + 2 ** 20, y=P + 2 ** 21, sc=P, **kw):
    c = dict(dtype=0, weight_dtype=2, residual_dtype=2, out_kind=1, n0=2, n1=3, width=512, scale_group=0, x_strides=(1536, 512),
             residual_strides=(1536, 512), residual_out_strides=(1536, 512), y_strides=(1536, 512), eps=1e-6)
    c.update(kw)
    pair = C.c_int64 * 2
    cfg = dt.dt_norm_config(*[pair(*c[n]) if isinstance(c[n], tuple) else c[n] for n, _ in dt.dt_norm_config._fields_])
    return lib.dt_add_rmsnorm(C.byref(cfg), x, w, r, ro, y, sc, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNS), (dict(dtype=9), UNS), (dict(weight_dtype=1), UNS), (dict(residual_dtype=1), UNS), (dict(out_kind=2), UNS),
    (dict(n0=-1), INV), (dict(n1=-2), INV), (dict(width=0), INV), (dict(width=12), UNS), (dict(width=16392), UNS),
    (dict(eps=-1e-6), INV), (dict(eps=math.nan), INV), (dict(eps=math.inf), INV), (dict(scale_group=16), UNS), (dict(scale_group=48), UNS),
    (dict(scale_group=128, width=576), INV), (dict(n0=2 ** 20, n1=2 ** 20), UNS),
    (dict(x=None), INV), (dict(y=None), INV), (dict(sc=None), INV), (dict(r=None), INV), (dict(ro=None), INV),
    (dict(x_strides=(1536, 516)), INV), (dict(x_strides=(-1536, 512)), INV), (dict(y_strides=(1536, 0)), INV), (dict(y_strides=(1536, 504)), INV),
    (dict(residual_out_strides=(0, 512)), INV), (dict(residual_strides=(1, 512)), INV),
    (dict(x=P + 8), INV), (dict(w=P + 4), INV), (dict(y=P + 4), INV), (dict(y=P + 8, out_kind=0), INV), (dict(sc=P + 2), INV), (dict(ro=P + 8), INV),
    (dict(y=P), INV), (dict(y=P, out_kind=0, y_strides=(1536, 520)), INV), (dict(y=P + 2 ** 20), INV), (dict(ro=P), INV),
    (dict(residual_out_strides=(4096, 512)), INV), (dict(ro=P, residual_dtype=0, residual_out_strides=(1600, 512)), INV),
])
def test_norm_refusals(lib, kw, status):
    assert norm_call(lib, **kw) == status
    assert lib.dt_last_error(None)


def cross_call(lib, q=P, qs=None, k=P + 2 ** 20, ks=None, v=P + 2 ** 20, vs=None, lens=None, mask=None, ms=0, o=P, os=None, lse=None, **kw):
    c = dict(dtype=0, B=2, Lq=3, Lk=5, H=4, H_kv=2, D=64, softmax_scale=0.125)
    c.update(kw)
    cfg = dt.dt_cross_config(*[c[n] for n, _ in dt.dt_cross_config._fields_])
    z = lambda s: s4(l=256) if s is None else s  # noqa: E731
    return lib.dt_cross_attn(C.byref(cfg), q, z(qs), k, z(ks), v, z(vs), lens, mask, ms, o, z(os), lse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNS), (dict(D=96), UNS), (dict(D=256), UNS), (dict(B=-1), INV), (dict(Lq=-1), INV), (dict(Lk=-1), INV), (dict(H=0), INV),
    (dict(H_kv=0), INV), (dict(H_kv=3), INV), (dict(B=20000, H=4), UNS), (dict(Lq=2 ** 29), UNS), (dict(Lk=2 ** 30), UNS),
    (dict(softmax_scale=0.0), INV), (dict(softmax_scale=-1.0), INV), (dict(softmax_scale=math.inf), INV), (dict(softmax_scale=math.nan), INV),
    (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(o=None), INV), (dict(q=P + 8), INV), (dict(o=P + 2), INV),
    (dict(ks=s4(l=0)), INV), (dict(ks=s4(h=0)), INV), (dict(vs=s4(d=2)), INV), (dict(vs=s4(l=260)), INV), (dict(os=s4(b=0)), INV), (dict(qs=s4(l=-256)), INV),
    (dict(mask=P, ms=4), INV), (dict(mask=P, ms=-5), INV), (dict(lens=P + 2), INV), (dict(lse=P + 1), INV),
    (dict(Lk=2 ** 26 + 1), UNS), (dict(o=P + 2 ** 20), INV), (dict(os=s4(l=512)), INV), (dict(o=P + 64, os=s4(l=128)), INV),
])
def test_cross_refusals(lib, kw, status):
    assert cross_call(lib, **kw) == status
    assert lib.dt_last_error(None)


def test_frequencies_follow_their_formulas(lib):
    r, base, s, trained = 64, 10000.0, 8.0, 4096
    plain, m = dt.dt_rope_freqs(r, base)
    i = torch.arange(r // 2, dtype=torch.float64)
    want = base ** (-2 * i / r)
    tight = dict(rtol=1e-13, atol=0.0)
    torch.testing.assert_close(plain, want, **tight)
    assert m == 1.0
    f, m = dt.dt_rope_freqs(r, base, dt.DT_ROPE_LINEAR, s)
    torch.testing.assert_close(f, want / s, **tight)
    f, m = dt.dt_rope_freqs(r, base, dt.DT_ROPE_BASE, s)
    assert abs(f[0] - 1) < 1e-15 and abs(f[-1] / (want[-1] / s) - 1) < 1e-13      # the fastest stays, the slowest is divided
    torch.testing.assert_close(f, (base * s ** (r / (r - 2))) ** (-2 * i / r), **tight)
    f, m = dt.dt_rope_freqs(r, base, dt.DT_ROPE_PARTS, s, trained, 32.0, 1.0)
    turns = trained * want / (2 * math.pi)
    assert abs(m - (0.1 * math.log(s) + 1)) < 1e-6
    assert (f[turns >= 32] == plain[turns >= 32]).all() and (turns >= 32).any()
    torch.testing.assert_close(f[turns <= 1], want[turns <= 1] / s, **tight)
    between = (turns > 1) & (turns < 32)
    keep = ((turns - 1) / 31)[between]
    torch.testing.assert_close(f[between], want[between] * (keep + (1 - keep) / s), **tight)
    assert dt.dt_rope_freqs(2)[0].tolist() == [1.0] and dt.dt_rope_freqs(2, kind=dt.DT_ROPE_BASE, factor=4.0)[0].tolist() == [1.0]
    grid = dt.dt_rope_grid_freqs((44, 42, 42))
    assert grid.shape == (3, 64) and (grid != 0).sum(1).tolist() == [22, 21, 21] and ((grid != 0).sum(0) == 1).all()
    assert grid[1, 22] == 1.0 and grid[1, 43] == 0.0


@pytest.mark.parametrize("kw", [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=8, base=1.0), dict(rotary_dim=8, base=math.inf),
                                dict(rotary_dim=8, kind=1, factor=0.5), dict(rotary_dim=8, kind=2, factor=math.nan), dict(rotary_dim=8, kind=4),
                                dict(rotary_dim=8, kind=3, factor=2.0), dict(rotary_dim=8, kind=3, factor=2.0, trained_length=9, turns_fast=1.0)])
def test_frequency_refusals(lib, kw):
    with pytest.raises(dt.DitangoError):
        dt.dt_rope_freqs(**kw)


def test_rows_of_views_collapse_to_two_strides(lib):
    x = torch.empty(2, 5, 9, 64)
    assert dt._norm_rows([x])[:2] == (1, 90)
    assert dt._norm_rows([x[:, :, :3], torch.empty(2, 5, 3, 64)]) == (10, 3, [(9 * 64, 64), (3 * 64, 64)])
    assert dt._norm_rows([x[:, :1, 0], x[:, :1, 1]]) == (1, 2, [(0, 45 * 64)] * 2)
    with pytest.raises(AssertionError):
        dt._norm_rows([x[:, :4, :3]])          # three strides
    with pytest.raises(AssertionError):
        dt._norm_rows([x[..., ::2]])


def test_the_binding_refuses_what_it_can_see_without_a_device(lib):
    x = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16)
    f = torch.ones((1, 32), dtype=torch.float64)
    with pytest.raises(AssertionError):
        dt.dt_rope(x, None, x, None, f)                       # not on a GPU
    with pytest.raises(AssertionError):
        dt.dt_add_rmsnorm(x, None, x, 1e-6)
    with pytest.raises(AssertionError):
        dt.dt_cross_attn(x, x, x, x, 0.1)
    for call in (lambda: dt.dt_rope(x, None, x), lambda: dt.dt_rope(x, None, x, None, f, turn=1), lambda: dt.dt_rope(x, None, x, None, f, q=x),
                 lambda: dt.dt_add_rmsnorm(*[x] * 9), lambda: dt.dt_cross_attn(x, x, x, out=x)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(AttributeError):
        dt.dt_cross_attn(1, 2, 3, 4, 0.1)
    assert "key_mask" in dt.dt_cross_attn.__doc__ and "scales" in dt.dt_add_rmsnorm.__doc__ and "freqs" in dt.dt_rope.__doc__
