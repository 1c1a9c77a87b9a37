"""Operators around the self-attention (rotary positions, norm with the residual, cross attention) on the GPU against plain
64-bit forms, at the sizes, strides and masks where they can go wrong.  Tolerances: tests/block_ops_reference.py."""
import ctypes
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build
from tests import block_ops_reference as ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3 = torch.float8_e4m3fn
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    dt.lib()


def rnd(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def check(got, want, tol, what):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), what
    assert torch.equal(got[~fine], want[~fine]), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, (what, over.max().item(), (got - want).abs()[fine].max().item())


# ---------------------------------------------------------------------------------------------- rotary positions
def rope_case(B, L, H, Hk, D, r, half, axes, dtype, *, in_place=False, packed=False, transpose=False, factor=1.0, positions=True,
              start=0, seed=0):
    if packed:   # q and k as views of one projection's output
        x = rnd((B, L, H + 2 * Hk, D), seed, dtype)
        q, k = x[:, :, :H], x[:, :, H:H + Hk] if Hk else None
    else:
        q, k = rnd((B, L, H, D), seed, dtype), rnd((B, L, Hk, D), seed + 1, dtype) if Hk else None
    freqs = torch.zeros((axes, r // 2), dtype=torch.float64)
    for i in range(r // 2):
        freqs[i * axes // (r // 2), i] = 10000.0 ** (-2 * i / r)
    freqs = freqs.cuda()
    pos = None
    n = torch.arange(L, device="cuda")
    if positions:
        p = torch.stack([start + n * (a + 1) % 977 + (n if a == 0 else 0) for a in range(axes)], 1)
        pos = (p[None] + 7 * torch.arange(B, device="cuda")[:, None, None]).to(torch.int32)
        angle = (pos.double()[..., None] * freqs).sum(2)
    else:
        angle = (n.double()[None, :, None] * freqs).expand(B, L, r // 2)
    want = [ref.rope(t, angle, half, r, factor, transpose) for t in (q, k) if t is not None]
    if in_place:
        qo, ko = q, k
    else:
        qo, ko = torch.full_like(q, 7), torch.full_like(k, 7) if Hk else None
    dt.dt_rope(q, k, qo, ko, freqs, pos, layout=dt.DT_ROPE_HALF if half else dt.DT_ROPE_INTERLEAVED, attn_factor=factor,
               transpose=transpose)
    torch.cuda.synchronize()
    for t, (w, tol), name in zip((qo, ko), want, "qk"):
        check(t, w, tol, (name, B, L, H, Hk, D, r, half, axes, dtype))
        assert torch.equal(t[..., r:].double(), w[..., r:])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("D,r", [(64, 64), (128, 128), (128, 96), (128, 38), (64, 18), (64, 2), (8, 8), (72, 40), (256, 256)])
def test_rope_heads_and_parts(D, r, half, dtype):
    rope_case(2, 37, 3, 2, D, r, half, 1, dtype)


@pytest.mark.parametrize("B,L,H,Hk", [(1, 1, 1, 0), (1, 1, 40, 8), (3, 1, 2, 2), (2, 1000, 5, 1), (1, 4441, 12, 12), (3, 300, 40, 40)])
@pytest.mark.parametrize("half", [False, True])
def test_rope_lengths_and_head_layouts(B, L, H, Hk, half):
    rope_case(B, L, H, Hk, 128, 128, half, 3, BF16, seed=4)


@pytest.mark.parametrize("half,r", [(False, 128), (False, 50), (True, 128), (True, 50), (True, 64)])
def test_rope_in_place_on_views_of_a_packed_projection(half, r):
    rope_case(2, 65, 4, 4, 128, r, half, 1, BF16, in_place=True, packed=True)


def test_rope_without_positions_and_far_positions():
    rope_case(2, 130, 2, 2, 64, 64, False, 1, FP16, positions=False)
    for start in (10 ** 5, 10 ** 8, 2 ** 31 - 5000):
        rope_case(1, 130, 2, 2, 64, 64, True, 1, FP16, start=start)


def test_rope_transpose_is_the_gradient_and_the_inverse():
    """The rotation is linear: its transpose on g is the gradient of sum(g * rope(x)), also by differences; with factor 1 it
    turns back."""
    rope_case(1, 33, 2, 2, 64, 48, True, 1, FP16, transpose=True, factor=1.25)
    x, g = rnd((1, 9, 2, 64), 1, FP16), rnd((1, 9, 2, 64), 2, FP16)
    freqs = dt.dt_rope_freqs(64)[0][None].cuda()
    y, gx, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dt.dt_rope(x, None, y, None, freqs, layout=dt.DT_ROPE_HALF)
    dt.dt_rope(g, None, gx, None, freqs, layout=dt.DT_ROPE_HALF, transpose=True)
    dt.dt_rope(y, None, back, None, freqs, layout=dt.DT_ROPE_HALF, transpose=True)
    u = torch.finfo(FP16).eps / 2
    # <g, R x> = <R^T g, x>: each side has one rounding per product
    lhs, rhs = (g.double() * y.double()).sum(), (gx.double() * x.double()).sum()
    bound = 2 * u * ((g.double() * y.double()).abs().sum() + (gx.double() * x.double()).abs().sum())
    assert (lhs - rhs).abs() <= bound
    # a difference along e: rope(x + e) - rope(x), e large enough to survive the rounding; the slope is <gx, e>
    e = torch.zeros_like(x); e[0, 5, 1, 10] = 2.0
    y2 = torch.empty_like(x)
    dt.dt_rope((x + e), None, y2, None, freqs, layout=dt.DT_ROPE_HALF)
    step = (x + e).double() - x.double()
    slope = (g.double() * (y2.double() - y.double())).sum()
    assert (slope - (gx.double() * step).sum()).abs() <= 4 * u * ((g.double() * y.double()).abs()[0, 5].sum() + (gx.double() * step).abs().sum() * 2 + 4 * g.double().abs()[0, 5, 1].sum())
    r = (x[..., :32].double().abs() + x[..., 32:].double().abs()).repeat(1, 1, 1, 2)
    assert ((back.double() - x.double()).abs() <= 3 * u * r).all()


def test_rope_untouched_values_keep_their_bits_and_rows_behind_the_last_token_stay():
    buf = torch.full((2, 20, 3, 64), float("nan"), device="cuda", dtype=BF16)
    x = buf[:, :17]
    x.copy_(rnd((2, 17, 3, 64), 3, BF16))
    x[0, 0, 0, 40:] = torch.tensor([float("inf"), float("nan")] * 12, device="cuda", dtype=BF16)
    before = buf.clone()
    dt.dt_rope(x, None, x, None, dt.dt_rope_freqs(32)[0][None].cuda())
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(buf[:, 17:].contiguous(), before[:, 17:].contiguous())
    assert same(x[..., 32:].contiguous(), before[:, :17, :, 32:].contiguous())
    assert torch.isfinite(x[..., :32]).all()


def test_rope_positions_of_an_expanded_batch():
    x = rnd((3, 11, 2, 64), 5, BF16)
    pos = torch.arange(11, device="cuda", dtype=torch.int32)[None].expand(3, 11)
    f = dt.dt_rope_freqs(64)[0][None].cuda()
    a, b = torch.empty_like(x), torch.empty_like(x)
    dt.dt_rope(x, None, a, None, f, pos)
    dt.dt_rope(x, None, b, None, f)
    assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------- norm
def norm_check(x, weight, residual, residual_out, y, scales, eps, want_h, want_y, what):
    if residual is not None:
        rt = residual_out.dtype
        u = torch.finfo(rt).eps / 2
        check(residual_out, want_h, want_h.abs() * (u + ref.U32) + torch.finfo(rt).tiny * u, (what, "residual_out"))
    if y.dtype != E4M3:
        u = torch.finfo(y.dtype).eps / 2
        check(y, want_y, want_y.abs() * (u + ref.NORM_REL) + torch.finfo(y.dtype).tiny * u, (what, "y"))
        return
    g = want_y.unflatten(-1, (scales.shape[-1], -1))
    want_s = g.abs().amax(-1).clamp_min(2.0 ** -100) / 448
    check(scales, want_s, want_s * (ref.NORM_REL + 2 * ref.U32), (what, "scales"))
    got = y.double().unflatten(-1, (scales.shape[-1], -1)) * scales.double()[..., None]
    # half a step of e4m3: 2^-4 relative, and 2^-10 of the scale below its normal range
    tol = torch.maximum(g.abs() * 2.0 ** -4, want_s[..., None] * 2.0 ** -10) + g.abs() * 4 * ref.NORM_REL
    check(got, g, tol, (what, "values"))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("residual", ["none", "same", "fp32"])
@pytest.mark.parametrize("out,group", [("same", 0), ("e4m3", 0), ("e4m3", 32), ("e4m3", 64), ("e4m3", 128)])
@pytest.mark.parametrize("rows,width", [(1, 128), (3, 5120), (7, 256), (5, 384), (33, 2176), (2, 16384), (257, 128), (4, 4224)])
def test_norm(rows, width, out, group, residual, dtype):
    x = rnd((rows, width), 1, dtype)
    w = rnd((width,), 2, FP32 if rows % 2 else dtype, 0.3) + 1
    res = None if residual == "none" else rnd((rows, width), 3, FP32 if residual == "fp32" else dtype, 3.0)
    h, y = ref.norm(x, w, 1e-6, res)
    got = torch.full((rows, width), 3.0, device="cuda").to(dtype if out == "same" else E4M3)
    sc = torch.full((rows, width // group if group else 1), -1.0, device="cuda") if out == "e4m3" else None
    ro = torch.empty_like(res) if res is not None else None
    dt.dt_add_rmsnorm(x, w, got, 1e-6, residual=res, residual_out=ro, scales=sc)
    torch.cuda.synchronize()
    norm_check(x, w, res, ro, got, sc, 1e-6, h, y, (rows, width, out, group, residual, dtype))


@pytest.mark.parametrize("width", [8, 16, 24, 64, 72, 136, 248, 264, 1000, 2056, 8200])
def test_norm_odd_widths(width):
    x, res = rnd((19, width), 1, BF16), rnd((19, width), 2, FP32)
    h, y = ref.norm(x, None, 1e-5, res)
    for out in (BF16, E4M3):
        got = torch.empty((19, width), device="cuda", dtype=out)
        sc = torch.empty((19, 1), device="cuda") if out == E4M3 else None
        ro = torch.empty_like(res)
        dt.dt_add_rmsnorm(x, None, got, 1e-5, residual=res, residual_out=ro, scales=sc)
        torch.cuda.synchronize()
        norm_check(x, None, res, ro, got, sc, 1e-5, h, y, (width, out))


@pytest.mark.parametrize("width", [264, 1536, 2176, 5120, 8200, 16384])
@pytest.mark.parametrize("residual", ["none", "same", "fp32"])
@pytest.mark.parametrize("out,group", [("same", 0), ("e4m3", 0), ("e4m3", 128)])
def test_norm_of_many_rows(width, residual, out, group):
    """More rows than the GPU has places for blocks (they stream through the blocks), some of them in place, of a strided
    view, and rows behind the last that stay as they were."""
    if group and width % group:
        group = 8 * math.gcd(width // 8, 4)
        group = group if group in (32, 64) else 0
    rows = 2500 + 37
    buf = rnd((rows + 2, width + 64), 1, BF16)
    x = buf[:rows, :width]
    res = None if residual == "none" else rnd((rows + 2, width), 3, FP32 if residual == "fp32" else BF16, 3.0)
    behind = None if res is None else res[rows:].clone()
    w = rnd((width,), 2, FP32, 0.3) + 1
    h, y = ref.norm(x, w, 1e-6, None if res is None else res[:rows])
    sc = None
    if out == "e4m3":
        got = torch.full((rows + 2, width), 9.0, device="cuda").to(E4M3)
        sc = torch.full((rows + 2, width // group if group else 1), 9.0, device="cuda")
    else:
        got = buf[:, :width]            # y in x's place
        last = got[rows:].clone()
    ro = None if res is None else res[:rows]
    dt.dt_add_rmsnorm(x, w, got[:rows], 1e-6, residual=ro, residual_out=ro, scales=None if sc is None else sc[:rows])
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    norm_check(x, w, ro, ro, got[:rows], None if sc is None else sc[:rows], 1e-6, h, y, (width, residual, out, group))
    if res is not None:
        assert torch.equal(res[rows:], behind)
    if sc is not None:
        assert (got[rows:].float() == 9).all() and (sc[rows:] == 9).all()
    else:
        assert torch.equal(got[rows:], last) and torch.equal(buf[:, width:], rnd((rows + 2, width + 64), 1, BF16)[:, width:])


@pytest.mark.parametrize("D", [64, 128])
def test_norm_over_heads_of_a_packed_projection_in_place(D):
    qkv = rnd((2, 70, 9, D), 1, BF16)
    w = rnd((D,), 2, BF16, 0.2) + 1
    for part in (qkv[:, :, 0:3], qkv[:, :, 3:6]):
        _, y = ref.norm(part, w, 1e-6, None)
        dt.dt_add_rmsnorm(part, w, part, 1e-6)
        torch.cuda.synchronize()
        norm_check(None, w, None, None, part, None, 1e-6, None, y, "heads")
    assert torch.equal(qkv[:, :, 6:], rnd((2, 70, 9, D), 1, BF16)[:, :, 6:])


def test_norm_residual_in_place_and_rows_behind_the_last_stay():
    buf = torch.full((12, 640), 9.0, device="cuda", dtype=FP32)
    res = buf[:9]
    res.copy_(rnd((9, 640), 5, FP32, 2.0))
    x = rnd((9, 640), 6, BF16)
    ybuf = torch.full((12, 640), 9.0, device="cuda").to(E4M3)
    sc = torch.full((12, 5), 9.0, device="cuda")
    h, y = ref.norm(x, None, 1e-6, res)
    dt.dt_add_rmsnorm(x, None, ybuf[:9], 1e-6, residual=res, residual_out=res, scales=sc[:9])
    torch.cuda.synchronize()
    norm_check(x, None, res, res, ybuf[:9], sc[:9], 1e-6, h, y, "in place")
    assert (buf[9:] == 9).all() and (ybuf[9:].float() == 9).all() and (sc[9:] == 9).all()


@pytest.mark.parametrize("rows,width", [(5, 64), (3000, 384), (9, 5120), (2000, 2560)])
def test_norm_sum_in_the_place_of_x_and_one_row_for_all(rows, width):
    x, res = rnd((rows, width), 1, BF16), rnd((1, width), 2, BF16, 2.0).expand(rows, width)
    h, want = ref.norm(x, None, 1e-6, res)
    y = torch.empty_like(x)
    dt.dt_add_rmsnorm(x, None, y, 1e-6, residual=res, residual_out=x)
    torch.cuda.synchronize()
    norm_check(None, None, res, x, y, None, 1e-6, h, want, (rows, width))


def test_norm_and_rope_offsets_beyond_32_bits():
    far = 2 ** 31 // 40 // 8 * 8 + 8
    room = torch.empty(far * 50 + 4096, device="cuda", dtype=BF16)
    for width, n in ((128, 51), (1024, 51), (2560, 51)):
        x = room.as_strided((n, width), (far, 1))
        x.copy_(rnd((n, width), 1, BF16))
        _, want = ref.norm(x, None, 1e-6, None)
        dt.dt_add_rmsnorm(x, None, x, 1e-6)
        torch.cuda.synchronize()
        norm_check(None, None, None, None, x, None, 1e-6, None, want, width)
    q = room.as_strided((1, 51, 2, 64), (0, far, 64, 1))
    q.copy_(rnd((1, 51, 2, 64), 2, BF16))
    angle = (torch.arange(51, device="cuda").double()[None, :, None] * dt.dt_rope_freqs(64)[0].cuda()).expand(1, 51, 32)
    want, tol = ref.rope(q, angle, False, 64)
    dt.dt_rope(q, None, q, None, dt.dt_rope_freqs(64)[0][None].cuda())
    torch.cuda.synchronize()
    check(q, want, tol, "far")


def test_rope_and_norm_repeat_bit_for_bit_on_other_streams_and_in_graphs():
    q, k = rnd((2, 700, 6, 128), 1, FP16), rnd((2, 700, 2, 128), 2, FP16)
    f = dt.dt_rope_freqs(128)[0][None].cuda()
    x, res = rnd((3000, 1536), 3, BF16), rnd((3000, 1536), 4, FP32)

    def passes(stream=None):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        y, sc, ro = torch.empty((3000, 1536), device="cuda", dtype=E4M3), torch.empty((3000, 12), device="cuda"), torch.empty_like(res)
        dt.dt_rope(q, k, qo, ko, f, layout=dt.DT_ROPE_HALF, stream=stream)
        dt.dt_add_rmsnorm(x, None, y, 1e-6, residual=res, residual_out=ro, scales=sc, stream=stream)
        return qo, ko, y.view(torch.uint8), sc, ro
    plain = passes()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [passes(s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = passes()
    for t in held:
        t.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    for other in got + [held]:
        assert all(torch.equal(a, b) for a, b in zip(plain, other))


def test_norm_of_zero_rows_large_values_and_no_rows():
    x = torch.zeros((3, 512), device="cuda", dtype=BF16)
    x[1] = rnd((512,), 1, BF16) * 1e18        # squares stay inside fp32
    y, sc = torch.empty((3, 512), device="cuda", dtype=E4M3), torch.empty((3, 4), device="cuda")
    dt.dt_add_rmsnorm(x, None, y, 1e-6, scales=sc)
    torch.cuda.synchronize()
    h, want = ref.norm(x, None, 1e-6, None)
    norm_check(x, None, None, None, y, sc, 1e-6, h, want, "zeros")
    assert (y[0].float() == 0).all() and torch.equal(sc[0], torch.full_like(sc[0], 2.0 ** -100 / 448))
    e = torch.empty((0, 512), device="cuda", dtype=BF16)
    dt.dt_add_rmsnorm(e, None, e.clone(), 1e-6)


# ---------------------------------------------------------------------------------------------- cross attention
def keep_of(B, Lk, lens, mask):
    keep = torch.ones((B, Lk), dtype=torch.bool, device="cuda")
    if lens is not None:
        keep &= torch.arange(Lk, device="cuda")[None] < lens[:, None]
    if mask is not None:
        keep &= mask != 0
    return keep


def cross_run(q, k, v, scale, lens=None, mask=None, out=None, what=""):
    B, Lq, H, D = q.shape
    keep = keep_of(B, k.shape[1], lens, mask) if lens is not None or mask is not None else None
    out = torch.full((B, Lq, H, D), 5.0, device="cuda", dtype=q.dtype) if out is None else out
    lse = torch.full((B, H, Lq), 5.0, device="cuda")
    dt.dt_cross_attn(q, k, v, out, scale, key_lens=lens, key_mask=mask, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    wo, wl, to, tl = ref.cross(q, k, v, scale, keep)
    check(lse, wl, tl, (what, "lse"))
    check(out, wo, to, (what, "out"))
    return out, lse


LQ = [1, 2, 15, 16, 17, 33, 65, 127, 128, 129, 255, 256, 257, 300, 513, 700]
LK = [1, 2, 7, 15, 16, 17, 63, 64, 65, 100, 127, 128, 129, 226, 255, 256, 257, 400, 512, 1000]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", range(20))
def test_cross_lengths(n, D, dtype):
    """Every query length meets several key lengths, with the head layouts in turn."""
    Lk = LK[n]
    H, Hk = [(1, 1), (2, 2), (4, 2), (5, 1), (6, 3)][n % 5]
    for j in range(4):
        Lq = LQ[(5 * n + 4 * j + n // 4) % len(LQ)]
        q, k, v = rnd((2, Lq, H, D), n, dtype, 1.5), rnd((2, Lk, Hk, D), n + 100, dtype, 1.5), rnd((2, Lk, Hk, D), n + 200, dtype)
        cross_run(q, k, v, D ** -0.5, what=(Lq, Lk, H, Hk, D, dtype))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq", [1, 3, 40, 130, 300, 600])
@pytest.mark.parametrize("Lk", [1, 64, 129, 226, 512, 777])
def test_cross_masks_with_nan_in_masked_places(Lk, Lq, D, dtype):
    """Lengths (0, 1, odd, all, beyond), masks with holes, both, and a request without any key; what stands in masked places
    is NaN and infinity in turn."""
    B, H, Hk = 4, 4, 2
    q, k, v = rnd((B, Lq, H, D), 1, dtype, 1.5), rnd((B, Lk, Hk, D), 2, dtype, 1.5), rnd((B, Lk, Hk, D), 3, dtype)
    lens = torch.tensor([0, 1, max(Lk - 5, 1), Lk + 1000], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda"); g.manual_seed(Lk)
    holes = (torch.rand((B, Lk), generator=g, device="cuda") < 0.6).to(torch.uint8) * 3
    holes[3] = 0
    if Lk > 200:
        holes[2, :190] = 0      # whole tiles without a key ahead of the first that counts
    for ln, mk in ((lens, None), (None, holes), (lens, holes), (None, holes.bool())):
        keep = keep_of(B, Lk, ln, mk)
        kk, vv = k.clone(), v.clone()
        kk[~keep] = float("nan")
        vv[~keep] = float("inf") if Lq % 2 else float("nan")
        out, lse = cross_run(q, kk, vv, D ** -0.5, ln, mk, what=(Lq, Lk, D, dtype))
        none = ~keep.any(1)
        assert (out[none] == 0).all() and torch.isinf(lse[none]).all() and none.any()


@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, FP16)])
@pytest.mark.parametrize("Lk", [1, 77, 128, 129, 226, 300, 640])
def test_cross_many_blocks_of_rows_per_sm(Lk, D, dtype):
    """More blocks of 256 rows than the GPU has SMs, so that every SM takes several one after the other: one tile of keys each,
    two, more, and (lengths) a mix with none.  A few (request, head) pairs are compared element by element."""
    B, Lq, H = 3, 4000, 12
    q, k, v = rnd((B, Lq, H, D), 1, dtype, 1.3), rnd((B, Lk, H, D), 2, dtype, 1.3), rnd((B, Lk, H, D), 3, dtype)
    for lens in (None, torch.tensor([Lk, 0, (Lk + 1) // 2], dtype=torch.int32, device="cuda")):
        out, lse = torch.full_like(q, 5.0), torch.full((B, H, Lq), 5.0, device="cuda")
        dt.dt_cross_attn(q, k, v, out, D ** -0.5, key_lens=lens, lse_out=lse)
        torch.cuda.synchronize()
        dt.dt_poll_ops()
        keep = keep_of(B, Lk, lens, None)
        for h in (0, 5, 11):
            wo, wl, to, tl = ref.cross(q[:, :, h:h + 1], k[:, :, h:h + 1], v[:, :, h:h + 1], D ** -0.5, keep)
            check(lse[:, h:h + 1], wl, tl, (Lk, D, h, "lse"))
            check(out[:, :, h:h + 1], wo, to, (Lk, D, h, "out"))


@pytest.mark.parametrize("D,dtype", [(64, FP16), (128, BF16)])
@pytest.mark.parametrize("Lk", [5, 128, 200, 226, 512, 700])
def test_cross_masks_in_many_blocks_of_rows(Lk, D, dtype):
    """Masks with holes, lengths, and both, with NaN in masked places, where every SM takes several blocks of rows; the groups of
    heads share keys, and one request has no key."""
    B, Lq, H, Hk = 3, 3000, 12, 4
    q, k, v = rnd((B, Lq, H, D), 1, dtype, 1.3), rnd((B, Lk, Hk, D), 2, dtype, 1.3), rnd((B, Lk, Hk, D), 3, dtype)
    g = torch.Generator(device="cuda"); g.manual_seed(Lk)
    holes = (torch.rand((B, Lk), generator=g, device="cuda") < 0.7).to(torch.uint8)
    holes[1] = 0
    lens = torch.tensor([Lk, Lk, (Lk + 2) // 3], dtype=torch.int32, device="cuda")
    for ln, mk in ((None, holes), (lens, None), (lens, holes)):
        keep = keep_of(B, Lk, ln, mk)
        kk, vv = k.clone(), v.clone()
        kk[~keep] = float("nan")
        vv[~keep] = float("inf")
        out, lse = torch.full_like(q, 5.0), torch.full((B, H, Lq), 5.0, device="cuda")
        dt.dt_cross_attn(q, kk, vv, out, D ** -0.5, key_lens=ln, key_mask=mk, lse_out=lse)
        torch.cuda.synchronize()
        dt.dt_poll_ops()
        for h in (0, 5, 11):
            ks = kk[:, :, h // 3:h // 3 + 1], vv[:, :, h // 3:h // 3 + 1]
            wo, wl, to, tl = ref.cross(q[:, :, h:h + 1], *ks, D ** -0.5, keep)
            check(lse[:, h:h + 1], wl, tl, (Lk, D, h, "lse"))
            check(out[:, :, h:h + 1], wo, to, (Lk, D, h, "out"))


@pytest.mark.parametrize("D,dtype", [(64, FP16), (128, BF16), (128, FP16)])
@pytest.mark.parametrize("B,Lq,H,Hk,Lk", [(1, 700, 8, 8, 2500), (2, 1000, 4, 4, 3001), (1, 2000, 2, 1, 1152), (1, 3000, 1, 1, 5000), (3, 513, 12, 4, 1024),
                                          (1, 2049, 8, 8, 520)])
def test_cross_long_states_of_many_tokens(B, Lq, H, Hk, Lk, D, dtype):
    """Too few blocks of rows to fill the GPU: the keys are split as well.  All keys, lengths that leave some of the splits
    nothing (or a request nothing), and a mask with NaN in masked places."""
    q, k, v = rnd((B, Lq, H, D), 1, dtype, 1.3), rnd((B, Lk, Hk, D), 2, dtype, 1.3), rnd((B, Lk, Hk, D), 3, dtype)
    g = torch.Generator(device="cuda"); g.manual_seed(Lk)
    holes = (torch.rand((B, Lk), generator=g, device="cuda") < 0.5).to(torch.uint8)
    holes[0, Lk // 4:Lk // 2 + 300] = 0
    for lens, mask in ((None, None), (torch.tensor([100, 0, Lk][:B], dtype=torch.int32, device="cuda"), None), (None, holes),
                       (torch.tensor([Lk - 7, Lk // 2, 1][:B], dtype=torch.int32, device="cuda"), holes)):
        keep = keep_of(B, Lk, lens, mask)
        kk, vv = k.clone(), v.clone()
        kk[~keep] = float("nan")
        vv[~keep] = float("nan")
        cross_run(q, kk, vv, D ** -0.5, lens, mask, what=(Lq, Lk, H))


@pytest.mark.parametrize("Lq,Lk", [(1, 0), (300, 0), (0, 5), (0, 0)])
def test_cross_without_keys_or_queries(Lq, Lk):
    q, k = rnd((2, Lq, 4, 64), 1, BF16), rnd((2, Lk, 4, 64), 2, BF16)
    out, lse = torch.full_like(q, 3), torch.full((2, 4, Lq), 3.0, device="cuda")
    dt.dt_cross_attn(q, k, k, out, 0.125, lse_out=lse)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("Lq,Lk,H,Hk", [(1, 300, 8, 1), (5, 200, 4, 4), (300, 226, 4, 2), (520, 512, 2, 2)])
def test_cross_strided_views_and_an_expanded_batch(Lq, Lk, H, Hk, dtype):
    D = 128
    packed_q = rnd((2, Lq, 3, H, D), 1, dtype)                       # q as one of three of a packed projection
    packed_kv = rnd((2, Lk, 2, Hk, D), 2, dtype)
    q, k, v = packed_q[:, :, 1], packed_kv[:, :, 0], packed_kv[:, :, 1]
    buf = torch.full((2, Lq + 3, H + 1, D), 9.0, device="cuda", dtype=dtype)
    cross_run(q, k, v, 0.09, out=buf[:, :Lq, :H], what="packed")
    assert (buf[:, Lq:] == 9).all() and (buf[:, :, H:] == 9).all()   # rows behind the last token and another's head: as they were
    heads_first = rnd((2, Hk, Lk, D), 3, dtype).transpose(1, 2)      # [B, H, L, D] in memory
    cross_run(rnd((2, H, Lq, D), 4, dtype).transpose(1, 2), heads_first, v, 0.09, out=rnd((2, H, Lq, D), 5, dtype).transpose(1, 2), what="heads first")
    one = rnd((1, Lk, Hk, D), 6, dtype).expand(2, Lk, Hk, D)         # one prompt for both requests
    mask = (torch.rand((1, Lk), device="cuda") < 0.8).expand(2, Lk)
    cross_run(q, one, one, 0.09, mask=mask, what="expanded")
    odd = rnd((1, Lq, H, D), 7, dtype)
    cross_run(odd.as_strided(odd.shape, (1, H * D, D, 1)), rnd((1, Lk, Hk, D), 8, dtype), rnd((1, Lk, Hk, D), 9, dtype), 0.09, what="stride of one batch")


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("Lq", [1, 20, 300])
def test_cross_logits_that_climb_fall_and_jump(Lq, dtype):
    """The running maximum has to move within a tile and between tiles, by little and by hundreds; equal logits; one key that
    takes everything."""
    D, Lk = 64, 700
    q = torch.zeros((1, Lq, 2, D), device="cuda", dtype=dtype)
    q[..., 0] = 8.0
    v = rnd((1, Lk, 2, D), 3, dtype)
    j = torch.arange(Lk, device="cuda", dtype=torch.float32)
    for x in (j / 2, -j / 2, (j % 128) * 3, torch.where(j == 400, 300.0, 0.0), torch.zeros_like(j), torch.where(j > 350, 250.0, -250.0), j * 0 - 300):
        k = torch.zeros((1, Lk, 2, D), device="cuda", dtype=dtype)
        k[..., 0] = (x / 8)[None, :, None].to(dtype)
        cross_run(q, k, v, 1.0, what=("logits", Lq))


def test_cross_long_states_of_single_tokens():
    for B, H, Hk, D, Lk in ((1, 8, 1, 128, 20011), (2, 4, 4, 64, 5000), (1, 2, 2, 128, 32760)):
        q, k, v = rnd((B, 1, H, D), 1, FP16), rnd((B, Lk, Hk, D), 2, FP16), rnd((B, Lk, Hk, D), 3, FP16)
        lens = torch.tensor([Lk - 11 * b for b in range(B)], dtype=torch.int32, device="cuda")
        cross_run(q, k, v, D ** -0.5, lens, what=("long", Lk))


@pytest.mark.parametrize("B,Lq,H,Hk,Lk", [(2, 3, 8, 2, 300), (2, 5000, 12, 12, 200), (1, 600, 4, 4, 2000)])
def test_cross_output_in_the_place_of_q(B, Lq, H, Hk, Lk):
    """Few rows, many blocks of rows, keys split over a cluster."""
    q, k, v = rnd((B, Lq, H, 128), 1, BF16), rnd((B, Lk, Hk, 128), 2, BF16), rnd((B, Lk, Hk, 128), 3, BF16)
    out = torch.empty_like(q)
    dt.dt_cross_attn(q, k, v, out, 0.1)
    dt.dt_cross_attn(q, k, v, q, 0.1)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    assert torch.equal(q, out)


@pytest.mark.parametrize("Lq,Lk", [(1, 300), (4000, 300), (600, 2000)])
def test_cross_where_no_request_has_a_key(Lq, Lk):
    q, k = rnd((2, Lq, 4, 64), 1, FP16), torch.full((2, Lk, 4, 64), float("nan"), device="cuda", dtype=FP16)
    for kw in (dict(key_lens=torch.tensor([0, -3], dtype=torch.int32, device="cuda")), dict(key_mask=torch.zeros((2, Lk), dtype=torch.uint8, device="cuda"))):
        out, lse = torch.full_like(q, 3), torch.full((2, 4, Lq), 3.0, device="cuda")
        dt.dt_cross_attn(q, k, k, out, 0.125, lse_out=lse, **kw)
        torch.cuda.synchronize()
        dt.dt_poll_ops()
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk", [(2, 300), (4000, 300), (600, 2000)])
def test_cross_rows_of_q_without_a_number_and_without_keys(Lq, Lk, D, dtype):
    """A request whose mask leaves no key gives OUT = 0, LSE = -inf for every q; the other request is as it was."""
    q, k, v = (rnd((2, n, 4, D), i, dtype) for i, n in enumerate((Lq, Lk, Lk)))
    mask = torch.ones((2, Lk), dtype=torch.bool, device="cuda")
    mask[1] = False
    want = torch.empty_like(q)
    dt.dt_cross_attn(q, k, v, want, 0.1, key_mask=mask)
    q[1, ::3] = float("nan")
    q[1, 1::3] = float("inf")
    out, lse = torch.empty_like(q), torch.empty((2, 4, Lq), device="cuda")
    dt.dt_cross_attn(q, k, v, out, 0.1, key_mask=mask, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    assert torch.equal(out[0], want[0]) and torch.isfinite(lse[0]).all()
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("Lq,Lk", [(2, 300), (4000, 300), (600, 2000)])
def test_cross_a_row_of_q_without_a_number_stays_alone(Lq, Lk):
    """A NaN in a row of q with keys gives NaN there, and changes no other row."""
    q, k, v = (rnd((1, n, 4, 128), i, BF16) for i, n in enumerate((Lq, Lk, Lk)))
    wo, wl, to, tl = ref.cross(q, k, v, 0.1)
    q[0, Lq // 2, 1, 5] = float("nan")
    out, lse = torch.empty_like(q), torch.empty((1, 4, Lq), device="cuda")
    dt.dt_cross_attn(q, k, v, out, 0.1, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    assert out[0, Lq // 2, 1].isnan().all() and lse[0, 1, Lq // 2].isnan()
    out[0, Lq // 2, 1], lse[0, 1, Lq // 2] = wo[0, Lq // 2, 1].to(BF16), wl[0, 1, Lq // 2].float()
    check(out, wo, to, "out")
    check(lse, wl, tl, "lse")


@pytest.mark.parametrize("width", [64, 512, 2048, 5120])
def test_norm_scales_near_the_end_of_fp32(width):
    """y of 10^38: the scale is 10^38 / 448 and the largest values are 448."""
    x = rnd((7, width), 1, BF16).sign()
    x[x == 0] = 1
    y, sc = torch.empty((7, width), device="cuda", dtype=E4M3), torch.empty((7, 1), device="cuda")
    dt.dt_add_rmsnorm(x, torch.full((width,), 1e38, device="cuda"), y, 0.0, scales=sc)
    torch.cuda.synchronize()
    assert torch.equal(y.float(), 448 * x.float())
    # r, r * w, and the quotient by 448, of a few roundings each
    assert ((sc.double() * 448 / 1e38 - 1).abs() <= 2 ** -20).all()


def test_norm_called_from_two_threads():
    """Rows of two widths, both beyond the shared memory that a launch has without asking, from two threads at once (through
    ctypes, which lets go of the interpreter)."""
    lib = dt.lib()
    n = 3000
    work, status = [], []
    for i, width in enumerate((12800, 16384)):
        x = rnd((n, width), i, BF16)
        y = torch.empty_like(x)
        pair = ctypes.c_int64 * 2
        cfg = dt.dt_norm_config(0, 0, 0, 0, 1, n, width, 0, pair(0, width), pair(0, width), pair(0, width), pair(0, width), 1e-6)
        work.append((x, y, cfg, torch.cuda.Stream()))

    def run(x, y, cfg, stream):
        status.extend(lib.dt_add_rmsnorm(ctypes.byref(cfg), x.data_ptr(), None, None, None, y.data_ptr(), None, stream.cuda_stream) for _ in range(300))
    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert status == [dt.DT_OK] * 600
    for x, y, _, _ in work:
        h, want = ref.norm(x, None, 1e-6, None)
        norm_check(None, None, None, None, y, None, 1e-6, h, want, x.shape)


@pytest.mark.parametrize("call", ["dt.dt_rope(q, None, q, None, f)", "dt.dt_add_rmsnorm(q, None, q, 1e-6)",
                                  "dt.dt_cross_attn(q[:, :1], q, q, o[:, :1], 0.1)", "dt.dt_cross_attn(q, q, q, o, 0.1)"])
def test_first_call_of_a_process_inside_a_capture(call):
    text = f"""
import torch
from paper_2607_15650_b200 import binding as dt
q, o = torch.ones((1, 3000, 16, 64), device="cuda", dtype=torch.bfloat16), torch.zeros((1, 3000, 16, 64), device="cuda", dtype=torch.bfloat16)
f = dt.dt_rope_freqs(64)[0][None].cuda()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    {call}
g.replay()
torch.cuda.synchronize()
dt.dt_poll_ops()
print(q.isfinite().all().item() and o.isfinite().all().item())
"""
    r = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and r.stdout.split()[-1] == "True", r.stdout + r.stderr


def test_cross_offsets_beyond_32_bits():
    """The last head's keys lie more than 2^31 values behind the first's."""
    Lk, H, D = 300, 2, 64
    far = 2 ** 31 // Lk // 8 * 8 + 8
    room = torch.empty(far * (Lk - 1) + H * D + 64, device="cuda", dtype=BF16)
    k = room.as_strided((1, Lk, H, D), (0, far, D, 1))
    k.copy_(rnd((1, Lk, H, D), 1, BF16))
    for Lq in (1, 300):
        cross_run(rnd((1, Lq, H, D), 2, BF16), k, k, 0.125, what=("far", Lq))


def test_cross_repeats_bit_for_bit_on_other_streams_and_in_graphs():
    """Calls on two streams at once, and two captured graphs replayed in turn, give the bits of plain calls."""
    cases = [(2, 1, 300, 8, 2, 128), (1, 3000, 512, 16, 16, 64), (1, 40, 226, 2, 2, 128), (1, 1000, 2000, 4, 4, 128), (2, 9000, 300, 12, 12, 128)]
    ins = [(rnd((B, Lq, H, D), i, BF16), rnd((B, Lk, Hk, D), i + 10, BF16), rnd((B, Lk, Hk, D), i + 20, BF16)) for i, (B, Lq, Lk, H, Hk, D) in enumerate(cases)]
    plain = []
    for q, k, v in ins:
        o = torch.empty_like(q)
        dt.dt_cross_attn(q, k, v, o, 0.1)
        plain.append(o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for q, _, _ in ins] for _ in streams]
    for _ in range(5):
        for s, o in zip(streams, outs):
            for (q, k, v), x in zip(ins, o):
                dt.dt_cross_attn(q, k, v, x, 0.1, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, plain))
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for (q, k, v), x in zip(ins, o):
                dt.dt_cross_attn(q, k, v, x, 0.1)
        graphs.append(g)
    for o in outs:
        for x in o:
            x.zero_()
    for _ in range(3):
        for s, g in zip(streams, graphs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, plain))


def test_first_calls_of_a_process_may_be_captured():
    """Nothing an operator looks up on its first call is forbidden inside a capture."""
    code = (
        "import torch; from paper_2607_15650_b200 import binding as dt\n"
        "q=torch.randn(1,300,2,64,device='cuda',dtype=torch.bfloat16); k=q[:,:200]; o=torch.zeros_like(q); x=torch.zeros_like(q); y=torch.zeros_like(q)\n"
        "f=torch.ones(1,32,dtype=torch.float64,device='cuda'); g=torch.cuda.CUDAGraph()\n"
        "with torch.cuda.graph(g):\n"
        "    dt.dt_rope(q,None,x,None,f); dt.dt_add_rmsnorm(x,None,y,1e-6); dt.dt_cross_attn(y,k,k,o,0.125)\n"
        "g.replay(); torch.cuda.synchronize(); assert o.abs().sum() > 0; dt.dt_poll_ops(); print('captured')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


# ---------------------------------------------------------------------------------------------- together
def test_the_operators_of_a_block_together_with_the_self_attention():
    """residual + norm (8 bits) -> projection -> Q's and K's norm -> rotation -> self-attention through the state cache ->
    residual + norm -> cross attention -> residual + norm, against the same block in 64 bits with the 16-bit tensors between
    the calls taken from the run itself (so that every call is held to its own error)."""
    B, H, D, grid, text = 2, 4, 64, (3, 8, 10), 77
    L, W = grid[0] * grid[1] * grid[2], H * D
    off = [0, 90, 160, L]
    ctx = dt.Context(B, H, D, L, off, D ** -0.5)
    x, stream = rnd((B, L, W), 1, BF16), rnd((B, L, W), 2, FP32, 2.0)
    w1, wq, wk = rnd((W,), 3, FP32, 0.1) + 1, rnd((D,), 4, BF16, 0.1) + 1, rnd((D,), 5, BF16, 0.1) + 1
    proj = rnd((W, 3 * W), 6, BF16, W ** -0.5)
    enc = rnd((B, text, 2, H, D), 7, BF16)
    lens = torch.tensor([text, 13], dtype=torch.int32, device="cuda")
    h8, sc = torch.empty((B, L, W), device="cuda", dtype=E4M3), torch.empty((B, L, 1), device="cuda")
    want_h, want_y = ref.norm(x, w1, 1e-6, stream)
    dt.dt_add_rmsnorm(x, w1, h8, 1e-6, residual=stream, residual_out=stream, scales=sc)
    norm_check(x, w1, stream, stream, h8, sc, 1e-6, want_h, want_y, "first norm")
    qkv = ((h8.float() * sc) @ proj.float()).to(BF16).view(B, L, 3, H, D)
    q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
    for t, w in ((q, wq), (k, wk)):
        _, y = ref.norm(t, w, 1e-6, None)
        dt.dt_add_rmsnorm(t, w, t, 1e-6)
        norm_check(None, w, None, None, t, None, 1e-6, None, y, "head norm")
    freqs = dt.dt_rope_grid_freqs((24, 20, 20)).cuda()
    n = torch.arange(L, device="cuda")
    pos = torch.stack([n // 80, n // 10 % 8, n % 10], 1).to(torch.int32)[None].expand(B, L, 3)
    angle = (pos.double()[..., None] * freqs).sum(2)
    want = [ref.rope(t, angle, False, D) for t in (q, k)]
    dt.dt_rope(q, k, q, k, freqs, pos)
    for t, (w, tol) in zip((q, k), want):
        check(t, w, tol, "rope")
    mask = torch.ones(9, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty((B, L, H, D), device="cuda", dtype=BF16), torch.empty((B, H, L), device="cuda")
    ctx.dt_attn_states(q, k, v, mask, 1)
    ctx.dt_state_merge(out, lse)
    ctx.dt_poll()
    wo, wl, _, _ = ref.cross(q, k, v, D ** -0.5)
    assert (out.double() - wo).abs().max() <= 2e-2 and (lse.double() - wl).abs().max() <= 5e-3
    # self-attention over all keys is also what the cross attention of the tokens to themselves gives
    cross_run(q, k, v, D ** -0.5, what="tokens to themselves")
    y = torch.empty((B, L, W), device="cuda", dtype=BF16)
    want_h, want_y = ref.norm(out.view(B, L, W), w1, 1e-6, stream)
    dt.dt_add_rmsnorm(out.view(B, L, W), w1, y, 1e-6, residual=stream, residual_out=stream)
    norm_check(None, w1, stream, stream, y, None, 1e-6, want_h, want_y, "second norm")
    a, _ = cross_run(y.view(B, L, H, D), enc[:, :, 0], enc[:, :, 1], D ** -0.5, lens, what="prompt")
    want_h, want_y = ref.norm(a.view(B, L, W), w1, 1e-6, stream)
    dt.dt_add_rmsnorm(a.view(B, L, W), w1, h8, 1e-6, residual=stream, residual_out=stream, scales=sc)
    norm_check(None, w1, stream, stream, h8, sc, 1e-6, want_h, want_y, "third norm")
