"""Operators around the self-attention at the ends of their types' ranges, on the GPU against plain 64-bit forms."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build
from tests import block_ops_reference as ref
from tests.test_gpu_block_ops import norm_check, rope_case

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
U32 = 2.0 ** -24
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    dt.lib()


# ---------------------------------------------------------------------------------------------- cross attention
def falling(Lq, H, Lk, D, dtype, below, v):
    """One key in every 16 of the first 512 has logit 0 and V = 0, all others stand `below` (binades, a tensor [Lk]) under it;
    every query row is the same.  Returns the tensors and, for one row in 64 bits, LSE, OUT and what OUT may be off by."""
    j = torch.arange(Lk, device="cuda")
    first = (j < 512) & (j % 16 == 0)
    x = torch.where(first, torch.zeros_like(below), -below)
    q = torch.zeros((1, Lq, H, D), device="cuda", dtype=dtype)
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -6
    k = torch.zeros((1, Lk, 1, D), device="cuda", dtype=dtype)
    k[0, :, 0, 0] = x.to(dtype)
    k[0, :, 0, 1] = ((x - k[0, :, 0, 0].float()) * 64).to(dtype)     # (what the type's step leaves of x)
    vv = torch.where(first[:, None], torch.zeros_like(v), v).to(dtype)[None, :, None]
    scale = math.log(2.0)
    logit = (k[0, :, 0, 0].double() + k[0, :, 0, 1].double() / 64) * scale
    lse = torch.logsumexp(logit, 0)
    p = (logit - lse).exp()
    vd = vv[0, :, 0].double()
    u = torch.finfo(dtype).eps / 2
    # a P of the type's normal range is off by u of itself; under it by half of fp16's fixed step, 2^-25, where the largest P is
    # 2^top or more (bf16's range is fp32's).  The logit: two products and the scale in fp32.  The sums over the keys: in the tiles a
    # thread adds 16 pairs four ways and then tile by tile, in the few-row kernel a lane one key in 8 of every 64th; O likewise, with
    # a step of the running sum per addition of 16.
    rel = u + 2 * (8 * U32 * logit.abs().max()) + 2 * (32 + Lk / 8) * U32
    tol = (p @ vd.abs()) * rel + (p @ vd).abs() * u
    if dtype == FP16:
        top = min(13, max(7, math.ceil(math.log2(Lk)) - 4))
        tol = tol + vd.abs().sum(0) * 2.0 ** -(25 + top) * p.max() + 2.0 ** -25
    return q, k, vv, scale, lse, p @ vd, tol


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("Lq,H,Lk", [(1, 2, 32760), (1, 8, 2 ** 20), (1, 2, 1000), (256, 76, 1000), (256, 76, 6000), (256, 76, 32760), (256, 76, 2 ** 18), (512, 4, 32760)])
@pytest.mark.parametrize("kind", ["equal", "spread", "deep"])
def test_cross_many_small_weights_behind_a_large_one(kind, Lq, H, Lk, dtype):
    """Few rows, tiles, and tiles split over a cluster.  The keys behind the large ones have 2^-25.4 of their weight each, or 2^-10 to
    2^-25, or 2^-20 to 2^-34, and together they are all that OUT has."""
    g = torch.Generator(device="cuda")
    g.manual_seed(Lk)
    r = torch.rand((Lk,), generator=g, device="cuda")
    below = {"equal": torch.full_like(r, 25.4), "spread": 10 + 15 * r, "deep": 20 + 14 * r}[kind]
    v = torch.randn((Lk, 64), generator=g, device="cuda") * 0.3 + 1
    q, k, v, scale, wl, wo, tol = falling(Lq, H, Lk, 64, dtype, below, v)
    out, lse = torch.full_like(q, 5.0), torch.full((1, H, Lq), 5.0, device="cuda")
    dt.dt_cross_attn(q, k, v, out, scale, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    assert ((lse.double() - wl).abs() <= 8 * U32 * 34 + (32 + Lk / 8) * U32 + 4 * U32 * (1 + abs(wl))).all()
    over = (out.double() - wo).abs() - tol
    assert over.max() <= 0, (over.max().item(), (out.double() - wo).abs().max().item(), wo.abs().max().item())


@pytest.mark.parametrize("Lq,H", [(1, 2), (256, 76), (512, 4)])
def test_cross_logits_just_within_reach_of_the_reference(Lq, H):
    """Later keys that exceed the first ones by up to fp16's headroom, a binade at a time: P stays finite, and exact powers of two
    come out exactly where all V are one."""
    Lk, D = 4096, 64
    for step in (1, 3, 4, 5, 15, 16):
        j = torch.arange(Lk, device="cuda")
        x = (j // 512).float() * step
        q = torch.zeros((1, Lq, H, D), device="cuda", dtype=FP16)
        q[..., 0] = 1.0
        k = torch.zeros((1, Lk, 1, D), device="cuda", dtype=FP16)
        k[0, :, 0, 0] = x.to(FP16)
        v = torch.ones_like(k)
        out, lse = torch.zeros_like(q), torch.zeros((1, H, Lq), device="cuda")
        dt.dt_cross_attn(q, k, v, out, math.log(2.0), lse_out=lse)
        torch.cuda.synchronize()
        dt.dt_poll_ops()
        want = torch.logsumexp(x.double() * math.log(2.0), 0)
        assert (out == 1).all(), (step, out.min().item(), out.max().item())
        assert ((lse.double() - want).abs() <= 8 * U32 * (x.max().item() + 1) + (32 + Lk / 8) * U32 + 4 * U32 * (1 + abs(want))).all()


@pytest.mark.parametrize("Lq,B,H", [(256, 75, 1), (512, 2, 8)])
@pytest.mark.parametrize("D,dtype", [(64, FP16), (128, BF16)])
def test_cross_rows_without_a_number_under_masks_of_many_keys(D, dtype, Lq, B, H):
    """A request whose mask has one key, far behind the others, one without any, and one with all: whole items of tiles, and split ones.
    The rows of Q without a number look through the mask."""
    Lk = 2 ** 20 + 77
    q = torch.zeros((B, Lq, H, D), device="cuda", dtype=dtype)
    q[:, 3::7] = float("nan")
    kv = torch.ones((1, Lk, 1, D), device="cuda", dtype=dtype).expand(B, Lk, 1, D)
    mask = torch.ones((B, Lk), device="cuda", dtype=torch.uint8)
    mask[0] = 0
    mask[1] = 0
    mask[1, Lk - 1] = 1
    out, lse = torch.full_like(q, 5.0), torch.full((B, H, Lq), 5.0, device="cuda")
    dt.dt_cross_attn(q, kv, kv, out, 0.1, key_mask=mask, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    nan = torch.zeros(Lq, dtype=torch.bool, device="cuda")
    nan[3::7] = True
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert out[1:, nan].isnan().all() and lse[1:, :, nan].isnan().all()
    assert (out[1:, ~nan] == 1).all()
    # equal logits of zero: LSE is the logarithm of the number of keys, whose sum is exact up to 2^24
    assert (lse[1, :, ~nan].abs() <= 2 * U32).all()
    assert ((lse[2:, :, ~nan].double() - math.log(Lk)).abs() <= 16 * U32 * math.log(Lk)).all()


def test_cross_of_as_many_keys_as_there_may_be():
    """2^26 keys in one item, masked altogether, with rows of Q without a number: the longest that a part of the kernel waits for another."""
    B, Lk, D = 75, 2 ** 26, 64
    q = torch.zeros((B, 256, 1, D), device="cuda", dtype=FP16)
    q[:, ::2] = float("nan")
    kv = torch.zeros((1, Lk, 1, D), device="cuda", dtype=FP16).expand(B, Lk, 1, D)
    mask = torch.zeros((B, Lk), device="cuda", dtype=torch.uint8)
    out, lse = torch.full_like(q, 5.0), torch.full((B, 1, 256), 5.0, device="cuda")
    dt.dt_cross_attn(q, kv, kv, out, 0.1, key_mask=mask, lse_out=lse)
    torch.cuda.synchronize()
    dt.dt_poll_ops()
    assert (out == 0).all() and (lse == -math.inf).all()


def test_a_wait_that_runs_out_is_reported_once_and_the_next_call_is_right():
    q, k = (torch.randn((1, n, 4, 64), device="cuda").to(BF16) for n in (700, 500))
    out, again = torch.empty_like(q), torch.empty_like(q)
    dt.dt_cross_attn(q, k, k, out, 0.125)
    dt.dt_poll_ops()
    dt.dt_selftest_ops_timeout(limit_us=500)
    dt.dt_cross_attn(q, k, k, again, 0.125)
    with pytest.raises(dt.DitangoError) as e:
        dt.dt_poll_ops()
    assert e.value.status == dt.DT_ERR_TIMEOUT
    dt.dt_poll_ops()
    assert torch.equal(out, again) and out.isfinite().all()
    s = torch.cuda.Stream()
    dt.dt_selftest_ops_timeout(limit_us=0, stream=s)
    with pytest.raises(dt.DitangoError):
        dt.dt_poll_ops()
    dt.dt_poll_ops()


# ---------------------------------------------------------------------------------------------- norm
E4M3 = torch.float8_e4m3fn


def test_norm_rows_of_two_strides_either_way_round_and_packed():
    """Rows (i, j) with the larger stride on i or on j, as tight as they go."""
    for n0, n1, s0, s1 in ((2, 3, 1536, 512), (2, 3, 512, 1024), (3, 2, 1032, 512), (4, 5, 520, 2080)):
        room = torch.full((8192 * 2,), 9.0, device="cuda", dtype=BF16)
        x = torch.randn((n0, n1, 512), device="cuda").to(BF16)
        y = room.as_strided((n0, n1, 512), (s0, s1, 1))
        dt.dt_add_rmsnorm(x, None, y, 1e-6)
        torch.cuda.synchronize()
        norm_check(x, None, None, None, y, None, 1e-6, None, ref.norm(x, None, 1e-6, None)[1], (s0, s1))
        y.fill_(9.0)
        assert (room == 9).all()


@pytest.mark.parametrize("rows,width", [(5, 64), (1000, 128), (7, 264), (5, 1024), (7, 2048), (2500, 2048), (9, 5120), (2500, 5120), (3, 16384), (1300, 16384)])
@pytest.mark.parametrize("out,group", [("same", 0), ("e4m3", 0), ("e4m3", 128), ("e4m3", 32)])
@pytest.mark.parametrize("residual", ["none", "same", "fp32"])
@pytest.mark.parametrize("size,weight", [(100.0, 1e37), (1e6, 1e36), (1e-16, 1e-29)])
def test_norm_of_rows_and_weights_whose_product_leaves_fp32(size, weight, residual, out, group, rows, width):
    """Rows of hundreds or millions with weights near fp32's end, and tiny rows with tiny weights (eps 0): y is well inside
    fp32, h * weight is not."""
    if group and width % group:
        group = 0
    g = torch.Generator(device="cuda")
    g.manual_seed(width + rows)
    x = (torch.randn((rows, width), generator=g, device="cuda") * size).to(BF16)
    w = (torch.rand((width,), generator=g, device="cuda") + 0.5) * weight
    res = None if residual == "none" else (torch.randn((rows, width), generator=g, device="cuda") * size).to(torch.float32 if residual == "fp32" else BF16)
    h, y = ref.norm(x, w, 0.0, res)
    got = torch.full((rows, width), 3.0, device="cuda").to(BF16 if out == "same" else E4M3)
    sc = torch.full((rows, width // group if group else 1), -1.0, device="cuda") if out == "e4m3" else None
    ro = torch.empty_like(res) if res is not None else None
    dt.dt_add_rmsnorm(x, w, got, 0.0, residual=res, residual_out=ro, scales=sc)
    torch.cuda.synchronize()
    norm_check(x, w, res, ro, got, sc, 0.0, h, y, (rows, width, out, group, residual))


# ---------------------------------------------------------------------------------------------- first calls
@pytest.mark.parametrize("call", [
    "dt.dt_rope(q, None, o, None, f)", "dt.dt_rope(q, None, o, None, f, layout=dt.DT_ROPE_HALF)", "dt.dt_add_rmsnorm(q, w, o, 1e-6)",
    "dt.dt_add_rmsnorm(q.view(100, 15360), None, o.view(100, 15360), 1e-6)",
    "dt.dt_cross_attn(q[:, :1], q, q, o[:, :1], 0.1)", "dt.dt_cross_attn(q, q[:, :300], q[:, :300], o, 0.1)",
    "dt.dt_cross_attn(q[:, :600], q, q, o[:, :600], 0.1)", "dt.dt_cross_attn(q, q, q, o, 0.1, key_mask=m)"])
def test_the_first_call_of_a_process_captured_gives_what_a_plain_call_gives(call):
    """The capture runs nothing; every replay writes the whole output, over what stood there, bit for bit as a call does."""
    text = f"""
import torch
from paper_2607_15650_b200 import binding as dt
g = torch.Generator(device="cuda"); g.manual_seed(1)
q = torch.randn((1, 1500, 16, 64), generator=g, device="cuda").to(torch.bfloat16)
w = torch.rand((64,), generator=g, device="cuda") + 0.5
m = torch.rand((1, 1500), generator=g, device="cuda") < 0.7
f = dt.dt_rope_freqs(64)[0][None].cuda()
o = torch.full_like(q, float("nan"))
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    {call}
torch.cuda.synchronize()
assert o.isnan().all()
got = []
for _ in range(2):
    o.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    got.append(o.clone())
o.fill_(float("nan"))
{call}
torch.cuda.synchronize()
dt.dt_poll_ops()
written = ~o.isnan()
assert written.any() and (o[written] != q[written]).any()
rows = written.all(-1).all(-1)[0]
n = int(rows.sum())
assert n in (1, 600, 1500) and rows[:n].all() and not written[0, n:].any(), n
for x in got:
    assert torch.equal(x.view(torch.int16), o.view(torch.int16))
print("same")
"""
    r = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and r.stdout.split()[-1] == "same", r.stdout + r.stderr


# ---------------------------------------------------------------------------------------------- rotary positions, rows of the norm
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("B,L,H,Hk,D,r,axes", [(1, 6007, 32, 8, 128, 38, 3), (2, 3001, 5, 3, 64, 18, 1), (1, 9001, 40, 40, 128, 100, 3), (1, 20011, 1, 1, 256, 250, 1),
                                               (3, 4001, 7, 2, 72, 70, 1), (1, 30011, 3, 0, 8, 6, 1)])
def test_rope_halves_off_16_byte_borders_in_several_waves(B, L, H, Hk, D, r, axes, dtype):
    rope_case(B, L, H, Hk, D, r, True, axes, dtype, seed=9)
    rope_case(B, L, H, Hk, D, r, True, axes, dtype, in_place=True, packed=True, transpose=True, factor=1.25, seed=9)


def test_norm_of_tensors_whose_rows_collapse_differently():
    """x of two strides, the residual of one, the output of two others: the same rows in each."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    x, res = n(3, 7, 9, 64)[:, :, 2:7], n(3, 7, 5, 64)
    ybuf = torch.full((3, 7, 6, 64), 9.0, device="cuda", dtype=BF16)
    h, want = ref.norm(x, None, 1e-6, res)
    ro = torch.empty_like(res)
    dt.dt_add_rmsnorm(x, None, ybuf[:, :, :5], 1e-6, residual=res, residual_out=ro)
    torch.cuda.synchronize()
    norm_check(x, None, res, ro, ybuf[:, :, :5], None, 1e-6, h, want, "collapse")
    assert (ybuf[:, :, 5] == 9).all()
    one = n(1, 1, 1, 64).expand(3, 7, 5, 64)           # one row for all
    h, want = ref.norm(x, None, 1e-6, one)
    y8, sc = torch.empty((3, 7, 5, 64), device="cuda", dtype=E4M3), torch.empty((3, 7, 5, 2), device="cuda")
    dt.dt_add_rmsnorm(x, None, y8, 1e-6, residual=one, residual_out=ro, scales=sc)
    torch.cuda.synchronize()
    norm_check(x, None, one, ro, y8, sc, 1e-6, h, want, "one row")
