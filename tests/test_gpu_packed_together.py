"""The operators for packed requests as they are used: projections, attention within the same requests, projection, one behind another
without a wait in between; and the shapes and values at which their kernels' ways part.  Tolerances: tests/packed_ops_reference.py."""
import math

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build
from tests import packed_ops_reference as ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    dt.lib()


def rnd(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(got, want, tol, what):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, (what, over.max().item())


class Layer:
    """x -> q, k, v with adapters per request -> attention within requests -> projection with adapters."""

    def __init__(self, borders, which, H, D, dtype, rank=16, adapters=3, **attn):
        self.borders, self.which, self.H, self.D, self.attn = borders, which, H, D, attn
        M, W = borders[-1], H * D
        self.M, self.W = M, W
        self.w = [rnd((3 * W, W), 1, dtype, 1.3 * W ** -0.5), rnd((W, W), 2, dtype, W ** -0.5)]
        self.a = [rnd((adapters, rank, W), 3 + i, dtype, W ** -0.5) for i in range(2)]
        self.b = [rnd((adapters, n, rank), 5 + i, dtype, 0.3 * rank ** -0.5) for i, n in enumerate((3 * W, W))]
        self.scales, self.bias = rnd((adapters,), 7, FP32).abs(), rnd((3 * W,), 8, dtype, 0.1)
        self.starts, self.of = ints(borders), ints(which)
        self.ws = torch.empty(dt.dt_adapter_workspace_bytes(M, rank), dtype=torch.uint8, device="cuda")
        self.qkv, self.o = torch.empty((1, M, 3 * H, D), dtype=dtype, device="cuda"), torch.empty((1, M, H, D), dtype=dtype, device="cuda")
        self.lse = torch.empty((1, H, M), device="cuda")

    def heads(self):
        return (self.qkv[:, :, i * self.H:(i + 1) * self.H] for i in range(3))

    def steps(self, x, y):
        q, k, v = self.heads()
        return [lambda: dt.dt_adapter_linear(x, self.w[0], self.qkv.view(self.M, -1), self.a[0], self.b[0], self.starts, self.of, self.ws, scales=self.scales, bias=self.bias),
                lambda: dt.dt_packed_attn(q, k, v, self.o, self.D ** -0.5, q_starts=self.starts, k_starts=self.starts, lse_out=self.lse, **self.attn),
                lambda: dt.dt_adapter_linear(self.o.view(self.M, -1), self.w[1], y, self.a[1], self.b[1], self.starts, self.of, self.ws, scales=self.scales)]


SHAPES = [([0, 3, 4, 9], 2, 64), ([0, 5, 5, 130, 300], 4, 128), ([0, 700, 1300, 1301, 2000], 8, 64)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("borders,H,D", SHAPES)
def test_projections_and_attention_of_packed_requests(borders, H, D, dtype):
    for attn in (dict(), dict(causal=True, softcap=8.0)):
        n = len(borders) - 1
        t = Layer(borders, [(i + 1) % 4 - 1 for i in range(n)], H, D, dtype, **attn)
        x, y = rnd((t.M, t.W), 9, dtype), torch.empty((t.M, t.W), dtype=dtype, device="cuda")
        for f in t.steps(x, y):
            f()
        dt.dt_poll_ops()
        # every step against its plain form on what it was given
        check(t.qkv.view(t.M, -1), *ref.linear(x, t.w[0], t.bias, t.a[0], t.b[0], t.scales, t.borders, t.which), "qkv")
        docs = [[(lo, hi, lo, hi, 0) for lo, hi in zip(borders, borders[1:])]]
        out, lse, tol, tol_lse, _ = ref.attention(*t.heads(), t.D ** -0.5, docs, **attn)
        check(t.o, out, tol, "attention")
        check(t.lse, lse, tol_lse, "lse")
        check(y, *ref.linear(t.o.view(t.M, -1), t.w[1], None, t.a[1], t.b[1], t.scales, t.borders, t.which), "out")


@pytest.mark.parametrize("borders,H,D", SHAPES)
def test_a_call_waits_for_the_one_before(borders, H, D):
    """Launches begin beside the end of the launch before: layers in a row, each call reading what the one before wrote and writing what it
    read, with no wait in between, in a graph too, give the bits of calls that were waited for one by one."""
    n = len(borders) - 1
    layers = [Layer(borders, [(i + s) % 4 - 1 for i in range(n)], H, D, BF16, causal=bool(s % 2)) for s in range(3)]
    first = rnd((layers[0].M, layers[0].W), 1, BF16)
    h = first.clone()

    def run(wait):
        h.copy_(first)
        for _ in range(3):
            for t in layers:
                for f in t.steps(h, h):
                    f()
                    if wait:
                        torch.cuda.synchronize()
            h.mul_(0.7)            # (a launch that is none of ours)
    run(True)
    want = h.clone()
    assert torch.isfinite(want).all()
    for _ in range(5):
        run(False)
        assert torch.equal(h, want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(False)
    for _ in range(3):
        h.zero_()
        g.replay()
        assert torch.equal(h, want)


@pytest.mark.parametrize("M,K,N", [(300, 4096, 256), (600, 2048, 600), (100, 8192, 512), (64, 5120, 1280), (256, 1024, 1024), (33, 512, 64), (2000, 512, 1024),
                                   (130, 1368, 2056), (5000, 72, 1544), (17, 40, 8)])
def test_every_kind_of_tile(M, K, N):
    """Single CTAs, pairs, parts of K; more segments than a warp has lanes; a tail of every kind."""
    for n, rank, dtype in ((3, 24, BF16), (min(M, 70), 128, FP16)):
        borders = sorted({0, M} | {(i * M) // n + (i % 3 if (i * M) // n + i % 3 < M else 0) for i in range(1, n)})
        which = [i % 5 - 1 for i in range(len(borders) - 1)]
        x, w = rnd((M, K), 1, dtype), rnd((N, K), 2, dtype, K ** -0.5)
        a, b = rnd((4, rank, K), 3, dtype, K ** -0.5), rnd((4, N, rank), 4, dtype, rank ** -0.5)
        bias, y = rnd((N,), 5, FP32), torch.full((M, N + 8), 7.0, dtype=dtype, device="cuda")
        ws = torch.full((dt.dt_adapter_workspace_bytes(M, rank),), 0xFF, dtype=torch.uint8, device="cuda")
        dt.dt_adapter_linear(x, w, y[:, :N], a, b, ints(borders), ints(which), ws, bias=bias)
        dt.dt_poll_ops()
        check(y[:, :N], *ref.linear(x, w, bias, a, b, None, borders, which), (M, K, N, n))
        assert (y[:, N:] == 7).all()
        dt.dt_adapter_linear(x, w, y[:, :N], None, None, None, None, None)
        check(y[:, :N], *ref.linear(x, w, None, None, None, None, [], []), (M, K, N, "alone"))


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("L,H,D", [(5, 2, 64), (300, 24, 64), (300, 24, 128)])
@pytest.mark.parametrize("cap", [0.5, 40.0])
def test_what_stands_at_keys_that_do_not_count_has_no_effect_on_capped_logits(L, H, D, cap, value):
    """Products beyond and within the polynomial's reach; whole tiles and parts of them."""
    q, k, v = (rnd((2, L + 30, H, D), s, BF16) for s in (1, 2, 3))
    lens = [L, L // 2]
    clean = [t.clone() for t in (k, v)]
    for b, n in enumerate(lens):
        for t, c in zip((k, v), clean):
            t[b, n:], c[b, n:] = value, 0
    for causal in (False, True):
        out, lse = torch.empty_like(q), torch.empty((2, H, L + 30), device="cuda")
        want, want_lse = torch.empty_like(q), torch.empty_like(lse)
        kw = dict(causal=causal, softcap=cap, q_lens=ints(lens), key_lens=ints(lens))
        for o in (out, want):
            o.zero_()
        lse.zero_(), want_lse.zero_()
        dt.dt_packed_attn(q, k, v, out, D ** -0.5, lse_out=lse, **kw)
        dt.dt_packed_attn(q, *clean, want, D ** -0.5, lse_out=want_lse, **kw)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        docs = [[(0, n, 0, n, 0)] for n in lens]
        o, l, tol, tol_l, rows = ref.attention(q, *clean, D ** -0.5, docs, causal=causal, softcap=cap)
        check(out[rows], o[rows], tol[rows], "out")
        r = rows[:, None].expand_as(l)
        check(lse[r], l[r], tol_l[r], "lse")


@pytest.mark.parametrize("far", [1.0, 30.0])
def test_slopes_of_either_side_and_far_from_the_diagonal(far):
    """Biases linear in the column, before and behind the rows; slopes of both signs, whose bias then grows with the distance."""
    L, H = 1200, 24
    q, k, v = (rnd((1, L, H, 64), s, BF16) for s in (1, 2, 3))
    slopes = torch.linspace(-0.02, 0.5, H, device="cuda") * far
    out, lse = torch.empty_like(q), torch.empty((1, H, L), device="cuda")
    dt.dt_packed_attn(q, k, v, out, 0.125, bias_slopes=slopes, lse_out=lse)
    o, l, tol, tol_l, _ = ref.attention(q, k, v, 0.125, [[(0, L, 0, L, 0)]], slopes=slopes)
    check(out, o, tol, "out")
    check(lse, l, tol_l, "lse")


def test_many_small_documents():
    """More blocks than find a place at once: blocks of one and of two warps."""
    for L, n, H in ((14, 12, 40), (30, 25, 40), (60, 55, 40), (64, 20, 64)):
        at = [(i * L) // n for i in range(n + 1)]
        for causal in (False, True):
            q, k, v = (rnd((3, L, H, 128), s, FP16) for s in (1, 2, 3))
            out, lse = torch.empty_like(q), torch.empty((3, H, L), device="cuda")
            st = ints([at] * 3)
            dt.dt_packed_attn(q, k, v, out, 0.1, causal=causal, softcap=5.0, q_starts=st, k_starts=st, lse_out=lse)
            o, l, tol, tol_l, _ = ref.attention(q, k, v, 0.1, [[(a, b, a, b, 0) for a, b in zip(at, at[1:])]] * 3, causal=causal, softcap=5.0)
            check(out, o, tol, (L, n, causal))
            check(lse, l, tol_l, (L, n, causal))


@pytest.mark.parametrize("B,H,Hk,D", [(1, 2, 1, 64), (2, 8, 4, 128), (2, 40, 8, 64), (3, 20, 5, 128), (1, 20, 20, 128), (5, 8, 8, 64)])
def test_few_tokens_of_few_heads_behind_many_keys(B, H, Hk, D):
    """Clusters of every size and both numbers of warps, with lengths that leave some of them without keys."""
    L = 9001
    k, v = rnd((B, L, Hk, D), 1, BF16), rnd((B, L, Hk, D), 2, BF16)
    lens = [L, 40, 5000, 0, 8192][:B]
    for Lq in (1, 3):
        q = rnd((B, Lq, H, D), 3 + Lq, BF16, 2.0)
        for kw in (dict(), dict(softcap=20.0), dict(bias_slopes=2.0 ** -torch.arange(1.0, H + 1, device="cuda"))):
            out, lse = torch.empty_like(q), torch.empty((B, H, Lq), device="cuda")
            dt.dt_packed_attn(q, k, v, out, D ** -0.5, causal=True, key_lens=ints(lens), lse_out=lse, **kw)
            extra = dict(softcap=kw.get("softcap", 0.0), slopes=kw.get("bias_slopes"))
            o, l, tol, tol_l, _ = ref.attention(q, k, v, D ** -0.5, [[(0, Lq, 0, n, 0)] for n in lens], causal=True, **extra)
            check(out, o, tol, (Lq, lens, "out"))
            check(lse, l, tol_l, (Lq, lens, "lse"))
