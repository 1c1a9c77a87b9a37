"""The projection with low-rank adapters on the GPU against its plain 64-bit form, at the sizes, segments and values where it can
go wrong.  Tolerances: tests/packed_ops_reference.py."""
import threading

import pytest
import torch

from paper_2607_15650_b200 import binding as dt
from paper_2607_15650_b200 import build
from tests import packed_ops_reference as ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


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
    assert over.numel() == 0 or over.max() <= 0, (what, over.max().item(), (got - want).abs()[fine].max().item())


class Case:
    def __init__(self, M, K, N, r, n, starts, which, dtype, bias=None, scales=True, seed=0):
        self.x, self.w = rnd((M, K), seed, dtype), rnd((N, K), seed + 1, dtype, K ** -0.5)
        self.a, self.b = rnd((n, r, K), seed + 2, dtype, K ** -0.5), rnd((n, N, r), seed + 3, dtype, r ** -0.5)
        self.scales = rnd((n,), seed + 4, FP32) if scales else None
        self.bias = rnd((N,), seed + 5, bias) if bias else None
        self.starts, self.which = starts, which
        self.y = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
        self.d_starts, self.d_which = ints(starts), ints(which)
        self.ws = torch.full((dt.dt_adapter_workspace_bytes(M, r),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN, as far as it is read

    def call(self, **kw):
        dt.dt_adapter_linear(self.x, self.w, self.y, self.a, self.b, self.d_starts, self.d_which, self.ws, scales=self.scales, bias=self.bias, **kw)

    def want(self):
        return ref.linear(self.x, self.w, self.bias, self.a, self.b, self.scales, self.starts, self.which)

    def check(self, what=""):
        self.call()
        dt.dt_poll_ops()
        check(self.y, *self.want(), (what, self.x.shape, self.w.shape, self.a.shape, self.starts, self.which))


def borders(M, n, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return [0] + sorted(torch.randint(0, M + 1, (n - 1,), generator=g).tolist()) + [M]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 15, 16, 17, 63, 128, 129, 300])
@pytest.mark.parametrize("K,N,r", [(8, 8, 8), (72, 264, 24), (512, 256, 16), (1544, 520, 64), (200, 72, 128), (64, 1000, 72)])
def test_sizes(M, K, N, r, dtype):
    n = min(M, 3)
    Case(M, K, N, r, 4, borders(M, n, M + K), [(2 * s + M) % 4 for s in range(n)], dtype, bias=dtype if N % 16 else None, seed=M).check()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("M,K,N,r", [(1807, 1024, 1160, 32), (4000, 328, 2568, 8), (260, 5120, 640, 16), (19000, 264, 264, 48), (130, 8, 70000, 16)])
def test_larger_sizes_and_their_tiles(M, K, N, r, dtype):
    Case(M, K, N, r, 5, borders(M, 6, 3), [0, 4, -1, 2, 4, 1], dtype, bias=FP32, seed=9).check()


@pytest.mark.parametrize("M", [12, 16, 200, 520])
@pytest.mark.parametrize("name,starts,which", [
    ("no rows in any", [0, 0, 0], [0, 1]), ("empty ones between", [0, 3, 3, 3, 9, 9], [0, 1, 2, 0, 1]), ("rows before and behind", [2, 5, 10], [1, 2]),
    ("none has one", [0, 6, 12], [-1, -1]), ("not an adapter", [0, 4, 8, 12], [3, -7, 2 ** 30]), ("the same twice", [0, 4, 8, 12], [1, 1, 1]),
    ("beyond the rows", [-5, 4, 10 ** 9], [1, 2]), ("a row each", list(range(13)), [0, 1, 2, 0, 1, 2, -1, 0, 1, 2, 0, 1]),
])
def test_segments(M, name, starts, which):
    Case(M, 136, 200, 16, 3, starts, which, BF16, seed=2).check(name)


def test_a_segment_per_row_of_many_tiles_and_borders_at_tiles_ends():
    M = 700
    Case(M, 64, 136, 16, 7, list(range(M + 1)), [(3 * i) % 8 - 1 for i in range(M)], FP16, seed=1).check()
    Case(640, 320, 136, 40, 7, [0, 128, 256, 257, 383, 384, 512, 640], [0, 1, 2, 3, -1, 5, 6], BF16, seed=1).check()


@pytest.mark.parametrize("M", [5, 90])
def test_without_adapters_and_with_none_of_the_options(M):
    c = Case(M, 256, 264, 16, 2, [0, M], [1], BF16, scales=False)
    c.check()
    c.a = c.b = None
    dt.dt_adapter_linear(c.x, c.w, c.y, None, None, None, None, None, bias=rnd((264,), 4, BF16))
    check(c.y, *ref.linear(c.x, c.w, rnd((264,), 4, BF16), None, None, None, [], []), "alone")
    e = torch.empty
    dt.dt_adapter_linear(c.x, c.w, c.y, e((0, 16, 256), dtype=BF16, device="cuda"), e((0, 264, 16), dtype=BF16, device="cuda"), ints([0, M]), ints([0]),
                         e(0, dtype=torch.uint8, device="cuda"))
    check(c.y, *ref.linear(c.x, c.w, None, None, None, None, [], []), "no adapters")


@pytest.mark.parametrize("M", [0, 6, 140])
def test_rows_and_weights_with_strides_and_leading_dimensions(M):
    K, N, r = 136, 200, 16
    c = Case(2 * M, K, N, r, 2, [0, M, 2 * M], [0, 1], FP16)
    big_x, big_w, big_y = rnd((2, M, K + 72), 1, FP16), rnd((N, K + 8), 2, FP16, 0.1), torch.full((2, M, N + 24), 7.0, dtype=FP16, device="cuda")
    x, w, y = big_x[..., 64:64 + K], big_w[:, :K], big_y[..., 8:8 + N]
    before = big_y.clone()
    dt.dt_adapter_linear(x, w, y, c.a, c.b, c.d_starts, c.d_which, c.ws, scales=c.scales)
    check(y.reshape(2 * M, N), *ref.linear(x.reshape(2 * M, K), w, None, c.a, c.b, c.scales, c.starts, c.which), "views")
    assert torch.equal(big_y[..., :8], before[..., :8]) and torch.equal(big_y[..., 8 + N:], before[..., 8 + N:])


@pytest.mark.parametrize("M,starts", [(9, [0, 3, 6, 9]), (300, [0, 60, 130, 300])])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_broken_adapter_or_row_reaches_no_other(M, starts, value):
    c = Case(M, 200, 264, 24, 3, starts, [0, 1, -1], BF16)
    clean = Case(M, 200, 264, 24, 3, starts, [0, 1, -1], BF16)
    clean.call()
    c.a[1, 3, 5] = c.b[1, 7, 2] = value
    c.b[2] = value                       # nobody's
    c.x[1] = value
    c.call()
    lo, hi = starts[1], starts[2]
    other = [i for i in range(M) if not lo <= i < hi and i != 1]
    assert torch.equal(c.y[other], clean.y[other])
    assert not torch.isfinite(c.y[lo:hi]).all() and not torch.isfinite(c.y[1]).any()


def test_the_same_inputs_give_the_same_bits_and_the_workspace_may_hold_anything():
    for M in (11, 500):
        c = Case(M, 520, 520, 32, 3, borders(M, 4, 2), [0, 2, 1, 0], FP16, bias=FP16)
        c.call()
        first = c.y.clone()
        for fill in (0, 0x7F):
            c.ws.fill_(fill)
            c.y.zero_()
            c.call()
            assert torch.equal(c.y, first)


def test_graphs_streams_and_threads():
    cases = [Case(M, 256, 264, 16, 3, borders(M, 3, 1), [0, 2, 1], BF16, seed=M) for M in (4, 16, 130, 400)]
    want = []
    for c in cases:
        c.call()
        want.append(c.y.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for c in cases:
            c.call()
            c.call()
    for _ in range(3):
        for c in cases:
            c.y.zero_()
        g.replay()
        for c, w in zip(cases, want):
            assert torch.equal(c.y, w)
    for c in cases:
        c.x.mul_(2.0)            # the graph sees new inputs
    g.replay()
    for c in cases:
        check(c.y, *c.want(), "replayed on new inputs")
        c.x.mul_(0.5)
        c.y.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]

    def work(c, s):
        with torch.cuda.stream(s):
            for _ in range(20):
                c.call()
    threads = [threading.Thread(target=work, args=z) for z in zip(cases, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.y, w)
    c = cases[2]
    c.y.zero_()
    torch.cuda.synchronize()
    c.call(stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(c.y, want[2])


def test_calls_in_a_row_over_one_workspace():
    """The next call's adapters' products may only take the workspace's place once the projection before has read it."""
    cases = [Case(400, 128, 1160, 64, 2, [0, 200, 400], [i % 2, 1], BF16, seed=i) for i in range(4)]
    for c in cases:
        c.ws = cases[0].ws
    for _ in range(5):
        for c in cases:
            c.call()
    for c in cases:
        check(c.y, *c.want(), "shared")


def test_offsets_beyond_32_bits():
    M, K, N = 70000, 64, 72
    big = torch.zeros((M, 32768), dtype=BF16, device="cuda")       # rows 64 KiB apart: 4.6 GB
    x = big[:, :K]
    x.copy_(rnd((M, K), 1, BF16))
    c = Case(16, K, N, 16, 2, [0, M - 200, M], [0, 1], BF16)
    y = torch.empty((M, N), dtype=BF16, device="cuda")
    ws = torch.empty(dt.dt_adapter_workspace_bytes(M, 16), dtype=torch.uint8, device="cuda")
    dt.dt_adapter_linear(x, c.w, y, c.a, c.b, c.d_starts, c.d_which, ws, scales=c.scales)
    want, tol = ref.linear(x.contiguous(), c.w, None, c.a, c.b, c.scales, c.starts, c.which)
    check(y, want, tol, "far rows")


def test_a_thread_whose_first_call_is_an_operator():
    """Also the cross attention's tiles, which make tensor maps as well."""
    c = Case(300, 64, 72, 16, 2, [0, 300], [1], BF16)
    q, k = rnd((1, 600, 12, 128), 1, BF16), rnd((1, 2048, 12, 128), 2, BF16)
    out = torch.empty_like(q)
    s = torch.cuda.current_stream()
    torch.cuda.synchronize()
    failed = []

    def work(f):
        try:
            f()
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    for f in (lambda: c.call(stream=s), lambda: dt.dt_cross_attn(q, k, k, out, 0.1, stream=s)):
        t = threading.Thread(target=work, args=(f,))
        t.start()
        t.join()
    assert not failed
    check(c.y, *c.want(), "from a thread")
