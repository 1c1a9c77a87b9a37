"""Attention within documents on the GPU against its plain 64-bit form, at the sizes, masks, biases and values where it can go wrong.
Tolerances: tests/packed_ops_reference.py."""
import math
import threading

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
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()]), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, (what, over.max().item(), (got - want).abs()[fine].max().item())


class Case:
    """borders: (q_starts, k_starts) per row of the batch; else lengths (q_lens, key_lens) or None."""

    def __init__(self, B, Lq, Lk, H, Hk, D, dtype, *, borders=None, lens=None, causal=False, prefix=None, softcap=0.0, far=None, slopes=False,
                 scale=None, seed=0, lse=True):
        self.q, self.k, self.v = rnd((B, Lq, H, D), seed, dtype, 1.3), rnd((B, Lk, Hk, D), seed + 1, dtype, 1.3), rnd((B, Lk, Hk, D), seed + 2, dtype)
        self.out, self.lse = torch.full_like(self.q, 7), torch.full((B, H, Lq), 7.0, device="cuda") if lse else None
        self.scale = scale or D ** -0.5
        self.kw = dict(causal=causal, softcap=softcap)
        self.ref = dict(causal=causal, softcap=softcap)
        clamp = lambda x, n: min(max(x, 0), n)  # noqa: E731
        if borders:
            self.kw.update(q_starts=ints([x[0] for x in borders]), k_starts=ints([x[1] for x in borders]))
            self.docs = [[(clamp(a, Lq), max(clamp(b, Lq), clamp(a, Lq)), clamp(c, Lk), max(clamp(d, Lk), clamp(c, Lk)))
                          for a, b, c, d in zip(qs, qs[1:], ks, ks[1:])] for qs, ks in borders]
        else:
            ql, kl = lens or (None, None)
            if ql:
                self.kw["q_lens"] = ints(ql)
            if kl:
                self.kw["key_lens"] = ints(kl)
            self.docs = [[(0, clamp(ql[b], Lq) if ql else Lq, 0, clamp(kl[b], Lk) if kl else Lk)] for b in range(B)]
        if prefix:
            self.kw["prefix_lens"] = ints(prefix)
        self.docs = [[d + (clamp(prefix[b][i], d[3] - d[2]) if prefix else 0,) for i, d in enumerate(row)] for b, row in enumerate(self.docs)]
        if far is not None:
            self.kw["bias_table"] = self.ref["table"] = rnd((H, 2 * far + 1), seed + 3, FP32)
        if slopes:
            self.kw["bias_slopes"] = self.ref["slopes"] = 2.0 ** (-8 * (torch.arange(H, device="cuda", dtype=FP32) + 1) / H)

    def call(self, **kw):
        dt.dt_packed_attn(self.q, self.k, self.v, self.out, self.scale, lse_out=self.lse, **self.kw, **kw)

    def check(self, what="", call=True):
        out, lse, tol, tol_lse, rows = ref.attention(self.q, self.k, self.v, self.scale, self.docs, **self.ref)
        if call:
            self.call()
            dt.dt_poll_ops()
        what = (what, self.q.shape, self.k.shape, self.docs, {k: v for k, v in self.kw.items() if not torch.is_tensor(v)})
        out[~rows], tol[~rows] = 7, 0         # rows in no document are left as they were
        check(self.out, out, tol, (what, "out"))
        if self.lse is not None:
            r = rows[:, None].expand_as(lse)
            lse[~r], tol_lse[~r] = 7, 0
            check(self.lse, lse, tol_lse, (what, "lse"))


KINDS = [dict(), dict(softcap=5.0), dict(far=128), dict(slopes=True), dict(softcap=20.0, far=3), dict(softcap=2.0, slopes=True)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Lq,Lk,H,Hk", [(1, 1, 2, 2), (1, 333, 4, 1), (3, 50, 6, 2), (7, 2000, 2, 2), (200, 200, 2, 2), (257, 513, 4, 2), (640, 640, 3, 1)])
def test_lengths_heads_and_kinds(Lq, Lk, H, Hk, causal, kind, D, dtype):
    Case(2, Lq, Lk, H, Hk, D, dtype, causal=causal, seed=Lq, **kind).check()


MANY = dict(H=24, Hk=24)      # heads enough for the tiles


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal,prefix", [(False, None), (True, None), (True, 150)])
def test_tiles_of_many_heads(D, kind, causal, prefix):
    Case(2, 520, 700, **MANY, D=D, dtype=BF16, causal=causal, prefix=prefix and [[prefix], [700]], seed=4, **kind).check()


@pytest.mark.parametrize("far", [0, 1, 64, 200, 512])
@pytest.mark.parametrize("Lq,Lk", [(1, 1500), (40, 1500), (1400, 1500), (1500, 300)])
def test_tables_of_any_reach(Lq, Lk, far):
    Case(1, Lq, Lk, 8, 8, 64, FP16, far=far, seed=far).check()
    Case(1, Lq, Lk, 8, 2, 128, BF16, far=far, causal=True, seed=far).check()


def pieces(total, n, seed, spare=0):
    g = torch.Generator()
    g.manual_seed(seed)
    return [0] + sorted(torch.randint(0, total - spare + 1, (n - 1,), generator=g).tolist()) + [total - spare]


@pytest.mark.parametrize("H,Hk,D", [(2, 2, 64), (20, 20, 128), (16, 2, 64)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,L", [(1, 300), (2, 5), (9, 2011), (40, 777), (300, 900)])
def test_packed_documents(n, L, causal, H, Hk, D):
    """Some are empty, some of one token; a few rows behind the last are left as they were."""
    at = pieces(L, n, n + L, L // 50)
    for kind in (dict(), dict(far=128)):
        Case(1, L, L, H, Hk, D, BF16, borders=[(at, at)], causal=causal, seed=n, prefix=[[(7 * i) % 19 for i in range(n)]] if causal else None, **kind).check()


@pytest.mark.parametrize("H,D", [(2, 64), (30, 64), (24, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_documents_whose_queries_and_keys_differ(H, D, causal):
    """New tokens behind cached ones, prompts beside latents, documents without keys, without queries, and with fewer keys than
    queries."""
    q = [[0, 3, 200, 200, 560, 600], [0, 0, 256, 512, 513, 590]]
    k = [[0, 400, 500, 560, 600, 600], [10, 10, 100, 110, 900, 999]]
    Case(2, 600, 1000, H, H, D, BF16, borders=list(zip(q, k)), causal=causal, seed=2).check()
    Case(2, 600, 1000, H, H, D, FP16, borders=list(zip(q, k)), causal=causal, prefix=[[5] * 5, [0, 1, 2, 3, 1000]], slopes=True, seed=3).check()


@pytest.mark.parametrize("starts", [[-5, 100, 10 ** 9], [0, 0, 0], [50, 60, 70]])
def test_borders_outside_the_rows_are_clamped(starts):
    for H in (2, 48):
        Case(1, 300, 300, H, H, 64, BF16, borders=[(starts, starts)], seed=1).check()


@pytest.mark.parametrize("H,D", [(3, 128), (40, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_padded_batches(H, D, causal):
    for ql, kl in (([0, 1, 300, 500], [0, 1, 300, 500]), (None, [0, 1, 2, 10 ** 6]), ([3, -1, 400, 10 ** 6], None), ([500, 200, 100, 1], [100, 500, 0, 7])):
        Case(4, 500, 500, H, H, D, FP16, lens=(ql, kl), causal=causal, prefix=[[3], [0], [250], [9]] if causal else None, seed=7).check()


def test_empty_calls_and_no_keys():
    Case(0, 5, 5, 2, 2, 64, BF16).call()
    Case(2, 0, 5, 2, 2, 64, BF16).call()
    for L, H in ((3, 2), (700, 40)):
        Case(2, L, 0, H, H, 64, BF16).check()
        Case(2, L, 0, H, H, 64, BF16, borders=[([0, 2, L], [0, 0, 0])] * 2, causal=True, lse=False).check()


@pytest.mark.parametrize("Lq,H", [(8, 4), (300, 20)])
def test_heads_that_share_keys(Lq, H):
    for Hk in (1, 2, H):
        Case(2, Lq, 400, H, Hk, 64, FP16, causal=True, far=16, seed=Hk).check()
    Case(1, 5, 300, 40, 1, 128, BF16, causal=True, slopes=True).check()       # more heads than a block's rows


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("H,Lq", [(2, 6), (40, 6), (24, 400)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_what_stands_at_keys_that_do_not_count_has_no_effect(H, Lq, value, dtype):
    """Other documents' keys, padding, and later keys of the own document; a row that has the key gets it."""
    for causal in (False, True):
        at = [0, Lq // 2, Lq]
        c = Case(1, Lq, Lq, H, H, 128, dtype, borders=[(at, at)], causal=causal, seed=5)
        c.v[0, Lq // 2 + 2, 0, 3] = value
        c.v[0, Lq // 2 + 2, 1, 100] = value
        c.v[0, Lq - 1, 0, 64] = value
        c.check((causal, "v"))
        c = Case(3, Lq, Lq + 40, H, H, 64, dtype, lens=([Lq, Lq - 3, 1], [Lq, Lq - 3, 1]), causal=causal, seed=6)
        for b, n in enumerate((Lq, Lq - 3, 1)):
            c.k[b, n:], c.v[b, n:] = value, value
        c.check((causal, "padding"))
    c = Case(1, Lq, Lq, H, H, 64, dtype, causal=True, far=4, seed=8)
    c.k[0, Lq - 1], c.v[0, Lq - 1] = value, value        # the last key: the last row alone has it
    c.call()
    out, lse, tol, tol_lse, _ = ref.attention(c.q[:, :-1], c.k[:, :-1], c.v[:, :-1], c.scale, [[(0, Lq - 1, 0, Lq - 1, 0)]], **c.ref)
    check(c.out[:, :-1], out, tol, "rows before")
    check(c.lse[:, :, :-1], lse, tol_lse, "rows before")


def test_broken_rows_stay_alone():
    for L, H in ((5, 4), (500, 20)):
        for kind in KINDS:
            c, clean = (Case(1, L, L, H, H, 64, BF16, causal=True, seed=1, **kind) for _ in range(2))
            clean.call()
            c.q[0, L // 2, 1] = NAN
            c.call()
            assert torch.isnan(c.out[0, L // 2, 1]).all()
            c.out[0, L // 2, 1] = clean.out[0, L // 2, 1]
            c.lse[0, 1, L // 2] = clean.lse[0, 1, L // 2]
            if "softcap" not in kind:
                assert torch.equal(c.out, clean.out) and torch.equal(c.lse, clean.lse)
            else:      # how tanh is evaluated may differ beside it
                c.q[0, L // 2, 1] = clean.q[0, L // 2, 1]
                c.check(call=False)


def test_large_logits_and_caps():
    for cap in (0.0, 1.0, 30.0, 1e-3, 1e4):
        for L, H in ((3, 2), (300, 40)):
            Case(1, L, 600, H, H, 64, BF16, softcap=cap, scale=4.0, seed=3).check()
            Case(1, L, 600, H, H, 64, FP16, softcap=cap, scale=0.02, causal=True, seed=3).check()


def test_a_table_that_bars_distances():
    """-inf in the table: a window; rows whose window holds no key have none."""
    for L, H in ((6, 2), (700, 24)):
        c = Case(1, L, L, H, H, 64, BF16, far=3, seed=1)
        c.kw["bias_table"][:, 0] = c.kw["bias_table"][:, 6] = -INF
        c.check("window")
        c.kw["bias_table"][1] = -INF
        c.check("a head without keys")


def test_the_cross_attention_without_any_option():
    q, k, v = rnd((2, 300, 12, 128), 1, BF16), rnd((2, 512, 12, 128), 2, BF16), rnd((2, 512, 12, 128), 3, BF16)
    a, b, la, lb = torch.empty_like(q), torch.empty_like(q), torch.empty((2, 12, 300), device="cuda"), torch.empty((2, 12, 300), device="cuda")
    dt.dt_packed_attn(q, k, v, a, 0.1, lse_out=la)
    dt.dt_cross_attn(q, k, v, b, 0.1, lse_out=lb)
    # two states of one sum: each within its own bound
    out, lse, tol, tol_lse, _ = ref.attention(q, k, v, 0.1, [[(0, 300, 0, 512, 0)]] * 2)
    check(a, out, tol, "packed")
    check(b, out, tol, "cross")
    check(la, lse, tol_lse, "packed")
    check(lb, lse, tol_lse, "cross")


@pytest.mark.parametrize("L,H", [(5, 4), (400, 20)])
def test_views_and_in_place(L, H):
    c = Case(2, L, L, H, H, 64, BF16, causal=True, slopes=True, seed=3)
    qkv = torch.full((2, L + 3, 3 * H, 64), NAN, dtype=BF16, device="cuda")       # one projection's output, rows behind the last
    for i, t in enumerate((c.q, c.k, c.v)):
        qkv[:, :L, i * H:(i + 1) * H] = t
    before = qkv.clone()
    q, k, v = (qkv[:, :L, i * H:(i + 1) * H] for i in range(3))
    dt.dt_packed_attn(q, k, v, q, c.scale, lse_out=c.lse, **c.kw)
    c.out = q
    c.check("in place", call=False)
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))  # noqa: E731
    assert same(qkv[:, L:], before[:, L:]) and same(qkv[:, :, H:], before[:, :, H:])
    k1 = c.k[:1].expand(2, L, H, 64)                                               # one request's keys for all
    v1 = c.v[:1].expand(2, L, H, 64)
    dt.dt_packed_attn(c.q, k1, v1, c.out, c.scale, lse_out=c.lse, **c.kw)
    out, lse, tol, tol_lse, _ = ref.attention(c.q, k1, v1, c.scale, c.docs, **c.ref)
    check(c.out, out, tol, "expanded")


def test_same_bits_graphs_streams_and_threads():
    cases = [Case(1, 3, 900, 8, 2, 128, BF16, causal=True, softcap=9.0), Case(2, 600, 600, 20, 20, 64, FP16, causal=True, far=128),
             Case(1, 900, 900, 12, 12, 128, BF16, borders=[([0, 100, 350, 800], [0, 100, 350, 800])], slopes=True)]
    want = []
    for c in cases:
        c.call()
        want.append((c.out.clone(), c.lse.clone()))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for c in cases:
            c.call()
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.out.fill_(7)
    g.replay()
    for c, w in zip(cases, want):
        assert torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1])
    torch.cuda.synchronize()

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
        assert torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1])


def test_offsets_beyond_32_bits():
    """Keys 64 KiB apart: 70000 of them lie over 4.6 GB."""
    L = 70000
    big = torch.zeros((1, L, 512, 64), dtype=BF16, device="cuda")
    k, v = big[:, :, :2], big[:, :, 2:4]
    k.copy_(rnd((1, L, 2, 64), 1, BF16, 1.3))
    v.copy_(rnd((1, L, 2, 64), 2, BF16))
    for Lq in (1, 700):
        q = rnd((1, Lq, 2, 64), 3, BF16, 1.3)
        out, lse = torch.empty_like(q), torch.empty((1, 2, Lq), device="cuda")
        dt.dt_packed_attn(q, k, v, out, 0.125, causal=True, lse_out=lse)
        w = ref.attention(q, k, v, 0.125, [[(0, Lq, 0, L, 0)]], causal=True)
        check(out, w[0], w[2], Lq)
        check(lse, w[1], w[3], Lq)


def test_many_items_of_every_length():
    """More items than SMs, so that a CTA's stream of tiles goes over items with one tile, many and none."""
    g = torch.Generator()
    g.manual_seed(3)
    lens = [int(x) for x in torch.randint(0, 700, (40,), generator=g)]
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    L = at[-1] + 5
    for kind in (dict(), dict(far=100, causal=True), dict(softcap=6.0, causal=True)):
        Case(1, L, L, 8, 4, 64, BF16, borders=[(at, at)], seed=1, **kind).check()


NO_KEYS = [dict(D=64), dict(D=128), dict(D=64, far=128), dict(D=128, far=20), dict(D=128, slopes=True), dict(D=64, softcap=6.0)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("kind", NO_KEYS)
def test_many_blocks_without_keys_behind_blocks_with_keys(kind, dtype):
    """Many times as many blocks of 256 rows as there are SMs, most of them without keys, so that a CTA takes over several of those in
    a row behind one with keys: OUT = 0 and LSE = -inf there."""
    # a padded batch one of whose requests has no keys; and with the blocks without keys first and last
    for keys in ([300, 0], [0, 300, 0]):
        B = len(keys)
        Case(B, 4096, 300, 64, 64, dtype=dtype, lens=(None, keys), seed=1, **kind).check("padded")
    # a long causal sequence over few keys, the blocks with keys first
    Case(1, 9001, 300, 40, 8, dtype=dtype, causal=True, seed=2, **kind).check("causal")
    # latents beside prompts, some of which are empty
    q = [0, 1500, 3100, 3100, 5200, 5201, 7000, 9000, 10500, 12000]
    k = [0, 130, 130, 130, 130, 130, 430, 430, 430, 600]
    for causal in (False, True):
        Case(1, 12100, 600, 40, 40, dtype=dtype, borders=[(q, k)], causal=causal, lse=causal, seed=3, **kind).check("prompts")


def test_blocks_without_keys_in_the_place_of_q():
    """Rows of a view are written and nothing beside them."""
    L, H = 5000, 40
    qkv = rnd((2, L + 3, 3 * H, 64), 1, BF16)
    before = qkv.clone()
    q, k, v = (qkv[:, :L, i * H:(i + 1) * H] for i in range(3))
    c = Case(2, L, L, H, H, 64, BF16, lens=([L, L - 5], [700, 0]), seed=1)
    c.q, c.k, c.v = (t.clone() for t in (q, k, v))
    dt.dt_packed_attn(q, k, v, q, c.scale, lse_out=c.lse, **c.kw)
    dt.dt_poll_ops()
    assert torch.equal(qkv[:, L:], before[:, L:]) and torch.equal(qkv[:, :, H:], before[:, :, H:]) and torch.equal(q[1, L - 5:], before[1, L - 5:L, :H])
    c.out = q.clone()
    c.out[1, L - 5:] = 7
    c.check("in place", call=False)


def test_blocks_without_keys_replayed():
    """Captured, with lengths that change between the replays."""
    L = 4096
    c = Case(2, L, 400, 64, 64, 64, FP16, lens=([L, L], [400, 0]), seed=4)
    c.call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call()
    for keys in ([400, 0], [0, 17], [0, 0], [1, 400]):
        c.kw["key_lens"].copy_(ints(keys))
        c.docs = [[(0, L, 0, n, 0)] for n in keys]
        c.out.fill_(7)
        c.lse.fill_(7)
        g.replay()
        dt.dt_poll_ops()
        c.check(keys, call=False)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("L,H,D", [(1, 2, 128), (3, 8, 64), (300, 40, 64), (300, 40, 128)])
@pytest.mark.parametrize("cap", [1e4, 1e6, 1e9, 1e20])
def test_caps_far_above_the_logits(cap, L, H, D, dtype):
    """A capped logit is off by a part of itself (2^-20), not of the cap; also beside a row whose logits come near the cap."""
    q, k, v = rnd((1, L, H, D), 1, dtype, 1.5), rnd((1, 600, H, D), 2, dtype, 1.5), rnd((1, 600, H, D), 3, dtype)
    scale, docs = 4 * D ** -0.5, [[(0, L, 0, 600, 0)]]
    table = rnd((H, 65), 4, FP32)
    for kw, extra in ((dict(), dict()), (dict(bias_table=table), dict(table=table))):
        o, l, _, _, _ = ref.attention(q, k, v, scale, docs, softcap=cap, **extra)
        # (so far below the cap the weights are those without one, and so is what the other roundings may do)
        _, _, tol, tol_l, _ = ref.attention(q, k, v, scale, docs, **extra)
        x = torch.einsum("blhd,bkhd->bhlk", q.double(), k.double()).abs().amax(-1) * scale
        tol_l = tol_l + 2.0 ** -20 * x
        tol = tol + 2 * 2.0 ** -20 * x.transpose(1, 2)[..., None] * v.double().abs().amax()
        out, lse = torch.empty_like(q), torch.empty((1, H, L), device="cuda")
        dt.dt_packed_attn(q, k, v, out, scale, softcap=cap, lse_out=lse, **kw)
        check(out, o, tol, "out")
        check(lse, l, tol_l, "lse")
        if cap == 1e4 and L > 1:
            near = q.clone()
            near[0, 1] = (near[0, 1].double() * (cap / x[0, :, 1, None])).to(dtype)
            dt.dt_packed_attn(near, k, v, out, scale, softcap=cap, lse_out=lse, **kw)
            rest = [i for i in range(L) if i != 1]
            check(out[:, rest], o[:, rest], tol[:, rest], "out beside")
            check(lse[:, :, rest], l[:, :, rest], tol_l[:, :, rest], "lse beside")
            assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_very_many_documents_of_very_many_heads():
    """Nearly all of them without rows: as many numbers of blocks of 256 rows as tiles go through, and more, which few-row blocks take."""
    docs = 65535
    for H, Hk, Lq in ((256, 256, 512), (8192, 512, 64), (16384, 1024, 64)):
        at = [0] * 3 + [Lq // 3] * (docs - 5) + [Lq // 2] * 2 + [Lq - 1]
        assert len(at) == docs + 1
        q, k, v = rnd((1, Lq, H, 64), 1, BF16, 1.3), rnd((1, Lq, Hk, 64), 2, BF16, 1.3), rnd((1, Lq, Hk, 64), 3, BF16)
        out, lse = torch.full_like(q, 7), torch.full((1, H, Lq), 7.0, device="cuda")
        dt.dt_packed_attn(q, k, v, out, 0.125, q_starts=ints([at]), k_starts=ints([at]), lse_out=lse)
        dt.dt_poll_ops()
        heads = torch.arange(0, H, max(1, H // 32), device="cuda")      # of 32 heads
        some = [[(a, b, a, b, 0) for a, b in zip(at, at[1:]) if b > a]]
        o, l, tol, tol_l, rows = ref.attention(q[:, :, heads], k[:, :, heads // (H // Hk)], v[:, :, heads // (H // Hk)], 0.125, some)
        check(out[:, :, heads][rows], o[rows], tol[rows], "out")
        check(lse[:, heads][:, :, rows[0]], l[:, :, rows[0]], tol_l[:, :, rows[0]], "lse")
        assert (out[:, Lq - 1:] == 7).all() and (lse[:, :, Lq - 1:] == 7).all()
