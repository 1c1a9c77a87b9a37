"""Operators for several requests packed into one batch: a projection with every request's own low-rank adapter
(dt_adapter_linear), and attention within documents, with capped logits, biases by distance, causal and prefix masks
(dt_packed_attn), each in its plain form and as a call of this package.

listed() and draw() give cases, prepare() their inputs, run() makes one pass, exact() has the same outputs in 64 bits.
`own` decides whether run() computes the plain form or calls the package.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
CAP = 30.0              # where logits are capped
FAR = 128               # distances beyond it share the table's last entries

LARGEST_LINEAR = 75600 * 5120 * 5120
LARGEST_PAIRS = 40 * 128 * 17550 * 17551 // 2      # (query, key) pairs that count, times heads and values of a head


# ---------------------------------------------------------------------------------------------- cases
def linear_case(name, rows, K, N, rank, adapters, segments, dtype, bias):
    """`segments` requests behind one another in `rows` rows, each with one of `adapters` adapters or none."""
    c = dict(op="linear", rows=rows, K=K, N=N, rank=rank, adapters=adapters, segments=segments, dtype=dtype, bias=bias)
    return dict(c, name=name) if name else c


def attn_case(name, shape, B, docs, Lq, Lk, H, Hk, D, dtype, causal, prefix, cap, bias):
    """shape "packed": `docs` documents behind one another in each of B rows of Lq tokens; "padded": one per row, of lengths
    of their own; "cache": Lq new tokens of each request behind the keys that it has already."""
    c = dict(op="attn", shape=shape, B=B, docs=docs, Lq=Lq, Lk=Lk, H=H, Hk=Hk, D=D, dtype=dtype, causal=causal, prefix=prefix,
             cap=cap, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request through a narrow projection: latency only
        linear_case("linear one token", 1, 1536, 1536, 8, 2, 1, "bf16", False),
        # the next token of each of seven requests, five adapters: the weights are read once
        linear_case("linear a token each", 7, 5120, 5120, 16, 5, 7, "fp16", False),
        # the prompts of six requests on their way to keys, ragged lengths
        linear_case("linear prompts", 1807, 4096, 5120, 32, 4, 6, "bf16", True),
        # Wan's 1.3B width at 480p, three requests' latents
        linear_case("linear 480p", 32760, 1536, 1536, 24, 3, 3, "fp16", True),
        # Wan's 14B width at 720p, two requests' latents and a third without an adapter
        linear_case("linear 720p", 75600, 5120, 5120, 64, 2, 3, "bf16", True),
        # one new token of each of five prompts that are being written, heads in groups, capped logits: latency only
        attn_case("attn one token", "cache", 5, 1, 1, 512, 32, 8, 128, "bf16", True, False, True, "none"),
        # one new token of each of two requests with long histories, a slope per head
        attn_case("attn one token far", "cache", 2, 1, 1, 32760, 40, 8, 128, "fp16", True, False, False, "slopes"),
        # a text encoder over packed prompts: D = 64, a bias for each distance, both directions
        attn_case("attn packed prompts", "packed", 1, 9, 2011, 2011, 64, 64, 64, "bf16", False, False, False, "table"),
        # two padded sequences whose first third is seen by all their tokens, heads in groups, capped logits
        attn_case("attn prefix", "padded", 2, 1, 4441, 4441, 32, 8, 128, "bf16", True, True, True, "none"),
        # latents of three requests in one row (Wan's 1.3B at 480p in all)
        attn_case("attn packed 480p", "packed", 1, 3, 32760, 32760, 12, 12, 128, "bf16", False, False, False, "none"),
        # a long sequence, causal, a slope per head
        attn_case("attn long causal", "padded", 1, 1, 17550, 17550, 40, 40, 128, "fp16", True, False, False, "slopes"),
    ]


HEADS = [(2, 1), (4, 4), (12, 12), (16, 2), (32, 8), (32, 32), (40, 8), (40, 40), (64, 64)]   # (query heads, key heads)


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    dtype = rng.choice(["bf16", "fp16"])
    if rng.random() < 0.45:
        K, N = 8 * _log(rng, 16, 1024), 8 * _log(rng, 16, 1024)
        rows = _log(rng, 1, 16) if rng.random() < 0.35 else _log(rng, 17, max(17, min(75600, LARGEST_LINEAR // (K * N))))
        return linear_case(None, rows, K, N, rng.choice([8, 16, 16, 24, 32, 64, 72, 128]), rng.randint(1, 8), rng.randint(1, min(rows, 24)),
                           dtype, rng.random() < 0.5)
    D, (H, Hk), B = rng.choice([64, 128]), rng.choice(HEADS), rng.randint(1, 3)
    shape = rng.choice(["packed", "padded", "cache"])
    causal = shape == "cache" or rng.random() < 0.5
    more = dict(causal=causal, prefix=causal and rng.random() < 0.4, cap=rng.random() < 0.4, bias=rng.choice(["none", "table", "slopes"]))
    most = LARGEST_PAIRS // (B * H * D)
    if shape == "cache":
        Lq = _log(rng, 1, 8)
        return attn_case(None, shape, B, 1, Lq, _log(rng, Lq, min(40000, most // Lq)), H, Hk, D, dtype, **more)
    L = _log(rng, 2, min(32760, math.isqrt(most)))
    docs = rng.randint(1, min(12, L)) if shape == "packed" else 1
    return attn_case(None, shape, B, docs, L, L, H, Hk, D, dtype, **more)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(shape, seed, k, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000 + k)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _shares(total, parts, turn):
    """Borders of `parts` ragged pieces of 0 .. total, each of one at least."""
    weights = [1 + (5 * (i + turn)) % 7 for i in range(parts)]
    spare, borders, done = total - parts, [0], 0
    for i, w in enumerate(weights):
        done += w
        borders.append(i + 1 + spare * done // sum(weights))
    return borders


def _segments(case):
    """(borders, adapter of each segment); -1: none."""
    n = case["segments"]
    return _shares(case["rows"], n, 1), [-1 if i % 4 == 2 else i % case["adapters"] for i in range(n)]


def _documents(case):
    """For each request [(first query, end, first key, end, keys of the prefix)]."""
    B, Lq, Lk = case["B"], case["Lq"], case["Lk"]
    got = []
    for b in range(B):
        if case["shape"] == "packed":   # a few rows behind the last document are padding
            at = _shares(max(case["docs"], Lq - Lq // 50), case["docs"], b)
            docs = [(lo, hi, lo, hi) for lo, hi in zip(at, at[1:])]
        elif case["shape"] == "padded":
            n = max(1, Lq - Lq * b // (B + 1))
            docs = [(0, n, 0, n)]
        else:
            docs = [(0, Lq, 0, max(Lq, Lk - Lk * b // (B + 2)))]
        got.append([d + ((d[3] - d[2]) // 3 if case["prefix"] else 0,) for d in docs])
    return got


def _ints(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    if case["op"] == "linear":
        M, K, N, r, n = (case[k] for k in ("rows", "K", "N", "rank", "adapters"))
        borders, which = _segments(case)
        s.update(borders=borders, which=which, starts=_ints(borders), adapters_of=_ints(which))
        s.update(x=_randn((M, K), seed, 1, dt), weight=_randn((N, K), seed, 2, dt, K ** -0.5), a=_randn((n, r, K), seed, 3, dt, K ** -0.5),
                 b=_randn((n, N, r), seed, 4, dt, r ** -0.5), scales=0.25 + 0.5 * _randn((n,), seed, 5, torch.float32).abs(), bias=None)
        if case["bias"]:
            s["bias"] = _randn((N,), seed, 6, dt, 0.5)
        s["y"] = torch.empty((M, N), dtype=dt, device="cuda")
        s["workspace"] = None      # made in the first pass, by the package's own measure
        return s
    B, Lq, Lk, H, Hk, D = (case[k] for k in ("B", "Lq", "Lk", "H", "Hk", "D"))
    docs = _documents(case)
    s.update(q=_randn((B, Lq, H, D), seed, 1, dt, 1.3), k=_randn((B, Lk, Hk, D), seed, 2, dt, 1.3), v=_randn((B, Lk, Hk, D), seed, 3, dt),
             scale=(3.0 if case["cap"] else 1.0) / math.sqrt(D), documents=docs, table=None, slopes=None)
    s.update(out=torch.zeros_like(s["q"]), lse=torch.zeros((B, H, Lq), dtype=torch.float32, device="cuda"))
    s.update(starts=None, q_lens=None, key_lens=None, prefix_lens=None)
    if case["shape"] == "packed":
        s["starts"] = _ints([[d[0] for d in row] + [row[-1][1]] for row in docs])
    else:
        s["key_lens"] = _ints([row[0][3] for row in docs])
        if case["shape"] == "padded":
            s["q_lens"] = _ints([row[0][1] for row in docs])
    if case["prefix"]:
        s["prefix_lens"] = _ints([[d[4] for d in row] for row in docs])
    if case["bias"] == "table":         # 32 learned values per head; near distances have their own, far ones share
        d = torch.arange(-FAR, FAR + 1, device="cuda")
        n = d.abs()
        far = 8 + ((n.clamp_min(8).double() / 8).log() / math.log(FAR / 8) * 8).long().clamp_max(7)
        bucket = torch.where(n < 8, n, far) + 16 * (d > 0)
        s["table"] = _randn((H, 32), seed, 4, torch.float32)[:, bucket].contiguous()
    if case["bias"] == "slopes":
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(H, device="cuda", dtype=torch.float32) + 1) / H) + 0.001 * _randn((H,), seed, 4, torch.float32).abs()
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_linear(s):
    x = s["x"].float()
    y = x @ s["weight"].float().T
    for lo, hi, a in zip(s["borders"], s["borders"][1:], s["which"]):
        if a >= 0:
            y[lo:hi] += (x[lo:hi] @ s["a"][a].float().T * s["scales"][a]) @ s["b"][a].float().T
    if s["bias"] is not None:
        y += s["bias"].float()
    return [y.to(s["x"].dtype)]


def _plain_attn(s):
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    H, Hk, D = s["H"], s["Hk"], s["D"]
    for b, docs in enumerate(s["documents"]):
        for q0, q1, k0, k1, prefix in docs:
            nq, nk = q1 - q0, k1 - k0
            at = torch.arange(nq, device="cuda")[:, None] + (nk - nq)         # places among the keys
            key = torch.arange(nk, device="cuda")[None]
            keep = (key <= at) | (key < prefix) if s["causal"] else None
            step = max(1, (1 << 28) // (nq * nk))
            for h0 in range(0, H, step):
                heads = torch.arange(h0, min(H, h0 + step), device="cuda")
                q = s["q"][b, q0:q1, heads].float().transpose(0, 1)
                k, v = (s[n][b, k0:k1, heads // (H // Hk)].float().transpose(0, 1) for n in ("k", "v"))
                x = torch.matmul(q, k.transpose(1, 2)).mul_(s["scale"])
                if s["cap"]:
                    x = (x / CAP).tanh_().mul_(CAP)
                if s["table"] is not None:
                    x += s["table"][heads][:, (key - at).clamp(-FAR, FAR) + FAR]
                if s["slopes"] is not None:
                    x -= s["slopes"][heads, None, None] * (key - at).abs()
                if keep is not None:
                    x.masked_fill_(~keep, -math.inf)
                top = x.amax(-1, keepdim=True)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                p = x.sub_(top).exp_()
                total = p.sum(-1, keepdim=True)
                o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
                out[b, q0:q1, heads] = o.transpose(0, 1).to(out.dtype)
                lse[b, heads, q0:q1] = (top + total.log())[..., 0]
    return [out, lse]


def run(s):
    if not own:
        return _plain_linear(s) if s["op"] == "linear" else _plain_attn(s)
    from paper_2607_15650_b200 import binding as dt
    if s["op"] == "linear":
        if s["workspace"] is None:
            s["workspace"] = torch.empty(dt.dt_adapter_workspace_bytes(s["rows"], s["rank"]), dtype=torch.uint8, device="cuda")
        dt.dt_adapter_linear(s["x"], s["weight"], s["y"], s["a"], s["b"], s["starts"], s["adapters_of"], s["workspace"],
                             scales=s["scales"], bias=s["bias"])
        return [s["y"]]
    dt.dt_packed_attn(s["q"], s["k"], s["v"], s["out"], s["scale"], causal=s["causal"], softcap=CAP if s["cap"] else 0.0,
                      q_starts=s["starts"], k_starts=s["starts"], q_lens=s["q_lens"], key_lens=s["key_lens"],
                      prefix_lens=s["prefix_lens"], bias_table=s["table"], bias_slopes=s["slopes"], lse_out=s["lse"])
    return [s["out"], s["lse"]]


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "linear":
        M, K, N, r = (case[k] for k in ("rows", "K", "N", "rank"))
        borders, which = _segments(case)
        turned = sum(hi - lo for lo, hi, a in zip(borders, borders[1:], which) if a >= 0)
        used = len({a for a in which if a >= 0})
        return {"bytes": 2 * (M * K + N * K + M * N + used * r * (K + N) + (N if case["bias"] else 0)),
                "flops": 2 * M * K * N + 2 * turned * r * (K + N)}
    H, Hk, D = case["H"], case["Hk"], case["D"]
    queries = keys = pairs = 0
    for docs in _documents(case):
        for q0, q1, k0, k1, prefix in docs:
            nq, nk = q1 - q0, k1 - k0
            queries, keys = queries + nq, keys + nk
            if not case["causal"]:
                pairs += nq * nk
            else:       # row i: the first nk - nq + i + 1 keys, or the prefix where that is more
                near = max(0, min(nq, prefix - (nk - nq)))
                pairs += near * prefix + sum(range(nk - nq + near + 1, nk + 1))
    more = 4 * H * (2 * FAR + 1) if case["bias"] == "table" else 4 * H if case["bias"] == "slopes" else 0
    return {"bytes": 4 * queries * H * D + 4 * keys * Hk * D + 4 * queries * H + more, "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_linear(s):
    """Every request's rows with one weight of its own, W + s B A."""
    bias = 0.0 if s["bias"] is None else s["bias"].double()
    y = torch.empty(s["y"].shape, dtype=torch.float64, device="cuda")
    w = s["weight"].double()
    for i, a in enumerate(s["which"]):
        rows = slice(s["borders"][i], s["borders"][i + 1])
        whole = w if a < 0 else torch.addmm(w, s["b"][a].double(), s["a"][a].double(), alpha=float(s["scales"][a]))
        y[rows] = torch.nn.functional.linear(s["x"][rows].double(), whole) + bias
    return [y]


def _exact_attn(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    group = s["H"] // s["Hk"]
    for b, docs in enumerate(s["documents"]):
        for q0, q1, k0, k1, prefix in docs:
            j = torch.arange(k1 - k0, device="cuda")
            for first in range(q0, q1, 4096):
                rows = slice(first, min(first + 4096, q1))
                i = torch.arange(rows.start, rows.stop, device="cuda") - q1 + (k1 - k0)
                distance = j - i[:, None]
                for h in range(s["H"]):
                    k, v = (s[n][b, k0:k1, h // group].double() for n in ("k", "v"))
                    x = s["q"][b, rows, h].double() @ k.T * s["scale"]
                    if s["cap"]:
                        x = CAP * torch.tanh(x / CAP)
                    if s["table"] is not None:
                        x += s["table"][h].double()[(distance + FAR).clamp(0, 2 * FAR)]
                    if s["slopes"] is not None:
                        x -= s["slopes"][h].double() * distance.abs()
                    if s["causal"]:
                        x[(distance > 0) & (j >= prefix)] = -math.inf
                    total = torch.logsumexp(x, 1)
                    lse[b, h, rows] = total
                    out[b, rows, h] = torch.where(total == -math.inf, 0.0, 1.0)[:, None] * (x - total.clamp_min(-1e300)[:, None]).exp_() @ v
    return [out, lse]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_linear(s) if case["op"] == "linear" else _exact_attn(s)
