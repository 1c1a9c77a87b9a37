"""Plain 64-bit forms of the operators for packed requests, and the error their kernels may have: derived from the roundings that
the kernels make (half a step of the type each, torch.finfo(t).eps / 2 relative) and fp32's."""
import math

import torch

U32 = 2.0 ** -24


def sum_error(terms):
    """Relative to the sum of the terms' magnitudes: products are exact in fp32; the tensor cores add at most a step of the running
    sum for every 16 of them, the joins of parts and lanes a few more; every such addition may lose two halves of a step."""
    return (terms / 16 + 16) * 2 * U32


def linear(x, weight, bias, a, b, scales, starts, which):
    """x [M, K] -> fp64 (y, tolerance)."""
    u = torch.finfo(x.dtype).eps / 2
    M, K = x.shape
    xd, wd = x.double(), weight.double()
    y = xd @ wd.T
    tol = (xd.abs() @ wd.abs().T) * sum_error(K)
    if a is not None:
        adapters, r = a.shape[0], a.shape[1]
        for s in range(len(which)):
            lo, hi, i = max(0, starts[s]), min(M, starts[s + 1]), which[s]
            if lo >= hi or not 0 <= i < adapters:
                continue
            scale = 1.0 if scales is None else scales[i].double()
            ad, bd = a[i].double(), b[i].double()
            t = xd[lo:hi] @ ad.T * scale
            y[lo:hi] += t @ bd.T
            t_tol = (xd[lo:hi].abs() @ ad.abs().T) * abs(scale) * (sum_error(K) + 2 * U32)
            if M > 16:          # t is kept in x's type (half a step; fp16: half its fixed step near zero)
                t_tol = t_tol + t.abs() * u + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)
            tol[lo:hi] += t_tol @ bd.abs().T + ((t.abs() + t_tol) @ bd.abs().T) * sum_error(r)
    if bias is not None:
        y += bias.double()
        tol += bias.double().abs() * U32
    return y, tol * (1 + 2 * u) + y.abs() * (u + 2 * U32) + torch.finfo(x.dtype).tiny * u


def attention(q, k, v, scale, documents, causal=False, softcap=0.0, table=None, slopes=None):
    """q [B, Lq, H, D]; k, v [B, Lk, Hk, D]; documents[b] = [(q0, q1, k0, k1, prefix), ...] -> fp64 (out, lse, tol_out, tol_lse, bool
    [B, Lq]: rows in a document)."""
    B, Lq, H, D = q.shape
    rep = H // k.shape[2]
    u = torch.finfo(q.dtype).eps / 2
    out = torch.zeros((B, Lq, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    rows = torch.zeros((B, Lq), dtype=torch.bool, device=q.device)
    for b in range(B):
        for q0, q1, k0, k1, prefix in documents[b]:
            rows[b, q0:q1] = True
            if q1 <= q0 or k1 <= k0:
                continue
            place = torch.arange(q0, q1, device=q.device)[:, None] - q1 + k1 - k0
            key = torch.arange(k1 - k0, device=q.device)[None]
            keep = (key <= place) | (key < prefix) if causal else torch.ones((q1 - q0, k1 - k0), dtype=torch.bool, device=q.device)
            for h in range(H):
                qq, kk, vv = q[b, q0:q1, h].double(), k[b, k0:k1, h // rep].double(), v[b, k0:k1, h // rep].double()
                kk = torch.where(torch.isfinite(kk), kk, 0.0) if not torch.isfinite(kk).all() else kk
                x = qq @ kk.T * scale
                # a logit's error: D products summed in fp32 (at most a step of the running sum per addition of 16), the scale's and
                # the base-2 reference's roundings; a capped one's within 2^-21 of the cap; a bias' two roundings
                d_logit = ((qq.abs() @ kk.abs().T * scale) * keep).amax(1) * (D / 16 + 8) * 2 * U32
                if softcap:
                    x = softcap * torch.tanh(x / softcap)
                    d_logit = d_logit + softcap * 2.0 ** -21
                if table is not None:
                    far = table.shape[1] // 2
                    bias = table[h].double()[(key - place).clamp(-far, far) + far]
                if slopes is not None:
                    bias = -slopes[h].double() * (key - place).abs()
                if table is not None or slopes is not None:
                    x = x + bias
                    d_logit = d_logit + 4 * U32 * torch.where(keep & torch.isfinite(bias), bias.abs(), 0.0).amax(1)
                x = torch.where(keep, x, -math.inf)
                d_logit = d_logit + 4 * U32 * torch.where(torch.isfinite(x), x.abs(), 0.0).amax(1)
                total = torch.logsumexp(x, 1)
                lse[b, h, q0:q1] = total
                p = torch.where(total[:, None] == -math.inf, 0.0, (x - total[:, None].clamp_min(-1e300)).exp())
                clean = torch.where(torch.isfinite(vv), vv, 0.0)
                out[b, q0:q1, h] = p @ clean
                # what is not finite counts for the rows that have the key
                for j, d in torch.nonzero(~torch.isfinite(vv)).tolist():
                    out[b, q0:q1, h, d] += torch.where(keep[:, j], vv[j, d], 0.0)
                # sums over the keys in fp32 (serial in a lane for a part of them) and the exponentials' 2^-22
                d_sum = (8 + (k1 - k0) / 8) * U32 + 8 * U32
                tol_lse[b, h, q0:q1] = d_logit + d_sum + 4 * U32 * (1 + torch.where(total == -math.inf, 0.0, total.abs()))
                rel = (u + 2 * d_logit + 2 * d_sum)[:, None]     # P is rounded to the inputs' type (u), as the output is
                tol[b, q0:q1, h] = (p @ clean.abs()) * rel * (1 + 1e-3) + torch.nan_to_num(out[b, q0:q1, h], 0.0, 0.0, 0.0).abs() * u
                tol[b, q0:q1, h] += torch.finfo(q.dtype).tiny * u
                if q.dtype == torch.float16:   # P under 2^-14 has fp16's fixed step, half of which is 2^-25 of the largest P
                    tol[b, q0:q1, h] += clean.abs().sum(0) * 2.0 ** -25 * p.amax(1, keepdim=True) + 2.0 ** -25
    return out, lse, tol, tol_lse, rows
