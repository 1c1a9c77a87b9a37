"""Plain 64-bit forms of the operators around the self-attention, and the error their kernels may have: derived from the
roundings that the kernels make (half a step of the type each, torch.finfo(t).eps / 2 relative) and fp32's."""
import math

import torch

U32 = 2.0 ** -24


def rope(x, angle, layout_half, r, factor=1.0, transpose=False):
    """x [B, L, H, D], angle fp64 [B, L, r / 2] -> (fp64 result, tolerance)."""
    xf = x.double()
    c, s = angle.cos()[:, :, None] * factor, angle.sin()[:, :, None] * factor * (-1 if transpose else 1)
    i = torch.arange(r // 2, device=x.device)
    ia, ib = (i, i + r // 2) if layout_half else (2 * i, 2 * i + 1)
    a, b = xf[..., ia], xf[..., ib]
    out, tol = xf.clone(), torch.zeros_like(xf)
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    # fp32: sine and cosine each within 2^-22 or so (the argument's rounding at half a turn included), three roundings
    t = (a.abs() + b.abs()) * abs(factor) * 16 * U32
    tol[..., ia], tol[..., ib] = t, t
    eps = torch.finfo(x.dtype).eps / 2
    tol[..., :r] += out[..., :r].abs() * eps + torch.finfo(x.dtype).tiny * eps   # values past r are copied: exact
    return out, tol


def norm(x, weight, eps, residual):
    h = x.double() + (residual.double() if residual is not None else 0)
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, y * weight.double() if weight is not None else y


# relative error of y before its rounding: the sum's rounding, the sum of squares (a thread adds at most 32 of them and a
# tree joins the threads: under 64 roundings, halved by the root), the root's 2 ulp and two products
NORM_REL = (1 + 32 + 4 + 2) * U32


def cross(q, k, v, scale, keep=None):
    """q [B, Lq, H, D]; k, v [B, Lk, Hk, D]; keep bool [B, Lk] or None -> fp64 (out, lse, tol_out, tol_lse)."""
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    u = torch.finfo(q.dtype).eps / 2
    out = torch.zeros((B, Lq, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        keys = torch.arange(Lk, device=q.device) if keep is None else torch.nonzero(keep[b])[:, 0]
        if len(keys) == 0:
            continue
        for h in range(H):
            qq = q[b, :, h].double()
            kk, vv = k[b, keys, h // (H // Hk)].double(), v[b, keys, h // (H // Hk)].double()
            x = qq @ kk.T * scale
            lse[b, h] = torch.logsumexp(x, 1)
            p = (x - lse[b, h][:, None]).exp()
            out[b, :, h] = p @ vv
            # a logit's error: D products summed in fp32 (at most a step of the running sum per addition of 16), the scale's
            # and the base-2 reference's roundings
            top = (qq.abs() @ kk.abs().T * scale).amax(1)
            d_logit = top * (D / 16 + 8) * 2 * U32 + 4 * U32 * x.abs().amax(1)
            # sums over the keys in fp32 (serial in a lane for a part of them) and the exponentials' 2^-22
            d_sum = (8 + len(keys) / 8) * U32 + 8 * U32
            tol_lse[b, h] = d_logit + d_sum + 4 * U32 * (1 + lse[b, h].abs())
            rel = (u + 2 * d_logit + 2 * d_sum)[:, None]     # P is rounded to the inputs' type (u), as the output is
            tol[b, :, h] = (p @ vv.abs()) * rel * (1 + 1e-3) + out[b, :, h].abs() * u
            if q.dtype == torch.float16:   # P under 2^-14 has fp16's fixed step, half of which is 2^-25 of the largest P
                tol[b, :, h] += vv.abs().sum(0) * 2.0 ** -25 * p.amax(1, keepdim=True) + 2.0 ** -25
    return out, lse, tol, tol_lse
