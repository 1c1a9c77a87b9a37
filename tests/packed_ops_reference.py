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
