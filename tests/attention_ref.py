"""Attention and group normalisation from their definitions, in 64 bits, and how far a kernel that sums in fp32 and rounds
its 16-bit operands and outputs may be from them. Plain torch, sequence by sequence and head by head."""
import math

import torch

BF16 = 2.0 ** -8  # half a step of a bf16 value, relative to it


def attention(q, k, v, lq, lk, y0, scale, cap=0.0, slopes=None, causal=False, prefix=None, q_at=None, k_at=None):
    """q [Mq, H, D], k, v [Mk, KV, D], y0 [Mq, H, D] (what y held before); lq, lk: lengths; q_at, k_at: first rows (default:
    one behind the other). Returns (y, tolerance), both [Mq, H, D] in 64 bits; tolerance -1 where nothing may change.

    The tolerance of y_i = sum_j w_j v_j, with A = sum_j w_j |v_j|, every term an upper bound:
      2^-8 |y|                     the output's rounding
      2^-8 A                       the weights' rounding to bf16
      (e^(2 dt) - 1) A             scores off by dt, in numerator and denominator: D fp32 additions of products, twice the
                                   half step for tensor cores that cut instead of rounding, scale times; eight roundings of
                                   the score's later forms; 2^-20 of the cap for its tanh
      (2^-13 + 2 Lk 2^-24) A       the exponential function, and fp32 sums of Lk terms
    """
    H, KV = q.shape[1], k.shape[1]
    y, tol = y0.double().clone(), torch.full(y0.shape, -1.0, dtype=torch.float64, device=y0.device)
    a = b = 0
    for s in range(len(lq)):
        if q_at is not None:
            a, b = q_at[s], k_at[s]
        nq, nk = lq[s], lk[s]
        dist = torch.arange(nq, device=q.device).view(-1, 1) + (nk - nq) - torch.arange(nk, device=q.device)
        hidden = torch.zeros_like(dist, dtype=torch.bool)
        if causal:
            hidden = (dist < 0) & (torch.arange(nk, device=q.device) >= (prefix[s] if prefix is not None else 0))
        for h in range(H):
            if nq == 0:
                continue
            qq, kk, vv = q[a:a + nq, h].double(), k[b:b + nk, h * KV // H].double(), v[b:b + nk, h * KV // H].double()
            t = qq @ kk.T * scale
            dt = scale * (q.shape[2] + 2) * 2.0 ** -23 * (qq.abs() @ kk.abs().T)
            if cap:
                t = cap * torch.tanh(t / cap)
                dt = dt + cap * 2.0 ** -20
            size = t.abs()
            if slopes is not None:
                bias = slopes[h].double() * dist.abs()
                t, size = t - bias, size + bias.abs()
            dt = (dt + 8 * 2.0 ** -24 * size).masked_fill(hidden, 0.0)
            t = t.masked_fill(hidden, -math.inf)
            w = torch.nan_to_num(torch.softmax(t, 1)) if nk else t  # (a row without a key: no weights)
            # a score that is far below the row's largest contributes nothing, however far off it is
            d = (dt * (w > 1e-9)).amax(1, keepdim=True) if nk else torch.zeros(nq, 1, dtype=torch.float64, device=q.device)
            vv = vv if nk else vv.view(0, q.shape[2])
            o, A = w @ vv, w @ vv.abs()
            y[a:a + nq, h] = o
            tol[a:a + nq, h] = BF16 * o.abs() + A * (BF16 + torch.expm1(2 * d) + 2.0 ** -13 + 2 * nk * 2.0 ** -24) * 1.01 + 1e-30
        a, b = a + nq, b + nk
    return y, tol


def group_norm(x, samples, rows, groups, gamma, beta, eps, silu):
    """x [samples * rows, C]. Returns (act(h), tolerance of its fp32 value), 64 bits.

    A group's sums add n values less a pivot p: at most K = 2 rows + 64 fp32 additions in a row (few are), so the mean is off
    by u (|mean - p| + std) and the variance by u (var + (mean - p)^2), u = K 2^-24, and h = (x - mean) rstd gamma + beta by
      |gamma| (u (1 + m) + |z| u (1 + m^2) + 4 2^-24 (|z| + m)) + 2 2^-24 |beta|,   z = (x - mean) rstd, m = |mean - p| rstd;
    the activation multiplies that by 1.1 at most and adds 2^-21 (2 + |h|) of its value."""
    C = x.shape[1]
    d = x.double().view(samples, rows, groups, C // groups)
    mean = d.mean((1, 3), keepdim=True)
    var = ((d - mean) ** 2).mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    z = ((d - mean) * rstd).reshape(samples * rows, C)
    m = ((mean - d[:, :1, :, :1]).abs() * rstd).expand_as(d).reshape(samples * rows, C)
    g = torch.ones(C, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(C, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    h = z * g + b
    u = (2 * rows + 64) * 2.0 ** -24
    tol = g.abs() * (u * (1 + m) + z.abs() * u * (1 + m * m) + 4 * 2.0 ** -24 * (z.abs() + m)) + 2 * 2.0 ** -24 * b.abs()
    if silu:
        y = h * torch.sigmoid(h)
        return y, 1.1 * tol + 2.0 ** -21 * (2 + h.abs()) * y.abs()
    return h, tol
