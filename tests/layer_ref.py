"""Plain 64-bit implementations of the recurrent layer's operators, each with a bound on what fp32
arithmetic may be off by (u = 2^-24 is one rounding of it)."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def conv(x, w, b, silu, first):
    """x [S, D], first [W-1, D] (double): y [S, D], the last W-1 inputs, bound on y."""
    W, S = w.shape[1], x.shape[0]
    seq = torch.cat([first, x])
    v, mag = b.repeat(S, 1), b.abs().repeat(S, 1)
    for j in range(W):
        v = v + seq[j:j + S] * w[:, j]
        mag = mag + (seq[j:j + S] * w[:, j]).abs()
    # W roundings of partial sums, each at most the sum of magnitudes
    err = (W + 1) * U * mag
    if silu:
        # slope of v sigmoid(v) below 1.1; exp at 3 + |v| roundings (argument times log2 e), times a
        # derivative of the sigmoid by it below 1/4 |v|; reciprocal and product two more
        y = v * sigmoid(v)
        err = 1.1 * err + U * (y.abs() * 6 + v.abs() * (1 + v.abs()) * sigmoid(-v.abs()) * 2)
    else:
        y = v
    return y, seq[S:], err


def scan(x, dt, bm, cm, z, A, dtb, skip, h, steps=None):
    """One sequence: x, dt, z [S, D] (z or None), bm, cm [S, D, N], h [D, N]: y, h, bounds on both."""
    S = x.shape[0]
    mag, err = h.abs(), torch.zeros_like(h)
    ys, es = [], []
    cut = S if steps is None else steps
    for t in range(S):
        v = dt[t] + dtb
        d = torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))
        # softplus: the sum dt + bias rounded once (slope at most 1, relative slope at most 1 below zero),
        # the exponential, the quotient and the series some ten roundings of the result
        dd = U * (v.abs() * torch.minimum(torch.ones_like(d), 1.3 * d) + 12 * d)
        e = d[:, None] * A
        a = torch.exp(e)
        u = (d * x[t])[:, None] * bm[t]
        # relative to a: the error of d, three roundings of the exponent (a cut of the axis sums up to `cut`
        # of them), two of the power; products and the sum: four more
        err = a * err + a * mag * ((dd[:, None] * A).abs() + U * ((3 + cut) * e.abs() + 4)) \
            + (dd * x[t].abs())[:, None] * bm[t].abs() + 4 * U * u.abs()
        h, mag = a * h + u, a * mag + u.abs()
        y = (cm[t] * h).sum(1) + skip * x[t]
        ym = (cm[t].abs() * mag).sum(1) + (skip * x[t]).abs()
        ye = (cm[t].abs() * err).sum(1) + (A.shape[1] + 4) * U * ym
        if z is not None:
            g = z[t] * sigmoid(z[t])
            ye = ye * g.abs() + (y.abs() + ye) * U * (g.abs() * 6 + z[t].abs() * (1 + z[t].abs()) * sigmoid(-z[t].abs()) * 2)
            y = y * g
        ys.append(y)
        es.append(ye)
    if not ys:
        return x.new_zeros(0, x.shape[1]), h, x.new_zeros(0, x.shape[1]), err
    return torch.stack(ys), h, torch.stack(es), err


def quantise(w, axis):
    """8-bit whole numbers (as int64) and scales (fp32) by the definition in fp32, with numpy."""
    w = np.asarray(w, np.float32)
    a = np.abs(w).max(axis=axis, keepdims=True)
    live = a >= np.float32(2.0 ** -100)
    r = np.where(live, np.float32(127) / np.where(live, a, np.float32(1)), np.float32(0)).astype(np.float32)
    q = np.rint((w * r).astype(np.float32)).astype(np.int64)
    return q, np.where(live, a / np.float32(127), np.float32(0)).astype(np.float32)


def product(x, W, bias):
    """y in 64 bits and a bound: the exact sum as fp32, two scales, the bias: four roundings."""
    qx, sx = quantise(x, 1)
    qw, sw = quantise(W, 0)
    p = (qx @ qw).astype(np.float64) * sw.astype(np.float64) * sx.astype(np.float64)
    y = p if bias is None else p + np.asarray(bias, np.float64)
    return y, 4 * U * (np.abs(p) + np.abs(y)) + 1e-44
