"""Plain 64-bit implementations of the attention layer's operators on the CPU, each with a bound on what fp32
arithmetic may be off by (u = 2^-24 is one rounding of it)."""
import math

import torch

U = 2.0 ** -24
LOG2E = math.log2(math.e)


def attention(q, k, v, seen, scale, weights_half_step=0.0):
    """q [n, D], k, v [L, D] (double), seen [n, L]: y [n, D] and a bound on it.  weights_half_step: half a step of the
    type that the softmax weights are rounded to before the products with the values (0: not rounded).

    A score is a sum of D products: D + 3 roundings of at most the sum of magnitudes A (in units of log2), its
    difference from the maximum two more of the largest score; the power turns an absolute error into a relative one
    times ln 2 and adds a few.  The sums over L keys, with the factors of a moving maximum, have L + 16 roundings each."""
    n, L = q.shape[0], k.shape[0]
    if L == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    k = torch.where(seen.any(0)[:, None], k, torch.zeros_like(k))
    v = torch.where(seen.any(0)[:, None], v, torch.zeros_like(v))
    s = (q @ k.T) * scale
    s = torch.where(seen, s, torch.full_like(s, float("-inf")))
    m = s.amax(1, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), torch.zeros_like(m), m))
    p = torch.where(seen, p, torch.zeros_like(p))
    w = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    A = torch.where(seen, (q.abs() @ k.abs().T) * (scale * LOG2E), torch.zeros_like(s)).amax(1, keepdim=True)
    eps_p = math.log(2) * U * ((q.shape[1] + 3) * A + 4 * A) + 8 * U
    err = (w @ v.abs()) * (2 * eps_p + weights_half_step + 4 * (L + 16) * U)
    return w @ v, err


def heads(q, k, v, seen, Hq, Hk, scale, weights_half_step=0.0):
    """q [n, Hq*D], k, v [L, Hk*D], seen [n, L]: y [n, Hq*D], bound."""
    D, G = q.shape[1] // Hq, Hq // Hk
    ys = [attention(q[:, h * D:(h + 1) * D], k[:, h // G * D:(h // G + 1) * D], v[:, h // G * D:(h // G + 1) * D], seen, scale,
                    weights_half_step) for h in range(Hq)]
    return torch.cat([y for y, _ in ys], 1), torch.cat([e for _, e in ys], 1)


def causal(first, n, L, window):
    """Which of L keys the queries of positions first .. first + n - 1 see."""
    p, j = torch.arange(first, first + n)[:, None], torch.arange(L)[None, :]
    return (j <= p) & (j > p - window if window else j >= 0)


def turn_heads(x, pos, D, norm, eps, gain, rot, pairs, freq):
    """Heads x [n, H*D] (double) at positions pos [n]: normalised, rotated; bound.

    The mean of squares has D + 1 roundings (half of them after the root), root, factor and gain some five.  An angle's
    turns are rounded once to 32 bits, below half a turn: 2^-26 of a turn, 1.6 u; sine and cosine two units of at most 1
    more; the products and the sum of a rotation three roundings of its two magnitudes."""
    n = x.shape[0]
    t = x.reshape(n, x.shape[1] // D, D).clone()
    e = torch.zeros_like(t)
    if norm:
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * gain
        e = t.abs() * U * ((D + 1) / 2 + 5)
    if rot:
        i = torch.arange(rot // 2)
        lo, hi = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        a = (pos.double()[:, None] * freq)[:, None, :]
        c, s, u, w = torch.cos(a), torch.sin(a), t[..., lo].clone(), t[..., hi].clone()
        mag = u.abs() + w.abs()
        err = e[..., lo] + e[..., hi] + mag * U * 8
        t[..., lo], t[..., hi] = u * c - w * s, w * c + u * s
        e[..., lo], e[..., hi] = err, err
    return t.reshape(x.shape), e.reshape(x.shape)


def advance(rows, row, add, page, n_blocks, n_pages):
    """Page tables row by row.  rows: (length, pages) of each; row, add: lists.  Returns (tables, lengths, free pages,
    copies (from, to, positions)), or None where there is no room."""
    out = [[0, []] if r < 0 else [rows[r][0], list(rows[r][1][:-(-rows[r][0] // page)])] for r in row]
    refs = [0] * n_pages
    for _, pages in out:
        for p in pages:
            refs[p] += 1
    free = [p for p in range(n_pages) if refs[p] == 0]
    copies = []
    for o, a in zip(out, add):
        n, pages = o
        if n + a > n_blocks * page:
            return None
        if a > 0 and n % page and refs[pages[-1]] > 1:
            if not free:
                return None
            refs[pages[-1]] -= 1
            copies.append((pages[-1], free[0], n % page))
            pages[-1] = free.pop(0)
        while len(pages) * page < n + a:
            if not free:
                return None
            pages.append(free.pop(0))
        o[0] = n + a
    return [o[1] for o in out], [o[0] for o in out], len(free), copies


def pack(rows, page):
    """(tables, used pages ascending) of rows (length, pages)."""
    pages = [r[1][:-(-r[0] // page)] for r in rows]
    used = sorted({p for r in pages for p in r})
    at = {p: i for i, p in enumerate(used)}
    return [[at[p] for p in r] for r in pages], used
