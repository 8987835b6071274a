"""The selective scan at its edges: every length around a tile, within the bound of the roundings that are made
(none for pieces that are not there); infinite and NaN inputs at state counts that the kernels pad;
steps that keep and that forget the state."""
import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref
from paper_1804_00344_amd import mtstep as mt
from test_gpu_layer import DEV, check, dev, gen, per_channel, run_scan, scan_cell, scan_inputs
from test_layer_cpu import scan_pieces

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def piece_of(B, S, D, N):
    """Positions of the pieces that the axis is cut into (the last one shorter), or 0: one piece.  The cut is
    ceil(S / 2^k) up to whole tiles; of those that give the same count the longest."""
    n, tile = scan_pieces(B, S, D, N), 8 if N <= 128 else 4
    if n == 1:
        return 0
    lens = [-(-(-(-S // c)) // tile) * tile for c in (2 ** k for k in range(1, 9))]
    return max(l for l in lens if -(-S // l) == n)


def scan_bound(x, dt, bm, cm, z, A, dtb, skip, h, piece):
    """As layer_ref.scan, with only the roundings that are made.  Per position, relative to the power a: the error
    dd of D_t times |A|, three roundings of the exponent D_t A (A log2 e, the product, one spare), four of the
    power, the sum and the products.  Where a piece ends and another follows, the power of the whole piece, w = the
    sum of its D_t: `piece` roundings of w at most and two of joining its lanes, two of the product with A, three
    of the power and the sum, and one of the state.  z None: no gate."""
    U = ref.U
    mag, err = h.abs(), torch.zeros_like(h)
    ys, es = [], []
    w, mag0 = torch.zeros_like(dtb), mag
    S = x.shape[0]
    for t in range(S):
        v = dt[t] + dtb
        d = torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))
        dd = U * (v.abs() * torch.minimum(torch.ones_like(d), 1.3 * d) + 12 * d)
        e = d[:, None] * A
        a = torch.exp(e)
        u = (d * x[t])[:, None] * bm[t]
        err = a * err + a * mag * ((dd[:, None] * A).abs() + U * (3 * e.abs() + 4)) + (dd * x[t].abs())[:, None] * bm[t].abs() \
            + 4 * U * u.abs()
        h, mag = a * h + u, a * mag + u.abs()
        y = (cm[t] * h).sum(1) + skip * x[t]
        ye = (cm[t].abs() * err).sum(1) + (A.shape[1] + 4) * U * ((cm[t].abs() * mag).sum(1) + (skip * x[t]).abs())
        if z is not None:
            g = z[t] * ref.sigmoid(z[t])
            ye = ye * g.abs() + (y.abs() + ye) * U * (g.abs() * 6 + z[t].abs() * (1 + z[t].abs()) * ref.sigmoid(-z[t].abs()) * 2)
            y = y * g
        ys.append(y)
        es.append(ye)
        w = w + d
        if piece and (t + 1) % piece == 0 and t + 1 < S:
            wa = (w[:, None] * A).abs()
            err = err + torch.exp(-wa) * mag0 * U * ((piece + 4) * wa + 3) + U * mag
            w, mag0 = torch.zeros_like(dtb), mag
    return torch.stack(ys), h, torch.stack(es), err


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [3, 8, 16, 200])
def test_scan_of_every_length(N, dtype):
    """Prompts of 0 to 34 positions: each length modulo a tile, with one and more tiles before the last."""
    S, D, G = 34, 6, 2
    B = S + 1
    cell, A, dtb, skip = scan_cell(D, N, G, dtype)
    x, dt, z, bc = scan_inputs((B, S), D, N, G, dtype, N)
    for n in range(B):
        for t in (x, dt, z, bc):
            t[n, n:] = float("nan")
    st = torch.randn(B, D, N, generator=gen(9))
    lens = torch.arange(B, dtype=torch.int32, device=DEV)
    y, so = run_scan(cell, x, dt, z, bc, G * N, lens, dev(st))
    assert torch.equal(so[0].cpu(), st[0]) and bool((y[0] == 7.0).all())
    piece = piece_of(B, S, D, N)
    for n in range(1, B):
        want, h, ye, he = scan_bound(x[n, :n].double(), dt[n, :n].double(), per_channel(bc[n, :n], D, N, G, False),
                                     per_channel(bc[n, :n], D, N, G, True), z[n, :n].double(), A, dtb, skip, st[n].double(), piece)
        check(y[n, :n], want, ye, ("y", n))
        check(so[n], h, he, ("state", n))
        assert bool((y[n, n:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,D,N,cut", [(1, 700, 16, 16, True), (3, 530, 20, 5, True), (1, 600, 12, 100, True),
                                         (1, 400, 8, 250, True), (64, 60, 300, 16, False), (1, 8, 16, 24, False)])
def test_scan_within_the_bound_of_its_roundings(B, S, D, N, cut, dtype):
    piece = piece_of(B, S, D, N)
    assert bool(piece) == cut
    cell, A, dtb, skip = scan_cell(D, N, 1, dtype)
    x, dt, z, bc = scan_inputs((B, S), D, N, 1, dtype, S)
    st = torch.randn(B, D, N, generator=gen(9))
    y, so = run_scan(cell, x, dt, z, bc, N, None, dev(st))
    for b in (0, B - 1):
        want, h, ye, he = scan_bound(x[b].double(), dt[b].double(), per_channel(bc[b], D, N, 1, False),
                                     per_channel(bc[b], D, N, 1, True), z[b].double(), A, dtb, skip, st[b].double(), piece)
        check(y[b], want, ye, "y")
        check(so[b], h, he, "state")


def run_steps(cell, x, dt, z, bc, N, st):
    """The same prompts [1, S, ..] token by token."""
    ys, h = [], dev(st).clone()
    for t in range(x.shape[1]):
        y = torch.empty(1, cell.D, dtype=x.dtype, device=DEV)
        w = dev(bc[:, t].contiguous())
        mt.mt_ssm_step(cell, dev(x[:, t].contiguous()), dev(dt[:, t].contiguous()), w[:, :N], w[:, N:], y, h, h,
                       z=None if z is None else dev(z[:, t].contiguous()))
        ys.append(y)
    return torch.stack(ys, 1), h


@pytest.mark.parametrize("N", [1, 5, 16, 24, 100, 200])
@pytest.mark.parametrize("S", [6, 300])  # whole; cut into pieces
@pytest.mark.parametrize("which,value", [("x", float("inf")), ("x", float("-inf")), ("x", float("nan")), ("dt", float("inf")),
                                         ("dt", float("nan"))])
def test_infinite_inputs(which, value, S, N):
    """An infinite or NaN input makes of its channel what the formula makes of it, whether or not the states are
    padded: B and C are positive here, so that the formula's sums of infinities have a sign."""
    D, c, at = 8, 3, min(4, S - 2)
    cell, A, dtb, skip = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = scan_inputs((1, S), D, N, 1, "f32", 3)
    bc, z = bc.abs() + 0.1, z.abs() + 0.1
    (x if which == "x" else dt)[0, at, c] = value
    st = torch.randn(1, D, N, generator=gen(2))
    want, h, _, _ = ref.scan(x[0].double(), dt[0].double(), per_channel(bc[0], D, N, 1, False), per_channel(bc[0], D, N, 1, True),
                             z[0].double(), A, dtb, skip, st[0].double())
    wild = ~torch.isfinite(want)
    assert bool(wild[at:, c].all()) and not bool(wild[:, [d for d in range(D) if d != c]].any())
    forms = [run_scan(cell, x, dt, z, bc, N, None, dev(st))] + ([run_steps(cell, x, dt, z, bc, N, st)] if S < 10 else [])
    for y, so in forms:
        for got, w in ((y[0].cpu().double(), want), (so[0].cpu().double(), h)):
            assert torch.equal(torch.isnan(got), torch.isnan(w))
            assert torch.equal(got[torch.isinf(w)], w[torch.isinf(w)])
            fin = torch.isfinite(w)
            assert bool(((got - w)[fin].abs() <= 1e-4 * (1 + w[fin].abs())).all())


@pytest.mark.parametrize("N", [5, 16, 24, 200])
def test_steps_that_keep_and_forget_the_state(N):
    """dt far below zero is a step of zero, which keeps the state to the bit; a large one leaves nothing of it."""
    D, S, at = 8, 5, 2
    cell, A, dtb, skip = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = scan_inputs((1, S), D, N, 1, "f32", 3)
    st = torch.randn(1, D, N, generator=gen(2))
    _, before = run_scan(cell, *(t[:, :at].contiguous() for t in (x, dt, z, bc)), N, None, dev(st))
    bound = lambda n: scan_bound(x[0, :n].double(), dt[0, :n].double(), per_channel(bc[0, :n], D, N, 1, False),
                                 per_channel(bc[0, :n], D, N, 1, True), z[0, :n].double(), A, dtb, skip, st[0].double(), 0)
    kept = []
    for value in (-1e4, -3e38, float("-inf")):
        dt[0, at] = value
        y, after = run_scan(cell, *(t[:, :at + 1].contiguous() for t in (x, dt, z, bc)), N, None, dev(st))
        assert torch.equal(after, before)
        kept.append(y)
    assert torch.equal(kept[0], kept[1]) and torch.equal(kept[0], kept[2])
    dt[0, at] = -1e4
    want, _, ye, _ = bound(at + 1)
    check(kept[0][0], want, ye, "kept")
    # D A below -200 for every rate: the powers are below the smallest float
    dt[0, at] = 200 / float(A.abs().min()) + 10
    y, after = run_scan(cell, x, dt, z, bc, N, None, dev(st))
    want, h, ye, he = bound(S)
    check(y[0], want, ye, "forgotten")
    check(after[0], h, he, "state")
    other, after2 = run_scan(cell, x, dt, z, bc, N, None, dev(st * 3 + 1))  # from another state: nothing of it is left
    assert torch.equal(y[:, at:], other[:, at:]) and torch.equal(after, after2)
    dt[0, at] = 1e20
    y, after = run_scan(cell, *(t[:, :at + 1].contiguous() for t in (x, dt, z, bc)), N, None, dev(st))
    want, h, ye, he = bound(at + 1)
    check(y[0], want, ye, "large")
    check(after[0], h, he, "state")


@pytest.mark.parametrize("N", [5, 16])
def test_an_infinite_state_outlasts_a_piece(N):
    """Steps that each leave something of the state, but a whole piece of them less than the smallest float: an
    infinite state stays infinite over a cut axis, as it does position by position."""
    D, S, at, c = 8, 300, 4, 3
    assert piece_of(1, S, D, N)
    cell, A, dtb, skip = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = scan_inputs((1, S), D, N, 1, "f32", 3)
    bc, z = bc.abs() + 0.1, z.abs() + 0.1
    dt = (4 - dtb).float().expand(1, S, D).contiguous()  # D_t of 4.02: a power above e^-80, a piece's below e^-110
    assert float(-A.min()) * 4.02 < 80 and float(-A[c].min()) * 4 * piece_of(1, S, D, N) > 110
    x[0, at, c] = float("inf")
    want, h, _, _ = ref.scan(x[0].double(), dt[0].double(), per_channel(bc[0], D, N, 1, False), per_channel(bc[0], D, N, 1, True),
                             z[0].double(), A, dtb, skip, torch.zeros(D, N, dtype=torch.float64))
    y, so = run_scan(cell, x, dt, z, bc, N, None, None)
    for got, w in ((y[0].cpu().double(), want), (so[0].cpu().double(), h)):
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(got[torch.isinf(w)], w[torch.isinf(w)])
    assert bool(torch.isinf(want[at:, c]).all())
