"""The recurrent layer's operators on the GPU against plain 64-bit implementations (layer_ref), within
the bounds derived there: fp32 arithmetic, plus half a step of the output's type."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref
from paper_1804_00344_amd import mtstep as mt

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def dev(t):
    return None if t is None else t.to(DEV)


def check(got, want, bound, what):
    """|got - want| within the bound and half a step of got's type (of the largest value it may round)."""
    g = got.detach().cpu().double()
    tol = bound + ref.HALF_STEP[got.dtype] * (want.abs() + bound) + 1e-37
    bad = ~((g - want).abs() <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float((g - want).abs().max()), float(tol.max()))


def wide(t, left, right, fill=float("nan")):
    """t as columns of a wider matrix whose other columns hold fill."""
    big = torch.full(t.shape[:-1] + (left + t.shape[-1] + right,), fill, dtype=t.dtype)
    big[..., left:left + t.shape[-1]] = t
    return big.to(DEV)[..., left:left + t.shape[-1]]


# ---- convolution --------------------------------------------------------------------------------

def conv_cell(D, W, dtype, silu=True, seed=0):
    g = gen(seed + 77)
    w, b = torch.randn(D, W, generator=g), torch.randn(D, generator=g)
    cfg = mt.make_ssm_config(D, 1, conv=W, conv_silu=silu, dtype=dtype)
    return mt.mt_ssm_load(cfg, dict(A=np.full((D, 1), -1.0, np.float32), conv_w=w, conv_b=b)), w.double(), b.double()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,D,W,lens,first,left", [
    (1, 1, 1, 1, None, False, 0), (1, 1, 8, 4, None, True, 0), (2, 3, 16, 8, [3, 1], True, 8),
    (3, 16, 24, 4, [16, 0, 9], True, 0), (3, 17, 33, 3, [0, 2, 17], False, 0), (2, 50, 40, 2, [50, 33], True, 3),
    (4, 70, 64, 5, [70, 64, 15, 16], True, 8), (1, 300, 2048, 4, None, False, 2048), (5, 33, 7, 6, [33, 1, 4, 5, 6], True, 1),
    (2, 40, 72, 7, [39, 40], False, 0)])
def test_conv(B, S, D, W, lens, first, left, dtype):
    silu = D != 40
    cell, w, b = conv_cell(D, W, dtype, silu)
    g, io = gen(B * S + D), IO[dtype]
    x = torch.randn(B, S, D, generator=g).to(io)
    st = torch.randn(B, W - 1, D, generator=g).to(io) if first else None
    for i, n in enumerate(lens or []):
        x[i, n:] = float("nan")  # behind a prompt: never read
    y = torch.full((B, S, D), 7.0, dtype=io, device=DEV)
    so = torch.empty(B, W - 1, D, dtype=io, device=DEV)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    mt.mt_ssm_conv(cell, wide(x, left, 5 if left else 0), y, lens=ln, state_in=dev(st), state_out=so)
    assert mt.mt_ssm_device_errors(cell) == 0
    for i in range(B):
        n = lens[i] if lens else S
        f = st[i].double() if first else torch.zeros(W - 1, D, dtype=torch.float64)
        want, state, err = ref.conv(x[i, :n].double(), w, b, silu, f)
        check(y[i, :n], want, err, "y")
        assert torch.equal(so[i].cpu().double(), state) and bool((y[i, n:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,n,D,W,left", [(1, 1, 1, 2, 0), (5, 3, 24, 4, 8), (12, 12, 33, 3, 1), (7, 20, 64, 8, 0),
                                          (3, 3, 16, 1, 0), (96, 64, 2048, 4, 0)])
def test_conv_step(M, n, D, W, left, dtype):
    cell, w, b = conv_cell(D, W, dtype)
    g, io = gen(M + D), IO[dtype]
    x, st = torch.randn(M, D, generator=g).to(io), torch.randn(n, W - 1, D, generator=g).to(io)
    row = torch.randint(0, n, (M,), generator=g, dtype=torch.int32)  # rows repeat
    y, so = torch.empty(M, D, dtype=io, device=DEV), torch.empty(M, W - 1, D, dtype=io, device=DEV)
    mt.mt_ssm_conv_step(cell, wide(x, left, 0), y, dev(st), so, src_row=dev(row))
    for m in range(M):
        want, state, err = ref.conv(x[m:m + 1].double(), w, b, True, st[row[m]].double())
        check(y[m:m + 1], want, err, "y")
        assert torch.equal(so[m].cpu().double(), state)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 3, 4])
def test_conv_at_any_alignment(dtype, shift):
    """Rows that start at any element, read and written, are the aligned ones to the bit."""
    B, S, D, W = 2, 700, 64, 4
    cell, _, _ = conv_cell(D, W, dtype)
    x = torch.randn(B, S, D, generator=gen(6)).to(IO[dtype])
    st = torch.randn(B, W - 1, D, generator=gen(7)).to(IO[dtype]).to(DEV)
    y = torch.empty(B, S, D, dtype=x.dtype, device=DEV)
    mt.mt_ssm_conv(cell, dev(x), y, state_in=st)
    big = torch.full((B, S, D + shift + 2), 7.0, dtype=x.dtype, device=DEV)
    mt.mt_ssm_conv(cell, wide(x, shift, 1), big[..., shift:shift + D], state_in=st)
    assert torch.equal(big[..., shift:shift + D], y) and bool((big[..., :shift] == 7).all()) and bool((big[..., shift + D:] == 7).all())
    so, so2 = torch.empty_like(st), torch.empty_like(st)
    tok, bt = torch.empty(B, D, dtype=x.dtype, device=DEV), torch.full((B, D + shift + 2), 7.0, dtype=x.dtype, device=DEV)
    mt.mt_ssm_conv_step(cell, dev(x[:, 0].contiguous()), tok, st, so)
    mt.mt_ssm_conv_step(cell, wide(x[:, 0], shift, 1), bt[:, shift:shift + D], st, so2)
    assert torch.equal(bt[:, shift:shift + D], tok) and torch.equal(so, so2)
    assert bool((bt[:, :shift] == 7).all()) and bool((bt[:, shift + D:] == 7).all())


def test_conv_pieces_and_tokens_are_the_whole():
    """A prompt in pieces, then token by token in place, gives what the whole prompt gives, to the bit."""
    B, S, D, W = 3, 41, 48, 4
    cell, _, _ = conv_cell(D, W, "bf16")
    x = torch.randn(B, S, D, generator=gen(3)).bfloat16().to(DEV)
    whole, st = torch.empty_like(x), torch.empty(B, W - 1, D, dtype=x.dtype, device=DEV)
    mt.mt_ssm_conv(cell, x, whole, state_out=st)
    y, prev, cut = torch.empty_like(x), None, 0
    for to in (2, 19, 36):
        part, nxt = torch.empty(B, to - cut, D, dtype=x.dtype, device=DEV), torch.empty_like(st)
        mt.mt_ssm_conv(cell, x[:, cut:to].contiguous(), part, state_in=prev, state_out=nxt)
        y[:, cut:to], prev, cut = part, nxt, to
    for t in range(cut, S):
        tok = torch.empty(B, D, dtype=x.dtype, device=DEV)
        mt.mt_ssm_conv_step(cell, x[:, t].contiguous(), tok, prev, prev)
        y[:, t] = tok
    assert torch.equal(y, whole) and torch.equal(prev, st)


@pytest.mark.parametrize("dtype,B,S,D,W,lens", [("bf16", 2, 2100, 2048, 4, [2100, 1999]), ("f32", 3, 1400, 1028, 3, None),
                                                ("bf16", 3, 4099, 1504, 8, [4099, 0, 4098]), ("f32", 2, 4100, 1200, 2, None)])
def test_conv_of_many_positions(dtype, B, S, D, W, lens):
    """Runs of eight positions; results above and below the size from which they are stored past the L2s."""
    cell, w, b = conv_cell(D, W, dtype)
    x = torch.randn(B, S, D, generator=torch.Generator(device=DEV).manual_seed(S), device=DEV).to(IO[dtype])
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    y = torch.full((B, S, D), 7.0, dtype=x.dtype, device=DEV)
    so = torch.empty(B, W - 1, D, dtype=x.dtype, device=DEV)
    mt.mt_ssm_conv(cell, x, y, lens=ln, state_out=so)
    for i in range(B):
        n = lens[i] if lens else S
        want, state, err = ref.conv(x[i, :n].double(), w.to(DEV), b.to(DEV), True,
                                    torch.zeros(W - 1, D, dtype=torch.float64, device=DEV))
        check(y[i, :n], want.cpu(), err.cpu(), "y")
        assert torch.equal(so[i].double(), state) and bool((y[i, n:] == 7.0).all())


# ---- scan ---------------------------------------------------------------------------------------

def scan_cell(D, N, G, dtype, seed=0, bias=True):
    g = gen(seed + 5)
    A = -torch.exp(torch.randn(D, N, generator=g))
    dtb = torch.randn(D, generator=g) - 3 if bias else None
    skip = torch.randn(D, generator=g) if bias else None
    cell = mt.mt_ssm_load(mt.make_ssm_config(D, N, groups=G, dtype=dtype), dict(A=A, dt_bias=dtb, skip=skip))
    zero = torch.zeros(D, dtype=torch.float64)
    return cell, A.double(), zero if dtb is None else dtb.double(), zero if skip is None else skip.double()


def scan_inputs(lead, D, N, G, dtype, seed, gate=True):
    g, io = gen(seed), IO[dtype]
    x, dt, z = (torch.randn(*lead, D, generator=g).to(io) for _ in range(3))
    bc = torch.randn(*lead, 2 * G * N, generator=g).to(io)
    return x, dt, (z if gate else None), bc


def per_channel(bc, D, N, G, second):
    m = bc.double()[..., G * N:] if second else bc.double()[..., :G * N]
    return m.reshape(*m.shape[:-1], G, N).repeat_interleave(D // G, -2)


SCANS = [
    # B, S, D, N, G, lens, first, gate, left
    (1, 1, 1, 1, 1, None, False, False, 0), (1, 1, 8, 16, 1, None, True, True, 0),
    (3, 5, 16, 4, 2, [5, 0, 3], True, True, 1), (2, 17, 40, 8, 5, [17, 16], False, True, 0),
    (4, 33, 70, 16, 1, [33, 0, 16, 1], True, True, 3), (2, 40, 24, 5, 24, None, True, False, 0),
    (2, 29, 33, 24, 3, [29, 7], True, True, 0), (1, 21, 20, 33, 2, None, False, True, 8),
    (2, 19, 12, 100, 4, [18, 19], True, True, 0), (1, 18, 10, 128, 1, None, True, True, 0),
    (1, 9, 6, 256, 3, None, True, True, 0), (2, 3, 300, 17, 300, None, False, True, 0),
    # long axes of few rows: cut into pieces, some of them behind a prompt's end
    (1, 700, 16, 16, 1, None, True, True, 0), (3, 530, 20, 8, 1, [530, 64, 300], True, True, 0),
    (2, 400, 9, 40, 3, [65, 400], False, True, 0),
    # one group over workgroups of four waves, the last one not full, whole and cut into pieces
    (2, 30, 300, 4, 1, [30, 11], True, True, 0), (1, 21, 150, 7, 1, None, False, False, 1),
    (1, 600, 70, 16, 1, None, True, True, 0), (2, 410, 40, 32, 1, [410, 209], False, True, 0),
    (1, 300, 37, 64, 1, None, True, False, 0), (1, 260, 34, 128, 1, None, True, True, 0),
    (1, 170, 40, 250, 1, None, True, True, 0),
    # several groups of many states, cut
    (1, 330, 24, 100, 4, None, True, True, 0), (1, 150, 34, 256, 17, None, False, True, 0)]


def run_scan(cell, x, dt, z, bc, GN, lens, st, left=0, y_fill=7.0, stream=None):
    B, S, D = x.shape
    y = torch.full((B, S, D), y_fill, dtype=x.dtype, device=DEV)
    so = torch.empty(B, cell.D, cell.N, device=DEV)
    ws = torch.full((mt.mt_ssm_workspace_bytes(cell, B, S),), 255, dtype=torch.uint8, device=DEV)
    r = 2 if left else 0
    w = wide(bc, left, r)
    mt.mt_ssm_scan(cell, wide(x, left, r), wide(dt, left, 0), w[..., :GN], w[..., GN:], y,
                   z=None if z is None else wide(z, 0, left), lens=lens, state_in=st, state_out=so, ws=ws, stream=stream)
    return y, so


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,D,N,G,lens,first,gate,left", SCANS)
def test_scan(B, S, D, N, G, lens, first, gate, left, dtype):
    cell, A, dtb, skip = scan_cell(D, N, G, dtype, bias=gate)
    x, dt, z, bc = scan_inputs((B, S), D, N, G, dtype, B + S + D + N, gate)
    st = torch.randn(B, D, N, generator=gen(9)) if first else None
    for i, n in enumerate(lens or []):
        for t in (x, dt, z, bc):
            if t is not None:
                t[i, n:] = float("nan")  # behind a prompt: never read
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    y, so = run_scan(cell, x, dt, z, bc, G * N, ln, dev(st), left)
    assert mt.mt_ssm_device_errors(cell) == 0
    for i in range(B):
        n = lens[i] if lens else S
        h0 = st[i].double() if first else torch.zeros(D, N, dtype=torch.float64)
        want, h, ye, he = ref.scan(x[i, :n].double(), dt[i, :n].double(), per_channel(bc[i, :n], D, N, G, False),
                                   per_channel(bc[i, :n], D, N, G, True), None if z is None else z[i, :n].double(), A, dtb,
                                   skip, h0)
        check(y[i, :n], want, ye, "y")
        check(so[i], h, he, "state")
        assert bool((y[i, n:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,n,D,N,G,gate,left", [(1, 1, 1, 1, 1, True, 0), (5, 3, 16, 16, 1, True, 8), (12, 12, 33, 8, 3, False, 1),
                                                 (7, 20, 20, 5, 20, True, 0), (3, 2, 10, 24, 2, True, 0), (4, 4, 9, 100, 3, True, 1),
                                                 (2, 5, 6, 256, 1, True, 0), (3, 3, 70, 33, 7, True, 0), (60, 60, 512, 16, 1, True, 0)])
def test_step(M, n, D, N, G, gate, left, dtype):
    cell, A, dtb, skip = scan_cell(D, N, G, dtype, bias=gate)
    x, dt, z, bc = scan_inputs((M,), D, N, G, dtype, M + D + N, gate)
    st = torch.randn(n, D, N, generator=gen(2))
    row = torch.randint(0, n, (M,), generator=gen(4), dtype=torch.int32)
    y, so = torch.empty(M, D, dtype=x.dtype, device=DEV), torch.empty(M, D, N, device=DEV)
    w = wide(bc, left, 0)
    mt.mt_ssm_step(cell, wide(x, left, 0), dev(dt), w[:, :G * N], w[:, G * N:], y, dev(st), so, z=dev(z), src_row=dev(row))
    for m in range(M):
        s = slice(m, m + 1)
        want, h, ye, he = ref.scan(x[s].double(), dt[s].double(), per_channel(bc[s], D, N, G, False),
                                   per_channel(bc[s], D, N, G, True), None if z is None else z[s].double(), A, dtb, skip,
                                   st[row[m]].double())
        check(y[s], want, ye, "y")
        check(so[m], h, he, "state")


@pytest.mark.parametrize("M,D,N", [(300, 2000, 16), (1100, 120, 64)])
def test_step_of_large_states(M, D, N):
    """States of more than 32 MB, which are stored past the L2s."""
    cell, A, dtb, skip = scan_cell(D, N, 1, "bf16")
    x, dt, z, bc = scan_inputs((M,), D, N, 1, "bf16", M)
    st = torch.randn(M, D, N, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    row = torch.randint(0, M, (M,), generator=gen(4), dtype=torch.int32)
    y, so = torch.empty(M, D, dtype=x.dtype, device=DEV), torch.empty(M, D, N, device=DEV)
    w = dev(bc)
    mt.mt_ssm_step(cell, dev(x), dev(dt), w[:, :N], w[:, N:], y, st, so, z=dev(z), src_row=dev(row))
    for m in (0, 1, M // 2, M - 1):
        s = slice(m, m + 1)
        want, h, ye, he = ref.scan(x[s].double(), dt[s].double(), per_channel(bc[s], D, N, 1, False),
                                   per_channel(bc[s], D, N, 1, True), z[s].double(), A, dtb, skip,
                                   st[row[m].item()].cpu().double())
        check(y[s], want, ye, "y")
        check(so[m], h, he, "state")
    # the same rows in place, by a smaller call: the same bits
    sub = st[row[:4].long().to(DEV)].clone()
    y2 = torch.empty(4, D, dtype=x.dtype, device=DEV)
    mt.mt_ssm_step(cell, dev(x[:4]), dev(dt[:4]), w[:4, :N], w[:4, N:], y2, sub, sub, z=dev(z[:4]))
    assert torch.equal(y2, y[:4]) and torch.equal(sub, so[:4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 3, 4])
def test_step_at_any_alignment(dtype, shift):
    M, D, N, G = 5, 70, 12, 2
    cell, *_ = scan_cell(D, N, G, dtype)
    x, dt, z, bc = scan_inputs((M,), D, N, G, dtype, 3)
    st = torch.randn(M, D, N, generator=gen(2)).to(DEV)
    out = []
    for w in (dev(bc), wide(bc, shift, 1)):
        y, so = torch.empty(M, D, dtype=x.dtype, device=DEV), torch.empty_like(st)
        mt.mt_ssm_step(cell, dev(x), dev(dt), w[:, :G * N], w[:, G * N:], y, st, so, z=dev(z))
        out.append((y, so))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_step_in_place_and_bad_rows():
    D, N = 40, 16
    cell, *_ = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = (dev(t) for t in scan_inputs((6,), D, N, 1, "f32", 1))
    st = torch.randn(6, D, N, generator=gen(2)).to(DEV)
    outs = []
    for row in (None, torch.arange(6, dtype=torch.int32, device=DEV)):
        y, so = torch.empty(6, D, device=DEV), torch.empty_like(st)
        mt.mt_ssm_step(cell, x, dt, bc[:, :N], bc[:, N:], y, st, so, z=z, src_row=row)
        outs.append((y, so))
    y, so = torch.empty(6, D, device=DEV), st.clone()
    mt.mt_ssm_step(cell, x, dt, bc[:, :N], bc[:, N:], y, so, so, z=z)
    for a, b in outs:
        assert torch.equal(a, y) and torch.equal(b, so)
    assert mt.mt_ssm_device_errors(cell) == 0
    # rows out of range are clamped and reported once
    row = torch.tensor([-1, 9, 2, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    a, b = torch.empty(6, D, device=DEV), torch.empty_like(st)
    mt.mt_ssm_step(cell, x, dt, bc[:, :N], bc[:, N:], a, st, b, z=z, src_row=row)
    mt.mt_ssm_step(cell, x, dt, bc[:, :N], bc[:, N:], y, st, so, z=z, src_row=row.clamp(0, 5))
    assert torch.equal(a, y) and torch.equal(b, so)
    assert mt.mt_ssm_device_errors(cell) == 2 and mt.mt_ssm_device_errors(cell) == 0


def test_bad_lengths_are_clamped_and_reported():
    D, N, S = 20, 8, 30
    cell, *_ = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = scan_inputs((3, S), D, N, 1, "f32", 1)
    run = lambda l: run_scan(cell, x, dt, z, bc, N, torch.tensor(l, dtype=torch.int32, device=DEV), None)
    a, b = run([-5, 31, 2 ** 31 - 1]), run([0, 30, 30])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert mt.mt_ssm_device_errors(cell) == 4 and mt.mt_ssm_device_errors(cell) == 0
    ccell, *_ = conv_cell(D, 4, "f32")
    ys = []
    for l in ([-5, 31, 2 ** 31 - 1], [0, 30, 30]):
        y = torch.zeros(3, S, D, device=DEV)
        mt.mt_ssm_conv(ccell, dev(x), y, lens=torch.tensor(l, dtype=torch.int32, device=DEV))
        ys.append(y)
        assert mt.mt_ssm_device_errors(ccell) == (4 if l[0] < 0 else 0)
    assert torch.equal(*ys)


@pytest.mark.parametrize("D,N,G", [(24, 16, 1), (36, 40, 3)])
def test_scan_pieces_and_tokens_are_the_whole(D, N, G):
    B, S = 2, 37
    cell, A, dtb, skip = scan_cell(D, N, G, "f32")
    x, dt, z, bc = scan_inputs((B, S), D, N, G, "f32", 8)
    whole, st = run_scan(cell, x, dt, z, bc, G * N, None, None)
    y, prev, cut = torch.empty_like(whole), None, 0
    for to in (1, 20):
        part, prev = run_scan(cell, *(t[:, cut:to].contiguous() for t in (x, dt, z, bc)), G * N, None, prev)
        y[:, cut:to], cut = part, to
    for t in range(cut, S):
        tok = torch.empty(B, D, device=DEV)
        w = dev(bc[:, t])
        mt.mt_ssm_step(cell, dev(x[:, t].contiguous()), dev(dt[:, t].contiguous()), w[:, :G * N], w[:, G * N:], tok, prev, prev,
                       z=dev(z[:, t].contiguous()))
        y[:, t] = tok
    # each form within its bound of the 64-bit values
    for i in range(B):
        _, h, ye, he = ref.scan(x[i].double(), dt[i].double(), per_channel(bc[i], D, N, G, False),
                                per_channel(bc[i], D, N, G, True), z[i].double(), A, dtb, skip,
                                torch.zeros(D, N, dtype=torch.float64))
        assert bool(((y[i] - whole[i]).abs().cpu() <= 2 * ye + 1e-37).all())
        assert bool(((prev[i] - st[i]).abs().cpu() <= 2 * he + 1e-37).all())


@pytest.mark.parametrize("value", [float("inf"), float("nan"), 3e38])
def test_large_and_infinite_steps(value):
    """dt of any size: an infinite step forgets the state (and NaN stays in its channel)."""
    D, N, S = 8, 16, 6
    cell, *_ = scan_cell(D, N, 1, "f32")
    x, dt, z, bc = scan_inputs((1, S), D, N, 1, "f32", 3)
    clean, _ = run_scan(cell, x, dt, z, bc, N, None, None)
    dt2 = dt.clone()
    dt2[0, 2, 3] = -value  # a step of zero: the state is kept
    y, _ = run_scan(cell, x, dt2, z, bc, N, None, None)
    dt3 = dt.clone()
    dt3[0, 2, 3] = float("-inf")
    keep, _ = run_scan(cell, x, dt3, z, bc, N, None, None)
    if value == value:
        assert torch.equal(y, keep) and bool(torch.isfinite(y).all())
    others = [c for c in range(D) if c != 3]
    assert torch.equal(y[..., others], clean[..., others]) and torch.equal(y[0, :2], clean[0, :2])
    if value != value:
        assert bool(torch.isnan(y[0, 2:, 3]).all())


def test_rates_up_to_the_largest_float():
    """A times log2(e) would leave fp32: the states forget in one step, and steps of zero keep them."""
    D, N, S = 6, 5, 3
    cell = mt.mt_ssm_load(mt.make_ssm_config(D, N), dict(A=torch.full((D, N), -torch.finfo(torch.float32).max)))
    x, dt, _, bc = scan_inputs((1, S), D, N, 1, "f32", 1, False)
    dt[0, 2, 0] = float("-inf")
    y, so = run_scan(cell, x, dt, None, bc, N, None, dev(torch.randn(1, D, N, generator=gen(2))))
    d = torch.log1p(torch.exp(dt.double()))
    for c in range(D):
        t = 1 if c == 0 else 2
        want = d[0, t, c] * x[0, t, c].double() * bc[0, t, :N].double()
        # softplus within 14 roundings, two products
        check(so[0, c], want, 16 * ref.U * want.abs(), "state")
    assert bool(torch.isfinite(y).all())


# ---- products in 8 bits -------------------------------------------------------------------------

def product(x, W, bias, ydt, left=0, pad=0):
    mat = mt.mt_i8_load(W, bias)
    M, N = x.shape[0], W.shape[1]
    big = torch.full((M, left + N + pad), 7.0, dtype=ydt, device=DEV)
    y = big[:, left:left + N]
    ws = torch.full((mt.mt_i8_workspace_bytes(mat, M),), 255, dtype=torch.uint8, device=DEV)
    mt.mt_i8_product(mat, wide(x, left, pad), y, ws)
    assert bool((big[:, :left] == 7.0).all()) and bool((big[:, left + N:] == 7.0).all())
    return y


PRODUCTS = [
    (1, 1, 1, True, 0), (1, 16, 32, False, 0), (2, 17, 33, True, 1), (5, 64, 257, True, 0), (16, 128, 64, False, 8),
    (31, 100, 96, True, 0), (32, 512, 40, True, 0), (33, 333, 300, False, 5), (63, 65, 129, True, 0), (64, 256, 1000, True, 0),
    (65, 130, 255, True, 0), (127, 200, 128, True, 0), (129, 1024, 513, True, 8), (257, 96, 600, False, 0),
    (300, 2000, 77, True, 0), (1, 4096, 200, True, 0), (3, 5000, 31, False, 0), (20, 65536, 48, False, 0),
    (4, 600, 70, True, 0), (3, 1500, 33, False, 1), (4, 3000, 2500, True, 0)]


@pytest.mark.parametrize("xdt,ydt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,K,N,bias,left", PRODUCTS)
def test_product(M, K, N, bias, left, xdt, ydt):
    g = gen(M + K + N)
    x = (torch.randn(M, K, generator=g) * torch.exp(2 * torch.randn(M, 1, generator=g))).to(IO[xdt])
    W = torch.randn(K, N, generator=g) * torch.exp(torch.randn(1, N, generator=g))
    b = torch.randn(N, generator=g) if bias else None
    y = product(x, W.numpy(), b, IO[ydt], left, 3 if left else 0)
    want, err = ref.product(x.float().numpy(), W.numpy(), None if b is None else b.numpy())
    check(y, torch.from_numpy(want), torch.from_numpy(err), "y")


# (M, K, N): the larger tiles, with part of the last one in rows and columns; results above and below the
# size from which they are stored past the L2s
LARGE_PRODUCTS = [(1100, 200, 2001), (70, 500, 50001), (4000, 2000, 500), (770, 513, 20002), (3000, 300, 4100), (2000, 6000, 8000)]


@pytest.mark.parametrize("ydt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", LARGE_PRODUCTS)
def test_large_products(M, K, N, ydt):
    g = torch.Generator(device=DEV).manual_seed(M)
    x, W = torch.randn(M, K, generator=g, device=DEV), torch.randn(K, N, generator=g, device=DEV)
    b = torch.randn(N, generator=g, device=DEV)
    mat = mt.mt_i8_load(W, b)
    ws = torch.full((mt.mt_i8_workspace_bytes(mat, M),), 255, dtype=torch.uint8, device=DEV)
    outs = []
    for ld in (N, (N + 15) // 8 * 8):  # rows of odd length; rows aligned for vectors
        y = torch.full((M + 1, ld), 7.0, dtype=IO[ydt], device=DEV)
        mt.mt_i8_product(mat, x, y[:M, :N], ws)
        assert bool((y[M] == 7.0).all()) and bool((y[:, N:] == 7.0).all())  # nothing beside the result
        outs.append(y[:M, :N])
    assert torch.equal(*outs)
    qx, sx = (torch.from_numpy(t) for t in ref.quantise(x.cpu().numpy(), 1))
    qw, sw = (torch.from_numpy(t) for t in ref.quantise(W.cpu().numpy(), 0))
    p = (qx.double().to(DEV) @ qw.double().to(DEV)) * sw.double().to(DEV) * sx.double().to(DEV)  # sums exact in 64 bits
    want = p + b.double()
    check(outs[0], want.cpu(), (4 * ref.U * (p.abs() + want.abs())).cpu(), "y")


def test_product_edges():
    """Ties, rows of zeros, of the smallest magnitudes, the largest sums; NaN and infinities stay in their row."""
    K, N = 300, 70
    g = gen(1)
    x = torch.randn(12, K, generator=g)
    x[0] = 0
    x[1] = 1e-38
    x[2] = x[2] * 2.0 ** -99
    x[3] = 127.0                      # the largest sum: all of one size
    x[4] = torch.arange(K) % 128 - 63.5  # halves: ties to even
    x[4, 0] = 127.0
    x[5] = x[5] * 1e30
    x[6, 17] = float("inf")
    x[7, 299] = float("nan")
    x[8, 0] = float("-inf")
    x[9, 1:] = 0
    W = torch.randn(K, N, generator=g)
    W[:, 0] = 0
    W[:, 1] = -127.0
    W[:, 2] = 1e-35
    want, err = ref.product(x.nan_to_num(0, 0, 0).numpy(), W.numpy(), None)
    bad = [6, 7, 8]
    good = [i for i in range(12) if i not in bad]
    for ws in (W, W.to(DEV)):
        y = product(x, ws, None, torch.float32)
        check(y[good], torch.from_numpy(want)[good], torch.from_numpy(err)[good], "y")
        assert bool(torch.isnan(y[bad]).all())
    assert float(y[3, 1]) == pytest.approx(-127.0 * 127 * K, rel=1e-6)


def test_load_refuses_values_that_have_no_scale():
    for bad in (float("nan"), float("inf")):
        W = torch.randn(40, 30)
        W[39, 29] = bad
        with pytest.raises(mt.MtError) as e:
            mt.mt_i8_load(W)
        assert e.value.status == mt.MT_ERR_ARG


@pytest.mark.parametrize("M,K,N", [(1, 40, 100), (3, 512, 70), (37, 300, 130), (129, 64, 257), (200, 512, 50000)])
@pytest.mark.parametrize("ydt", [torch.float32, torch.bfloat16])
def test_rows_behind_the_last_are_left(M, K, N, ydt):
    mat = mt.mt_i8_load(torch.randn(K, N, generator=gen(3)))
    x = torch.full((M + 64, K), float("nan"), device=DEV)
    x[:M] = torch.randn(M, K, generator=gen(4)).to(DEV)
    y = torch.full((M + 300, N), 7.0, dtype=ydt, device=DEV)
    ws = torch.empty(mt.mt_i8_workspace_bytes(mat, M), dtype=torch.uint8, device=DEV)
    mt.mt_i8_product(mat, x[:M], y[:M], ws)
    assert bool((y[M:] == 7.0).all()) and bool(torch.isfinite(y[:M]).all()) and not bool((y[:M] == 7.0).all(1).any())


def test_rows_do_not_depend_on_their_neighbours():
    """A row's result is the same alone and within any number of rows (whichever kernel form each takes)."""
    K, N = 520, 700
    x = torch.randn(300, K, generator=gen(5)).to(DEV)
    mat = mt.mt_i8_load(torch.randn(K, N, generator=gen(6)), torch.randn(N, generator=gen(7)))
    ws = torch.empty(mt.mt_i8_workspace_bytes(mat, 300), dtype=torch.uint8, device=DEV)
    ys = {}
    for M in (300, 129, 64, 33, 32, 9, 1):
        y = torch.empty(M, N, device=DEV)
        mt.mt_i8_product(mat, x[:M], y, ws)
        ys[M] = y
    for M, y in ys.items():
        assert torch.equal(y, ys[300][:M]), M


# ---- streams, graphs, devices -------------------------------------------------------------------

def test_calls_run_on_the_given_stream_and_replay():
    """All calls captured into one graph and replayed on new inputs, with eager work between the replays."""
    B, S, D, N, W, E = 2, 130, 48, 16, 4, 40
    g = gen(11)
    cell = mt.mt_ssm_load(mt.make_ssm_config(D, N, conv=W, dtype="f32"),
                          dict(A=-torch.exp(torch.randn(D, N, generator=g)), conv_w=torch.randn(D, W, generator=g)))
    mats = [mt.mt_i8_load(torch.randn(D, D + 2 * N, generator=g)), mt.mt_i8_load(torch.randn(D, E, generator=g))]
    f = lambda *s: torch.zeros(*s, device=DEV)
    u, x, dbc, y, out, cs, hs = f(B, S, D), f(B, S, D), f(B, S, D + 2 * N), f(B, S, D), f(B, S, E), f(B, W - 1, D), f(B, D, N)
    ws = torch.empty(max([mt.mt_ssm_workspace_bytes(cell, B, S)] + [mt.mt_i8_workspace_bytes(m, B * S) for m in mats]),
                     dtype=torch.uint8, device=DEV)

    def calls(stream):
        mt.mt_ssm_conv(cell, u, x, state_out=cs, stream=stream)
        mt.mt_i8_product(mats[0], x, dbc, ws, stream=stream)
        mt.mt_ssm_scan(cell, x, dbc[..., :D], dbc[..., D:D + N], dbc[..., D + N:], y, state_out=hs, ws=ws, stream=stream)
        mt.mt_i8_product(mats[1], y, out, ws, stream=stream)

    side = torch.cuda.Stream()
    u.copy_(torch.randn(B, S, D, generator=g))
    torch.cuda.synchronize()
    calls(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(None)
    for i in range(3):
        v = torch.randn(B, S, D, generator=g).to(DEV)
        u.copy_(v)
        out.zero_(), hs.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, hs, cs, y)]
        for t in (x, dbc, y, out, cs, hs):
            t.zero_()
        calls(None)
        torch.cuda.synchronize()
        for a, b in zip(got, (out, hs, cs, y)):
            assert torch.equal(a, b), i


def test_many_short_prompts_and_tokens():
    """More sentences than a grid dimension holds at once: every one is worked on, and none twice."""
    B, S, D, N, W = 40000, 2, 12, 4, 3
    g = gen(21)
    w = dict(A=-torch.exp(torch.randn(D, N, generator=g)), conv_w=torch.randn(D, W, generator=g))
    cell = mt.mt_ssm_load(mt.make_ssm_config(D, N, conv=W, dtype="f32"), w)
    x, dt = torch.randn(B, S, D, generator=g), torch.randn(B, S, D, generator=g)
    bc = torch.randn(B, S, 2 * N, generator=g)
    lens = torch.randint(0, S + 1, (B,), generator=g, dtype=torch.int32)
    st, cs = torch.randn(B, D, N, generator=g), torch.randn(B, W - 1, D, generator=g)

    def calls(i, j):  # sentences i .. j - 1
        n = j - i
        y, so = torch.zeros(n, S, D, device=DEV), torch.empty(n, D, N, device=DEV)
        yc, co = torch.zeros(n, S, D, device=DEV), torch.empty(n, W - 1, D, device=DEV)
        ys, ss = torch.empty(n, D, device=DEV), torch.empty(n, D, N, device=DEV)
        ysc, sc = torch.empty(n, D, device=DEV), torch.empty(n, W - 1, D, device=DEV)
        ws = torch.empty(mt.mt_ssm_workspace_bytes(cell, n, S), dtype=torch.uint8, device=DEV)
        xd, dd, bd, l, s0, c0 = (dev(t[i:j].contiguous()) for t in (x, dt, bc, lens, st, cs))
        mt.mt_ssm_scan(cell, xd, dd, bd[..., :N], bd[..., N:], y, lens=l, state_in=s0, state_out=so, ws=ws)
        mt.mt_ssm_conv(cell, xd, yc, lens=l, state_in=c0, state_out=co)
        mt.mt_ssm_step(cell, xd[:, 0], dd[:, 0], bd[:, 0, :N], bd[:, 0, N:], ys, s0, ss)
        mt.mt_ssm_conv_step(cell, xd[:, 0], ysc, c0, sc)
        return y, so, yc, co, ys, ss, ysc, sc

    parts = [calls(i, min(B, i + 9000)) for i in range(0, B, 9000)]
    for whole, *pieces in zip(calls(0, B), *parts):
        assert torch.equal(whole, torch.cat(pieces))
    assert mt.mt_ssm_device_errors(cell) == 0


def test_one_handle_on_two_streams():
    B, S, D, N = 3, 700, 64, 16
    cell, *_ = scan_cell(D, N, 1, "f32")
    mat = mt.mt_i8_load(torch.randn(D, 300, generator=gen(1)))
    runs = []
    for seed in (1, 2):
        x, dt, z, bc = (dev(t) for t in scan_inputs((B, S), D, N, 1, "f32", seed))
        runs.append(dict(x=x, dt=dt, z=z, bc=bc, y=torch.zeros_like(x), so=torch.empty(B, D, N, device=DEV),
                         out=torch.empty(B, S, 300, device=DEV), st=torch.cuda.Stream(),
                         ws=torch.empty(max(mt.mt_ssm_workspace_bytes(cell, B, S), mt.mt_i8_workspace_bytes(mat, B * S)),
                                        dtype=torch.uint8, device=DEV)))

    def go(r, stream):
        mt.mt_ssm_scan(cell, r["x"], r["dt"], r["bc"][..., :N], r["bc"][..., N:], r["y"], z=r["z"], state_out=r["so"], ws=r["ws"],
                       stream=stream)
        mt.mt_i8_product(mat, r["y"], r["out"], r["ws"], stream=stream)

    want = []
    for r in runs:
        go(r, None)
        want.append([r[k].clone() for k in ("y", "so", "out")])
    torch.cuda.synchronize()
    for _ in range(5):
        for r in runs:
            go(r, r["st"])
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        for k, v in zip(("y", "so", "out"), w):
            assert torch.equal(r[k], v)
