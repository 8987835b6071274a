"""The attention layer's operators at the edges of their contracts, on every kernel that a call may take: scores of any finite
size, windows of any size."""
from decimal import Decimal, getcontext

import pytest

torch = pytest.importorskip("torch")

from paper_1804_00344_amd import mtstep as mt
from test_gpu_attn import HALF, fill_cache, layer, pages_for, run_cross, run_paged
from test_gpu_layer import DEV, IO, check, dev, gen

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

U = 2.0 ** -24

# B, S, Hq, Hk, Dh, longest row (paged) or keys (cross): vector units, tiles of 32 and of 128 rows, each whole and in parts
SIZES = [(1, 1, 2, 2, 64, 90), (2, 1, 2, 2, 256, 5000), (1, 4, 2, 2, 128, 900), (2, 20, 2, 1, 64, 90), (1, 20, 2, 2, 128, 3000),
         (1, 40, 2, 2, 192, 90), (8, 300, 16, 16, 64, 310), (8, 260, 16, 16, 128, 300), (1, 300, 8, 8, 64, 4700)]


def one_feature(B, S, Hq, Hk, Dh, L, size, sign, g):
    """q, k, v of which only feature 5 of a head counts: a score is one product of two values of 8 bits, exact in fp32.  Two
    different scores of size 2^26 or more differ by far more than a weight's range, equal ones have equal weights."""
    q = torch.zeros(B, S, Hq, Dh)
    q[..., 5] = torch.ldexp(1 + torch.randint(0, 128, (B, S, Hq), generator=g) / 128.0, torch.tensor(size))
    k, v = torch.randn(B, L, Hk, Dh, generator=g), torch.randn(B, L, Hk, Dh, generator=g)
    k[..., 5] = 1 + torch.randint(0, 128, (B, L, Hk), generator=g) / 128.0
    if sign == "minus":
        k[..., 5] *= -1
    elif sign == "both":
        k[..., 5] *= torch.randint(0, 2, (B, L, Hk), generator=g) * 2.0 - 1
    return q, k, v


def largest(q, k, v, seen, G, half_step):
    """The mean of the values whose keys score highest, q [n, Hq, Dh], k, v [L, Hk, Dh], seen [n, L]; bound: equal weights,
    each rounded once, over as many values."""
    n, Hq, Dh = q.shape
    want, err = torch.zeros(n, Hq, Dh, dtype=torch.float64), torch.zeros(n, Hq, Dh, dtype=torch.float64)
    for h in range(Hq):
        s = q[:, h, 5:6].double() * k[None, :, h // G, 5].double()
        s = torch.where(seen, s, torch.full_like(s, float("-inf")))
        first = ((s == s.amax(1, keepdim=True)) & seen).double()
        count = first.sum(1, keepdim=True).clamp(min=1)
        want[:, h] = first @ v[:, h // G] / count
        err[:, h] = first @ v[:, h // G].abs() / count * (half_step + (count + 16) * U)
    return want.reshape(n, -1), err.reshape(n, -1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sign", ["plus", "minus", "both"])
@pytest.mark.parametrize("size", [26, 37, 100])
@pytest.mark.parametrize("case", SIZES, ids=lambda c: "-".join(str(v) for v in c))
def test_scores_of_any_finite_size(case, size, sign, dtype):
    """Scores from 1e7 to 1e30: the weight of the largest is one, whatever the product with the scale is rounded by."""
    B, S, Hq, Hk, Dh, L = case
    g = gen(size + S)
    q, k, v = one_feature(B, S, Hq, Hk, Dh, L, size, sign, g)
    q, k, v = (t.to(IO[dtype]) for t in (q, k, v))
    a = layer(Hq, Hk, Dh, dtype, page=16)
    lens = [L - 7 * b for b in range(B)]
    table, n_pages = pages_for(lens, 16, -(-L // 16), g)
    _, _, kc, vc = fill_cache(table, lens, 16, Hk, Dh, n_pages, dtype, g)
    for t, c in ((k, kc), (v, vc)):
        for b in range(B):
            for j in range(0, lens[b], 16):
                part = t[b, j:min(j + 16, lens[b])]
                c[table[b, j // 16], :, :part.shape[0]] = part.transpose(0, 1)
    new = [min(S, n) for n in lens]
    y = run_paged(a, dev(q.flatten(2)), lens, table, kc, vc, new)
    mask = (torch.rand(B, L, generator=g) < 0.7).float()
    x = run_cross(a, dev(q.flatten(2)), dev(k.flatten(2)), dev(v.flatten(2)), mask)
    for b in range(B):
        n = lens[b]
        p, j = torch.arange(n - new[b], n)[:, None], torch.arange(n)[None]
        want, err = largest(q[b, :new[b]], k[b, :n], v[b, :n].double(), j <= p, Hq // Hk, HALF[dtype])
        check(y[b, :new[b]], want, err, (b, "paged"))
        want, err = largest(q[b], k[b], v[b].double(), (mask[b] != 0)[None].expand(S, -1), Hq // Hk, HALF[dtype])
        check(x[b], want, err, (b, "cross"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sign", ["plus", "minus", "both"])
@pytest.mark.parametrize("size", [24, 27, 28, 29, 32])
@pytest.mark.parametrize("case", [SIZES[i] for i in (2, 3, 6, 7)] + [(2, 102, 48, 16, 128, 107)], ids=lambda c: "-".join(str(v) for v in c))
def test_scores_of_neighbouring_rows_on_both_sides_of_a_size(case, size, sign, dtype):
    """Equal scores of a row have equal weights, wherever those of the rows beside it lie."""
    test_scores_of_any_finite_size(case, size, sign, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S,Hq,Hk,Dh,B", [(4, 2, 2, 64, 3), (4, 2, 2, 256, 3), (20, 4, 2, 64, 3), (300, 16, 16, 64, 8)])
def test_a_window_past_every_position(S, Hq, Hk, Dh, B, dtype):
    """The largest window is none, also where rows have fewer positions than new ones."""
    g = gen(S + Dh)
    lens = [[1, S // 2 + 1, S + 9][b % 3] for b in range(B)]
    table, n_pages = pages_for(lens, 16, -(-max(lens) // 16) + 1, g)
    _, _, kc, vc = fill_cache(table, lens, 16, Hk, Dh, n_pages, dtype, g)
    q = dev(torch.randn(B, S, Hq * Dh, generator=g).to(IO[dtype]))
    want = run_paged(layer(Hq, Hk, Dh, dtype), q, lens, table, kc, vc)
    assert bool(torch.isfinite(want).all()) and bool((want[0, -1] != 0).any())
    for window in (2 ** 31 - 1, 2 ** 31 - S, 2 ** 30 + 1, 2 ** 30, 2 ** 30 - 1):
        y = run_paged(layer(Hq, Hk, Dh, dtype, window=window), q, lens, table, kc, vc)
        assert torch.equal(y, want), window


def test_append_of_more_than_2_to_the_30_heads():
    """Neither norm nor rotation: queries, keys and values are copied, whatever B*S*Hq is."""
    Hq, page, S = 512, 256, 2 ** 21 + 5
    a = layer(Hq, 1, 8, "bf16", page=page)
    nb = -(-S // page)
    q = torch.empty(1, S, Hq * 8, dtype=torch.bfloat16, device=DEV)
    for part in q.flatten().split(2 ** 28):
        part.normal_()
    k, v = (torch.randn(1, S, 8, device=DEV).bfloat16() for _ in range(2))
    kc, vc = (torch.zeros(nb, 1, page, 8, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    out = torch.empty_like(q)
    table = torch.arange(nb, dtype=torch.int32, device=DEV)[None]
    mt.mt_attn_append(a, q, k, v, out, torch.tensor([S], dtype=torch.int32, device=DEV), table, kc, vc)
    assert mt.mt_attn_device_errors(a) == 0
    assert all(torch.equal(x, y) for x, y in zip(out.flatten().split(2 ** 30), q.flatten().split(2 ** 30)))
    for t, c in ((k, kc), (v, vc)):
        assert torch.equal(c.reshape(-1, 8)[:S], t[0]) and bool((c.reshape(-1, 8)[S:] == 0).all())


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("base", [500.0, 10000.0, 1e30])
def test_angles_at_any_position(base, given):
    """Against angles of 50 digits: a frequency in turns and its product with the position are rounded to 64 bits, 2^-53 of it
    each; what is left of the last turn to 32 bits, 1.6 u (which the bound of a rotation has)."""
    getcontext().prec = 60
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    base = float(torch.tensor(base, dtype=torch.float32))
    Dh, page, positions = 64, 256, [5, 1000003, 2 ** 24 + 1, 2 ** 30 - 5]
    exact = [Decimal(base) ** (Decimal(-2 * i) / Dh) for i in range(Dh // 2)]
    given_freq = torch.tensor([float(f) for f in exact]).float() * 3 if given else None
    if given:
        exact = [Decimal(float(f)) for f in given_freq]
    a = layer(1, 1, Dh, "f32", dict(freq=given_freq) if given else None, page=page, rot=Dh, rot_base=base)
    g = gen(5)
    q, k, v = (torch.randn(4, 1, Dh, generator=g) for _ in range(3))
    table = torch.arange(4, dtype=torch.int32, device=DEV)[:, None].repeat(1, 2 ** 30 // page)
    kc, vc = (torch.zeros(4, 1, page, Dh, device=DEV) for _ in range(2))
    out = torch.empty(4, 1, Dh, device=DEV)
    lens = torch.tensor([p + 1 for p in positions], dtype=torch.int32, device=DEV)
    mt.mt_attn_append(a, dev(q), dev(k), dev(v), out, lens, table, kc, vc)
    assert mt.mt_attn_device_errors(a) == 0
    far = torch.tensor([[float(p * f) for f in exact] for p in positions], dtype=torch.float64).repeat(1, 2)
    rest = torch.tensor([[float(p * f % turn) for f in exact] for p in positions], dtype=torch.float64)  # of the last turn
    c, s = torch.cos(rest), torch.sin(rest)
    for got, x in ((out[:, 0], q), (torch.stack([kc[b, 0, p % page] for b, p in enumerate(positions)]), k)):
        lo, hi = x[:, 0].double().split(Dh // 2, 1)
        mag = (lo.abs() + hi.abs()).repeat(1, 2)
        check(got, torch.cat([lo * c - hi * s, hi * c + lo * s], 1), mag * (8 * U + far * 2.0 ** -51), "rotated")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S,Hq,Dh", [(1, 2, 64), (1, 2, 256), (4, 2, 128), (20, 2, 64)])
def test_scores_that_are_minus_infinity_in_powers_of_two(S, Hq, Dh, dtype):
    """Finite scores below -2^128 / log2(e), as many parts of the key axis hold alone: their keys weigh nothing beside others."""
    L, page = 9000, 64
    g = gen(S)
    a = layer(Hq, Hq, Dh, dtype, page=page, scale=1.0)
    table, n_pages = pages_for([L], page, -(-L // page), g)
    ks, vs, kc, vc = fill_cache(table, [L], page, Hq, Dh, n_pages, dtype, g, fill=0.0)
    kc.zero_()
    q = torch.zeros(1, S, Hq * Dh)
    q.view(1, S, Hq, Dh)[..., 5] = 2.0 ** 64
    far = torch.arange(L) < L - S - 2500
    far[-S - 7::5] = False
    for j in range(L):
        if far[j]:
            kc[table[0, j // page], :, j % page, 5] = -2.0 ** 62 * 3.75
    y = run_paged(a, dev(q.to(IO[dtype])), [L], table, kc, vc)[0]
    v = vs[0].double()
    for i in range(S):
        seen = (~far) & (torch.arange(L) <= L - S + i)
        n = int(seen.sum())
        want = v[seen].mean(0, keepdim=True)
        check(y[i:i + 1], want, v[seen].abs().mean(0, keepdim=True) * (HALF[dtype] + 4 * (n + 16) * U), i)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", SIZES, ids=lambda c: "-".join(str(v) for v in c))
def test_scores_of_minus_infinity_give_zeros_whatever_the_values(case, dtype):
    B, S, Hq, Hk, Dh, L = case
    g = gen(S + L)
    a = layer(Hq, Hk, Dh, dtype, page=16)
    lens = [L - 7 * b for b in range(B)]
    table, n_pages = pages_for(lens, 16, -(-L // 16), g)
    _, _, kc, vc = fill_cache(table, lens, 16, Hk, Dh, n_pages, dtype, g, fill=0.0)
    vc[table[0, ::2].long(), :, 3, ::5] = float("nan")
    vc[table[0, ::2].long(), :, 7, 1::7] = float("inf")
    vc[table[0, -(-L // 16) - 1], :, :, 1] = float("-inf")
    kc.zero_()
    kc[..., 0] = float("-inf")
    q = dev(torch.ones(B, S, Hq * Dh).to(IO[dtype]))
    assert bool((run_paged(a, q, lens, table, kc, vc, [min(S, n) for n in lens])[0] == 0).all())
    k, v = torch.zeros(B, L, Hk * Dh), torch.randn(B, L, Hk * Dh, generator=g)
    k[..., ::Dh] = float("-inf")
    v[0, ::3, 5], v[0, L // 2:, 2] = float("nan"), float("inf")
    assert bool((run_cross(a, q, dev(k.to(IO[dtype])), dev(v.to(IO[dtype])))[0] == 0).all())
