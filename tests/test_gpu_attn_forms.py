"""The attention layer's operators at sizes that every form of their kernels takes (which one, tests/test_attn_forms_cpu.py says
without a GPU): tiles of 128 rows, whole and in parts, joins of many parts, the shapes of a launch of mt_attn_append, plans of many
workgroups."""
import math

import pytest

torch = pytest.importorskip("torch")

import attn_ref as ref
import test_gpu_attn as attn
from paper_1804_00344_amd import mtstep as mt
from test_gpu_attn import HALF, NAN, fill_cache, layer, pages_for, run_cross, run_paged
from test_gpu_layer import DEV, IO, dev, gen, wide

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def i32(a):
    return dev(torch.tensor(a, dtype=torch.int32))


def name(c):
    return "-".join(str(v) for v in c[:7])


# B, S, Hq, Hk, Dh, page, window, lens, n_new: tiles of 128 rows
TILES = [
    (4, 500, 16, 16, 128, 16, 0, [500, 433, 500, 77], [500, 433, 300, 77]),
    (8, 130, 32, 8, 96, 32, 0, [130, 190, 0, 131, 60, 130, 150, 180], [130, 129, 0, 130, 60, 1, 7, 130]),
    (8, 130, 32, 8, 128, 16, 57, [130 + 3 * b for b in range(8)], [130 - 11 * b for b in range(8)]),
    (8, 300, 16, 16, 72, 8, 0, [300 - 20 * b for b in range(8)], [300 - 20 * b for b in range(8)]),
    (8, 300, 16, 16, 64, 16, 33, [300 + b for b in range(8)], [300 - b for b in range(8)]),
]
TILE_PARTS = [  # and in parts
    (1, 300, 8, 8, 128, 64, 0, [4100], [299]),
    (1, 300, 16, 16, 72, 16, 2500, [4100], None),
    (3, 500, 16, 16, 128, 16, 0, [6000, 1500, 600], [500, 500, 433]),  # twice the parts, for sequences of different lengths
    (3, 300, 8, 8, 64, 32, 0, [5900, 400, 300], [300, 299, 300]),
]
# one to eight rows of one key head over more than 16640 positions: more than 64 parts, in a row's and a join's second round
MANY_PARTS = [(1, 1, 1, 1, 64, 64, 0, [20400], None), (1, 1, 8, 1, 64, 128, 0, [20400], None), (1, 1, 1, 1, 128, 64, 0, [17001], None),
              (1, 1, 8, 1, 256, 256, 0, [20400], None), (2, 1, 1, 1, 200, 64, 0, [17000, 3], None)]
# B, T, S, Hq, Hk, Dh, mask, n_q
TILE_CROSS = [(4, 500, 300, 16, 16, 128, "ends", [500, 499, 3, 500]), (8, 520, 100, 16, 16, 96, "holes", None),
              (16, 520, 90, 16, 8, 128, "holes", [520 - 31 * b for b in range(16)]), (8, 300, 150, 16, 16, 72, None, None)]
TILE_CROSS_PARTS = [(1, 300, 4200, 8, 8, 128, "holes", None), (2, 200, 5000, 8, 4, 104, "ends", [200, 199])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", TILES + TILE_PARTS + MANY_PARTS, ids=name)
def test_paged_forms(case, dtype):
    attn.test_paged(case, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", TILE_CROSS + TILE_CROSS_PARTS, ids=name)
def test_cross_forms(case, dtype):
    attn.test_cross(case, dtype)


# B, S, Hq, Hk, Dh, L, window: tiles of 128 rows in which rows see different keys
UNSEEN = [(8, 300, 16, 16, 64, 310, 0), (8, 300, 16, 16, 64, 310, 90), (4, 500, 16, 16, 128, 520, 0), (8, 130, 32, 8, 96, 180, 57)]
UNSEEN_PARTS = [(1, 300, 8, 8, 64, 4700, 0), (1, 300, 8, 8, 128, 4200, 0), (1, 300, 16, 16, 72, 4160, 2500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", UNSEEN + UNSEEN_PARTS, ids=name)
def test_unseen_nonfinite_values_in_tiles(case, dtype):
    """Infinities and NaN at positions that some rows of a tile see and others not: those that do not give what the formula
    gives over theirs, the others no numbers; the other key heads and sequences are as they were."""
    B, S, Hq, Hk, Dh, L, window = case
    g = gen(S + L)
    a = layer(Hq, Hk, Dh, dtype, page=16, window=window)
    lens = [L - 3 * b for b in range(B)]
    table, n_pages = pages_for(lens, 16, -(-L // 16), g)
    ks, vs, kc, vc = fill_cache(table, lens, 16, Hk, Dh, n_pages, dtype, g)
    q = torch.randn(B, S, Hq * Dh, generator=g).to(IO[dtype])
    clean = run_paged(a, dev(q), lens, table, kc, vc)
    bad = {L - S // 2: NAN, L - S // 2 + 1: float("inf"), L - 40: float("-inf")}
    if window:
        bad = {L - 20: NAN, L - S - window + S // 2: float("inf")}
    for j, x in bad.items():
        for c in (kc, vc):
            c[table[0, j // 16], 0, j % 16, 3:9] = x
        ks[0][j], vs[0][j] = 0, 0
    y = run_paged(a, dev(q), lens, table, kc, vc)
    assert torch.equal(y[1:], clean[1:]) and torch.equal(y[0, :, Hq // Hk * Dh:], clean[0, :, Hq // Hk * Dh:])
    G, seen = Hq // Hk, ref.causal(L - S, S, L, window)
    dirty = seen[:, sorted(bad)].any(1)
    assert bool(dirty.any()) and bool((~dirty).any())
    y = y[0, :, :G * Dh].cpu().double()
    assert not bool(torch.isfinite(y[dirty][:, :Dh]).all(1).any())
    want, err = ref.heads(q[0, :, :G * Dh].double(), ks[0][:, :Dh].double(), vs[0][:, :Dh].double(), seen, G, 1, 1 / math.sqrt(Dh),
                          HALF[dtype])
    tol = err + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (want.abs() + err) + 1e-37
    assert bool(((y - want).abs() <= tol)[~dirty].all())


# and of the other forms: B, S, Hq, Hk, Dh, L, window
UNSEEN_FEW = [(2, 1, 8, 1, 64, 90, 40), (1, 20, 2, 2, 128, 3000, 0), (3, 9, 6, 2, 40, 120, 30), (2, 4, 2, 2, 256, 300, 0), (300, 5, 8, 8, 64, 60, 0),
              (2, 60, 4, 4, 192, 200, 70)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", UNSEEN + UNSEEN_PARTS + UNSEEN_FEW, ids=name)
def test_values_that_are_no_numbers_reach_their_features_alone(case, dtype):
    """Infinities and NaN among the values, in features of their own: the formula's results for who sees them (infinities of
    their sign, NaN for NaN and for both signs together) and for every other feature and row."""
    B, S, Hq, Hk, Dh, L, window = case
    g = gen(S + L + 1)
    a = layer(Hq, Hk, Dh, dtype, page=16, window=window)
    table, n_pages = pages_for([L] * B, 16, -(-L // 16), g)
    ks, vs, kc, vc = fill_cache(table, [L] * B, 16, Hk, Dh, n_pages, dtype, g)
    inf, far = float("inf"), max(L - S - (window or 99) + S // 2, 0)
    bad = [(L - S // 2 - 1, 3, NAN), (L - 1, 4, inf), (L - S // 2 - 1, 5, -inf), (L - S // 3 - 1, 6, inf), (L - 1, 6, -inf), (far, 7, inf),
           (far, 2, NAN), (min(far + 1, L - 1), Dh - 1, -inf)]
    bad = [(j, f, x) for (j, f), x in {(j, f): x for j, f, x in bad}.items()]  # of a position's two the last
    for j, f, x in bad:
        vc[table[0, j // 16], 0, j % 16, f] = x
        vs[0][j, f] = 0
    q = torch.randn(B, S, Hq * Dh, generator=g).to(IO[dtype])
    y = run_paged(a, dev(q), [L] * B, table, kc, vc)
    seen, G = ref.causal(L - S, S, L, window), Hq // Hk
    want, err = ref.heads(q[0].double(), ks[0].double(), vs[0].double(), seen, Hq, Hk, 1 / math.sqrt(Dh), HALF[dtype])
    for j, f, x in bad:
        for h in range(G):
            want[:, h * Dh + f] += torch.where(seen[:, j], torch.tensor(x, dtype=torch.float64), 0.0)
    got, half = y[0].cpu().double(), 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    numbers = torch.isfinite(want)
    assert bool((~numbers).any()) and torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    tol = err + half * (want.abs() + err) + 1e-37
    assert bool(((got - want).abs() <= tol)[numbers].all())
    assert bool(torch.isfinite(y[1:]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dh", [64, 128, 192])
@pytest.mark.parametrize("shift", [1, 3])
def test_rows_of_wider_matrices_in_tiles(shift, Dh, dtype):
    """Rows that start at any element, read and written by tiles of 128 rows, are the aligned ones to the bit."""
    a = layer(16, 16, Dh, dtype)
    g = gen(7)
    lens = [300 - b for b in range(8)]
    table, n_pages = pages_for(lens, 16, 19, g)
    _, _, kc, vc = fill_cache(table, lens, 16, 16, Dh, n_pages, dtype, g)
    W = 16 * Dh
    q = torch.randn(8, 300, W, generator=g).to(IO[dtype])
    k, v = (torch.randn(8, 100, W, generator=g).to(IO[dtype]) for _ in range(2))
    for run, want in ((lambda x, y: run_paged(a, x, lens, table, kc, vc, lens, y=y), run_paged(a, dev(q), lens, table, kc, vc, lens)),
                      (lambda x, y: run_cross(a, x, wide(k, shift, 1), wide(v, 0, shift), y=y), run_cross(a, dev(q), dev(k), dev(v)))):
        big = torch.full((8, 300, W + shift + 3), 7.0, dtype=q.dtype, device=DEV)
        run(wide(q, shift, 2), big[..., shift:shift + W])
        assert torch.equal(big[..., shift:shift + W], want)
        assert bool((big[..., :shift] == 7).all()) and bool((big[..., shift + W:] == 7).all())


FAR = (1, 600, 64, 8, 128, 1000)


def test_a_cache_past_32_bits_in_tiles():
    """Pages beyond 2^32 bytes and 2^31 elements, read by tiles of 128 rows."""
    B, S, Hq, Hk, Dh, L = FAR
    page = 64
    n_pages = 2 ** 33 // (Hk * Dh * page * 2) + 40  # 8 GiB each
    a = layer(Hq, Hk, Dh, "bf16", page=page)
    g = gen(9)
    small = torch.arange(16, dtype=torch.int32)[None]
    _, _, kc, vc = fill_cache(small, [L], page, Hk, Dh, 16, "bf16", g)
    k, v = (torch.empty(n_pages, Hk, page, Dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    at = [n_pages - 1 - 3 * i if i % 2 else 2 ** 31 // (Hk * Dh * page) + i for i in range(16)]
    for i, p in enumerate(at):
        k[p], v[p] = dev(kc[i]), dev(vc[i])
    q = torch.randn(B, S, Hq * Dh, generator=g).bfloat16()
    y = run_paged(a, dev(q), [L], torch.tensor([at], dtype=torch.int32), k, v)
    assert torch.equal(y, run_paged(a, dev(q), [L], small, kc, vc)) and bool(torch.isfinite(y).all())


# B, S, Hq, Hk, Dh, page, norm, rot, pairs, lens, n_new
APPEND_STREAM = [(3, 2051, 32, 8, 128, 16, True, 128, False, [2051, 9000, 2051], [2051, 1026, 3])]
APPEND_16 = [(20, 1003, 2, 1, 64, 16, True, 64, False, [1003 + 50 * b for b in range(20)], [1003 - 52 * b for b in range(20)]),
             (20, 1003, 2, 1, 64, 32, True, 40, True, [1003] * 20, [1003 - 7 * b for b in range(20)]),
             (41, 400, 3, 1, 40, 8, False, 40, False, [400 + b for b in range(41)], [400 - 9 * b for b in range(41)])]
APPEND_4 = [(5, 1001, 2, 1, 64, 16, True, 64, False, [1001, 2000, 1001, 1005, 999], [1001, 999, 2, 0, 999]),
            (9, 500, 6, 2, 128, 64, True, 128, False, [500] * 9, [500 - 41 * b for b in range(9)])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", APPEND_STREAM + APPEND_16 + APPEND_4, ids=lambda c: "-".join(str(v) for v in c[:9]))
def test_append_forms(case, dtype):
    """And in place, whose rows of odd strides take the form without streaming, to the bit."""
    attn.test_append(case, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_graphs_share_the_workspace_of_a_plan_of_many_workgroups(dtype):
    """Tables and packed caches beyond one workgroup's plan, captured in two graphs that share a workspace, replayed in turn over
    changed inputs with eager calls between them: every replay gives the eager result."""
    io = IO[dtype]
    a = layer(1, 1, 8, dtype, page=8)
    g = gen(8)
    sizes = [(700, 9000, 4), (2500, 6000, 2)]  # rows, pages, blocks
    ws = torch.empty(max(mt.mt_pages_workspace_bytes(a, M, n) for M, n, _ in sizes), dtype=torch.uint8, device=DEV)
    src = [i32(list(range(M))) for M, _, _ in sizes]
    table = [torch.arange(M, dtype=torch.int32, device=DEV)[:, None].repeat(1, nb) for M, _, nb in sizes]
    lens = [torch.full((M,), 5, dtype=torch.int32, device=DEV) for M, _, _ in sizes]
    pool = [[torch.randn(1, n, 1, 8, 8, generator=g).to(io).to(DEV) for _, n, _ in sizes] for _ in range(2)]

    def outputs(i):
        M, n, nb = sizes[i]
        e = lambda *s: torch.empty(*s, dtype=torch.int32, device=DEV)
        return e(M, nb), e(M), e(1), e(M, nb), e(M), e(1), torch.empty_like(pool[0][i]), torch.empty_like(pool[1][i])

    def call(i, out):
        mt.mt_pages_advance(a, src[i], None, table[i], lens[i], out[0], out[1], pool[0][i], pool[1][i], free_out=out[2], ws=ws)
        mt.mt_pages_pack(a, out[0], out[1], pool[0][i], pool[1][i], out[3], out[4], out[6], out[7], out[5], ws=ws)

    outs, graphs = [outputs(0), outputs(1)], []
    for i in range(2):
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            call(i, outs[i])
        torch.cuda.synchronize()
        graphs.append(graph)
    for _ in range(4):
        for i in (0, 1, 0):
            M, n, nb = sizes[i]
            src[i].copy_(torch.randint(-1, M, (M,), generator=g).int())
            lens[i].copy_(torch.randint(1, 8, (M,), generator=g).int())
            pages = [p.clone() for p in pool[0][i:i + 1] + pool[1][i:i + 1]]
            want = outputs(i)
            for x in want + outs[i]:
                x.fill_(7)
            call(i, want)
            after = [p.clone() for p in (pool[0][i], pool[1][i])]
            pool[0][i].copy_(pages[0]), pool[1][i].copy_(pages[1])
            graphs[i].replay()
            torch.cuda.synchronize()
            assert int(want[5]) > 0 and int(want[5]) + int(want[2]) == n
            for x, y in zip(outs[i] + (pool[0][i], pool[1][i]), want + tuple(after)):
                assert torch.equal(x, y), i
    assert mt.mt_attn_device_errors(a) == 0
