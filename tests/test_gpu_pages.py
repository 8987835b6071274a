"""Page tables along the beam on the GPU against their definition row by row (attn_ref)."""
import pytest

torch = pytest.importorskip("torch")

import attn_ref as ref
from paper_1804_00344_amd import mtstep as mt
from test_gpu_attn import layer, space
from test_gpu_layer import DEV, IO, dev, gen

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def i32(a):
    return dev(torch.tensor(a, dtype=torch.int32))


def as_table(rows, n_blocks, junk):
    t = torch.full((len(rows), n_blocks), junk, dtype=torch.int32)
    for m, r in enumerate(rows):
        t[m, :len(r)] = torch.tensor(r, dtype=torch.int32)
    return t


class Pool:
    """A cache of several layers, its tables, and the same on the host."""

    def __init__(self, a, layers, n_pages, n_blocks, seed):
        self.a, self.n_pages, self.n_blocks, self.page = a, n_pages, n_blocks, a.cfg.page
        g = gen(seed)
        shape = (layers, n_pages) + tuple(a.page_shape)
        self.k, self.v = (torch.randn(shape, generator=g).to(a.dtype) for _ in range(2))
        self.dk, self.dv = dev(self.k), dev(self.v)
        self.rows = []

    def advance(self, row, add, plain=False):
        """One call, checked against the definition; False where there is no room."""
        M, ws = len(row), space(mt.mt_pages_workspace_bytes(self.a, len(row), self.n_pages))
        ws.fill_(255)
        rows = self.rows or [(0, [])]
        want = ref.advance(rows, row, add, self.page, self.n_blocks, self.n_pages)
        table, lens = as_table([r[1] for r in rows], self.n_blocks, -77), [r[0] for r in rows]
        to = torch.empty(M, self.n_blocks, dtype=torch.int32, device=DEV)
        ln, fr = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
        mt.mt_pages_advance(self.a, None if plain else i32(row), None if plain else i32(add), dev(table), i32(lens), to, ln,
                            self.dk, self.dv, free_out=fr, ws=ws)
        err = mt.mt_attn_device_errors(self.a)
        if want is None:
            assert err == 8 and bool((ln == 0).all()) and bool((to == -1).all()) and int(fr) == self.n_pages
            assert torch.equal(self.dk.cpu(), self.k) and torch.equal(self.dv.cpu(), self.v)
            return False
        assert err == 0
        tables, lengths, free, copies = want
        assert torch.equal(to.cpu(), as_table(tables, self.n_blocks, -1)), (to.cpu(), tables)
        assert ln.tolist() == lengths and int(fr) == free
        for t in (self.k, self.v):
            for s, d, n in copies:
                t[:, d, :, :n] = t[:, s, :, :n]
        assert torch.equal(self.dk.cpu(), self.k) and torch.equal(self.dv.cpu(), self.v)
        self.rows = list(zip(lengths, tables))
        return True


@pytest.mark.parametrize("dtype,Hk,Dh,page,layers", [("f32", 1, 8, 8, 1), ("bf16", 3, 40, 16, 2), ("bf16", 2, 64, 32, 3)])
def test_prompts_then_beam(dtype, Hk, Dh, page, layers):
    """Prompts, a beam started from them, steps that shuffle it, finished hypotheses, new prompts in their place."""
    a = layer(Hk, Hk, Dh, dtype, page=page)
    p = Pool(a, layers, 150, 12, 1)
    lens = [0, 1, page, page + 1, 3 * page - 1]
    assert p.advance([-1] * 5, lens)
    K = 4
    assert p.advance([m // K for m in range(5 * K)], [1] * (5 * K))
    g = gen(2)
    for t in range(10):
        row = [b * K + int(r) for b in range(5) for r in torch.randint(0, K, (K,), generator=g)]
        add = [1] * 20 if t % 3 else torch.randint(0, 4, (20,), generator=g).tolist()
        if t == 5:
            row[3] = row[9] = -1
        assert p.advance(row, add)
    assert p.advance(list(range(20)), [1] * 20, plain=True)
    assert p.advance([-1, 7, -1, 7], [page, 0, 5, 2 * page])
    assert p.advance([-1] * 3, [0] * 3) and p.rows == [(0, [])] * 3


def test_shared_pages_of_rows_that_stay_and_grow():
    """A row that does not grow, and one whose length was cut, hold on to what others copy."""
    a = layer(1, 1, 8, "f32", page=8)
    p = Pool(a, 2, 40, 6, 3)
    assert p.advance([-1], [13])
    assert p.advance([0, 0, 0], [0, 1, 2])
    assert p.advance([0, 0, 1, 1, 2], [1, 1, 1, 0, 0])
    n, pages = p.rows[2]
    p.rows[1] = (n - 3, pages)  # shorter than another row of the same pages
    p.rows[0] = (6, pages)      # and one that ends inside a page that others have filled
    assert p.advance([0, 1, 2, 0], [1, 1, 1, 1])


def test_no_room():
    a = layer(1, 1, 8, "f32", page=8)
    p = Pool(a, 1, 5, 3, 4)
    assert p.advance([-1, -1], [16, 17])            # all five pages
    assert not p.advance([0, 1], [1, 0])            # none is left
    assert not p.advance([0, 1, 1], [0, 1, 1])      # for the copy neither
    assert p.advance([0, 1], [0, 7])                # inside a page there is room
    assert not p.advance([0, 1], [0, 1])            # past the blocks of a table
    assert not p.advance([0, -1], [2 ** 30, 0])
    assert p.advance([0, -1], [8, 0])               # a row given back makes room
    assert p.advance([-1, 0], [16, 0])


@pytest.mark.parametrize("M,n_pages", [(1, 1), (300, 5000), (700, 9000)])
def test_many_rows_and_pages(M, n_pages):
    """More rows and pages than one workgroup takes."""
    a = layer(1, 1, 8, "bf16", page=8)
    p = Pool(a, 1, n_pages, 20, 5)
    g = gen(M)
    most = min(8 * n_pages // M, 90)
    assert p.advance([-1] * M, torch.randint(0, most + 1, (M,), generator=g).tolist())
    if M > 1:
        for _ in range(3):
            row = torch.randint(-1, M, (M,), generator=g).tolist()
            p.advance(row, torch.randint(0, 9, (M,), generator=g).tolist())


def test_out_of_range_is_clamped_and_reported():
    a = layer(1, 1, 8, "f32", page=8)
    k, v = (torch.randn(1, 6, 1, 8, 8, device=DEV) for _ in range(2))
    ws = space(mt.mt_pages_workspace_bytes(a, 2, 6))
    to, ln = torch.empty(2, 3, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)

    def call(row, add, table, lens):
        mt.mt_pages_advance(a, i32(row), i32(add), i32(table), i32(lens), to, ln, k, v, ws=ws)
        return mt.mt_attn_device_errors(a), to.tolist(), ln.tolist()

    t = [[2, 3, -5], [4, -5, -5]]
    assert call([0, 9], [1, 0], t, [10, 5]) == (1, [[2, 3, -1], [4, -1, -1]], [11, 5])
    assert call([0, 1], [1, -3], t, [10, 5]) == (2, [[2, 3, -1], [4, -1, -1]], [11, 5])
    assert call([0, 1], [0, 0], t, [10, -5]) == (2, [[2, 3, -1], [-1, -1, -1]], [10, 0])
    assert call([0, 1], [0, 0], [[2, 3, 1], [4, 5, 0]], [99, 5]) == (2, [[2, 3, 1], [4, -1, -1]], [24, 5])
    assert call([0, 1], [0, 0], [[2, 77, 1], [-4, 5, 0]], [10, 5]) == (4, [[2, 5, -1], [0, -1, -1]], [10, 5])


@pytest.mark.parametrize("dtype,Hk,Dh,page,layers,M", [("f32", 1, 8, 8, 1, 4), ("bf16", 3, 40, 16, 2, 9), ("bf16", 1, 8, 8, 1, 600)])
def test_pack(dtype, Hk, Dh, page, layers, M):
    a = layer(Hk, Hk, Dh, dtype, page=page)
    n_pages = 40 * M // 4 + 30
    p = Pool(a, layers, n_pages, 8, 6)
    g = gen(7)
    assert p.advance([-1] * M, torch.randint(0, 5 * page, (M,), generator=g).tolist())
    assert p.advance(torch.randint(-1, M, (M,), generator=g).tolist(), [1] * M)
    tables, used = ref.pack(p.rows, page)
    ws = space(mt.mt_pages_workspace_bytes(a, M, n_pages))
    for n_out in (len(used), len(used) + 7, len(used) - 1):
        ws.fill_(255)
        ko, vo = (torch.full((layers, n_out) + tuple(a.page_shape), 7.0, dtype=IO[dtype], device=DEV) for _ in range(2))
        to, ln = torch.empty(M, 8, dtype=torch.int32, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV)
        un = torch.empty(1, dtype=torch.int32, device=DEV)
        mt.mt_pages_pack(a, dev(as_table([r[1] for r in p.rows], 8, -77)), i32([r[0] for r in p.rows]), p.dk, p.dv, to, ln, ko,
                         vo, un, ws=ws)
        if n_out < len(used):
            assert mt.mt_attn_device_errors(a) == 8 and int(un) == 0 and bool((ln == 0).all()) and bool((to == -1).all())
            assert bool((ko == 7).all()) and bool((vo == 7).all())
            continue
        assert mt.mt_attn_device_errors(a) == 0 and int(un) == len(used) and ln.tolist() == [r[0] for r in p.rows]
        assert torch.equal(to.cpu(), as_table(tables, 8, -1))
        for out, src in ((ko, p.k), (vo, p.v)):
            assert torch.equal(out[:, :len(used)].cpu(), src[:, used]) and bool((out[:, len(used):] == 7).all())


@pytest.mark.parametrize("M,n_pages,n_blocks,layers", [
    (256, 1024, 8, 2), (256, 1024, 8, 3), (255, 1023, 3, 6), (257, 1024, 7, 1), (200, 1025, 10, 1), (100, 1000, 21, 1),
    (2048, 8192, 16, 1), (2049, 8192, 15, 1)])
def test_at_the_sizes_where_the_plan_changes(M, n_pages, n_blocks, layers):
    """Every workgroup its own plan, one workgroup's, many workgroups': room, no room, entries out of range, packed."""
    a = layer(1, 1, 8, "bf16", page=8)
    p = Pool(a, layers, n_pages, n_blocks, 8)
    g = gen(M + layers)
    most = min(8 * n_pages // (2 * M), 8 * n_blocks - 3)
    assert p.advance([-1] * M, torch.randint(0, most + 1, (M,), generator=g).tolist())
    row = torch.randint(-1, M, (M,), generator=g).tolist()
    assert p.advance(row, torch.randint(0, 3, (M,), generator=g).tolist())
    kept = list(p.rows)
    assert not p.advance(list(range(M)), [0] * (M - 1) + [8 * n_blocks])  # past the blocks of a table
    if n_pages < M * n_blocks:
        assert not p.advance(list(range(M)), [8 * n_blocks - n for n, _ in kept])  # all that tables have room for
    # pages out of range: clamped and reported
    table = as_table([r[1] for r in kept], n_blocks, -77)
    long = [m for m, (n, _) in enumerate(kept) if n > 8]
    table[long[0], 0], table[long[-1], 1] = -3, n_pages + 5
    clean = table.clone()
    clean[long[0], 0], clean[long[-1], 1] = 0, n_pages - 1
    ws = space(mt.mt_pages_workspace_bytes(a, M, n_pages))
    got = []
    for t in (table, clean):
        to, ln = torch.empty(M, n_blocks, dtype=torch.int32, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV)
        mt.mt_pages_advance(a, i32(list(range(M - 1)) + [M]), i32([0] * M), dev(t), i32([n for n, _ in kept]), to, ln, p.dk, p.dv, ws=ws)
        got.append((mt.mt_attn_device_errors(a), to, ln))
    assert got[0][0] == 1 | 4 and got[1][0] == 1
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2]) and got[1][2].tolist() == [n for n, _ in kept]
    # packed
    tables, used = ref.pack(kept, 8)
    n_out = len(used) + 2
    ko, vo = (torch.full((layers, n_out) + tuple(a.page_shape), 7.0, dtype=IO["bf16"], device=DEV) for _ in range(2))
    to, ln, un = torch.empty(M, n_blocks, dtype=torch.int32, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV), i32([0])
    mt.mt_pages_pack(a, dev(as_table([r[1] for r in kept], n_blocks, -77)), i32([n for n, _ in kept]), p.dk, p.dv, to, ln, ko, vo,
                     un, ws=ws)
    assert mt.mt_attn_device_errors(a) == 0 and int(un) == len(used) and ln.tolist() == [n for n, _ in kept]
    assert torch.equal(to.cpu(), as_table(tables, n_blocks, -1))
    for out, src in ((ko, p.k), (vo, p.v)):
        assert torch.equal(out[:, :len(used)].cpu(), src[:, used]) and bool((out[:, len(used):] == 7).all())
