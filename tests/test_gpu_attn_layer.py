"""The attention layer's operators together, as runner.AttnLayer calls them: pieces of ragged prompts, then hypotheses that
fork along a beam, two layers over one page table, cross attention to encoder states.  Every stage is checked in 64 bits
from the inputs that the GPU's stage read, the cache against the history of every hypothesis to the bit."""
import math

import pytest

torch = pytest.importorskip("torch")

import attn_ref as aref
import layer_ref as ref
from paper_1804_00344_amd import mtstep as mt
from test_gpu_attn import HALF
from test_gpu_layer import DEV, check, gen
from test_gpu_ssm_layer import check_product

if torch.cuda.is_available():
    from paper_1804_00344_amd.runner import AttnLayer, PagedCache

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

E, HQ, HK, DH, PAGE, C = 48, 4, 2, 40, 8, 64
QD, KD = HQ * DH, HK * DH
FREQ = 500.0 ** (-torch.arange(0, DH, 2, dtype=torch.float64) / DH)


def weights(seed, cross=True):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    w = dict(Wqkv=r(E, QD + 2 * KD) / 4, bqkv=r(QD + 2 * KD) / 4, Wo=r(QD, E) / 12, bo=r(E), gq=1 + r(DH) / 8, gk=1 + r(DH) / 8)
    if cross:
        w.update(Wcq=r(E, QD) / 4, Wckv=r(C, 2 * KD) / 6, Wco=r(QD, E) / 12, bco=r(E))
    return w


def make(seed, dtype, **kw):
    w = weights(seed)
    return w, AttnLayer(w, HQ, HK, page=PAGE, dtype=dtype, qk_norm=True, rot=DH, rot_base=500.0, **kw)


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def cached(cache, layer, m):
    """Row m's keys and values [len, KD] through its table."""
    n, t = int(cache.lens[m]), cache.table[m].tolist()
    rows = [c[layer][t[p // PAGE], :, p % PAGE].reshape(-1) for c in (cache.k, cache.v) for p in range(n)]
    return (torch.stack(rows[:n]).cpu(), torch.stack(rows[n:]).cpu()) if n else (torch.zeros(0, KD), torch.zeros(0, KD))


def check_self(f, w, u, cache, li, new, hist):
    """One pass of layer li over rows with `new` new positions each; hist: (k, v) of each row, which it extends."""
    check_product(u.reshape(-1, E), "Wqkv", "bqkv", w, before(f, u, w), "qkv")
    for m, n in enumerate(new):
        k, v = cached(cache, li, m)
        L = len(k)
        old = hist[m]
        assert L == len(old[0]) + n and torch.equal(k[:L - n], old[0]) and torch.equal(v[:L - n], old[1]), m
        raw = f["raw"][m, :n].double().cpu()
        pos = torch.arange(L - n, L)
        want, err = aref.turn_heads(raw[:, :QD], pos, DH, True, 1e-6, w["gq"].double(), DH, False, FREQ)
        check(f["qkv"][m, :n, :QD], want, err, "q")
        want, err = aref.turn_heads(raw[:, QD:QD + KD], pos, DH, True, 1e-6, w["gk"].double(), DH, False, FREQ)
        check(k[L - n:], want, err, "k")
        assert torch.equal(v[L - n:].double(), raw[:, QD + KD:])
        q = f["qkv"][m, :n, :QD].double().cpu()
        want, err = aref.heads(q, k.double(), v.double(), aref.causal(L - n, n, L, 0), HQ, HK, 1 / math.sqrt(DH), HALF[f["dt"]])
        check(f["y"][m, :n], want, err, "y")
        if n:
            check_product(f["y"][m, :n], "Wo", "bo", w, f["out"][m, :n], "out")
        hist[m] = (k, v)


def before(f, u, w):
    """The projection before q was rotated in place, made again by the same call."""
    return f["raw"].reshape(-1, QD + 2 * KD)


def project(layer, f, u, dtype):
    f["raw"], f["dt"] = torch.zeros_like(f["qkv"]), dtype
    mt.mt_i8_product(layer.wqkv, u, f["raw"], f["ws"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_then_beam(dtype):
    B, S, K, S_src, n_blocks = 3, 19, 4, 23, 8
    both = [make(s, dtype) for s in (3, 4)]
    attn = both[0][1].attn
    cache = PagedCache(attn, 2, 100, n_blocks)
    for _, l in both:
        l.set_batch(B, S, K, n_blocks * PAGE, S_src)
    g = gen(5)
    rand = lambda *s: torch.randn(*s, generator=g).to(attn.dtype).to(DEV)
    hist = [[(torch.zeros(0, KD).to(attn.dtype),) * 2 for _ in range(B)] for _ in both]
    rows = i32([-1] * B)
    for new in ([19, 0, 7], [5, 3, 19]):  # two pieces of each prompt
        cache.advance(rows, i32(new))
        rows = i32(list(range(B)))
        for li, (w, l) in enumerate(both):
            u = rand(B, S, E)
            project(l, l.pb, u, dtype)
            l.prompt(u, cache, li, i32(new))
            check_self(l.pb, w, u, cache, li, new, hist[li])
    ctx = rand(B, S_src, C)
    mask = (torch.rand(B, S_src, generator=g) < 0.7).float()
    mask[1] = 0
    for _, l in both:
        l.set_source(ctx, mask.to(DEV))
    src = [m // K for m in range(B * K)]
    for t in range(6):
        cache.advance(i32(src))
        for li, (w, l) in enumerate(both):
            hist[li] = [hist[li][r] for r in src]
            u = rand(B * K, E)
            project(l, l.sb, u[:, None], dtype)
            l.step(u, cache, li)
            check_self(l.sb, w, u[:, None], cache, li, [1] * (B * K), hist[li])
            out = l.cross(u)
            f = l.xb
            q = f["qkv"].view(-1)[:B * K * QD].view(B, K, QD)
            check_product(u, "Wcq", None, w, q.reshape(-1, QD), "cq")
            check_product(ctx.reshape(-1, C), "Wckv", None, w, l.src_kv.reshape(-1, 2 * KD), "ckv")
            for b in range(B):
                kv = l.src_kv[b].cpu().double()
                want, err = aref.heads(q[b].cpu().double(), kv[:, :KD], kv[:, KD:], (mask[b] != 0)[None].expand(K, -1), HQ, HK,
                                       1 / math.sqrt(DH), HALF[dtype])
                check(f["y"][b], want, err, "cross")
            check_product(f["y"], "Wco", "bco", w, out, "co")
        if t == 3:  # into a cache of just the pages in use, and on from there
            used = cache.k.shape[1] - int(cache.free)
            cache = cache.pack(used + B * K * 2)
            assert int(cache.free) == B * K * 2
        src = [b * K + int(r) for b in range(B) for r in torch.randint(0, K, (K,), generator=g)]
    for _, l in both:
        assert mt.mt_attn_device_errors(l.attn) == 0


def test_a_step_in_a_graph():
    """A step of the tables and two layers captured once and replayed over the same buffers, with eager work between the
    replays: every replay gives the eager result."""
    B, K, n_blocks = 2, 4, 4
    (w, l), (_, l2) = make(3, "bf16"), make(4, "bf16")
    cache = PagedCache(l.attn, 2, 60, n_blocks)
    for x in (l, l2):
        x.set_batch(B, 9, K, n_blocks * PAGE, 0)
    g = gen(6)
    cache.advance(i32([-1] * B), i32([9, 4]))
    u = torch.randn(B, 9, E, generator=g).bfloat16().to(DEV)
    l.prompt(u, cache, 0, i32([9, 4]))
    l2.prompt(u, cache, 1, i32([9, 4]))
    src = i32([m // K for m in range(B * K)])
    prompt = cache.table, cache.lens
    k0, v0 = cache.k.clone(), cache.v.clone()
    tok = torch.zeros(B * K, E, dtype=torch.bfloat16, device=DEV)

    def step():
        cache.table, cache.lens = prompt
        cache.advance(src)
        return l2.step(l.step(tok, cache, 0), cache, 1)

    def eager(x):
        tok.copy_(x)
        cache.k.copy_(k0), cache.v.copy_(v0)
        return step().clone(), cache.table.clone(), cache.lens.clone(), cache.k.clone(), cache.v.clone()

    tokens = [torch.randn(B * K, E, generator=g).bfloat16().to(DEV) for _ in range(4)]
    want = [eager(x) for x in tokens]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = step()
    torch.cuda.synchronize()
    for x, (y, *state) in zip(tokens, want):
        tok.copy_(x)
        cache.k.copy_(k0), cache.v.copy_(v0)
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, cache.table, cache.lens, cache.k, cache.v), (y, *state)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """One layer's calls on two streams, each with its own outputs and workspace."""
    from test_gpu_attn import fill_cache, layer, pages_for, space
    a = layer(8, 2, 64, "bf16", page=16)
    g = gen(7)
    lens = [3000, 2000]
    table, n = pages_for(lens, 16, 200, g)
    _, _, kc, vc = fill_cache(table, lens, 16, 2, 64, n, "bf16", g, fill=0.0)
    table, kc, vc, ln = table.to(DEV), kc.to(DEV), vc.to(DEV), i32(lens)
    qs = [torch.randn(2, S, 512, generator=g).bfloat16().to(DEV) for S in (1, 300)]
    wss = [space(mt.mt_attn_workspace_bytes(a, 2, q.shape[1], 200 * 16)) for q in qs]
    want = []
    for q, ws in zip(qs, wss):
        y = torch.empty_like(q)
        mt.mt_attn_paged(a, q, ln, table, kc, vc, y, ws=ws)
        want.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    ys = [[torch.empty_like(q) for q in qs] for _ in range(5)]
    torch.cuda.synchronize()
    for row in ys:
        for q, ws, y, st in zip(qs, wss, row, streams):
            mt.mt_attn_paged(a, q, ln, table, kc, vc, y, ws=ws, stream=st)
    torch.cuda.synchronize()
    for row in ys:
        assert torch.equal(row[0], want[0]) and torch.equal(row[1], want[1])


def test_a_packed_cache_counts_its_free_pages():
    """Also where other streams than the current one pack and go on."""
    attn = mt.mt_attn_load(mt.make_attn_config(2, 1, 64, page=8))
    cache = PagedCache(attn, 2, 40, 6)
    cache.advance(i32([-1] * 5), i32([3, 0, 17, 8, 9]))  # 1 + 0 + 3 + 1 + 2 pages
    assert int(cache.free) == 33
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    small = cache.pack(12, stream=first)
    assert int(small.free) == 5 and small.lens.tolist() == [3, 0, 17, 8, 9]
    small = cache.pack(12, stream=first)
    small.advance(i32([0, 0, 3]), i32([1, 1, 1]), stream=second)  # a copy of the first page, and a page behind the fourth's
    torch.cuda.synchronize()
    assert int(small.free) == 8 and small.lens.tolist() == [4, 4, 9]
    assert cache.pack(6).lens.tolist() == [0] * 5 and mt.mt_attn_device_errors(attn) == 8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_graphs_with_one_workspace(dtype):
    """Calls of several launches (sorted sentences, long masks, parts, tables of every size) captured in two graphs that share
    a workspace, replayed in turn over changed inputs with eager calls between them: every replay gives the eager result."""
    from test_gpu_attn import layer, space
    io = torch.bfloat16 if dtype == "bf16" else torch.float32
    a = layer(16, 16, 64, dtype, page=8)
    g = gen(8)
    rand = lambda *s: torch.randn(*s, generator=g).to(io).to(DEV)
    # 24 sentences of 300 queries, sorted by their work; 2 of 3 queries over a long mask, in parts
    sizes = [(24, 300, 200), (2, 3, 8400)]
    qs, ks = [rand(B, T, 1024) for B, T, _ in sizes], [rand(B, S, 1024) for B, _, S in sizes]
    masks = [torch.ones(B, S, device=DEV) for B, _, S in sizes]
    need = [mt.mt_attn_workspace_bytes(a, *s) for s in sizes]
    rows = [(40, 300), (300, 2000)]  # and tables: a plan in every workgroup, one workgroup's
    need += [mt.mt_pages_workspace_bytes(a, M, n) for M, n in rows]
    ws = space(max(need))
    table_in = [torch.arange(M, dtype=torch.int32, device=DEV)[:, None].repeat(1, 4) for M, _ in rows]
    len_in, src = [torch.full((M,), 5, dtype=torch.int32, device=DEV) for M, _ in rows], [i32(list(range(M))) for M, _ in rows]
    pool = [[torch.zeros(1, n, 16, 8, 64, dtype=io, device=DEV) for _, n in rows] for _ in range(2)]
    outs = [(torch.empty_like(q), torch.empty_like(t), torch.empty_like(n)) for q, t, n in zip(qs, table_in, len_in)]

    def call(i, out):
        mt.mt_attn_cross(a, qs[i], ks[i], ks[i], out[0], mask=masks[i], ws=ws)
        mt.mt_pages_advance(a, src[i], None, table_in[i], len_in[i], out[1], out[2], pool[0][i], pool[1][i], ws=ws)

    graphs = []
    for i in range(2):
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            call(i, outs[i])
        torch.cuda.synchronize()
        graphs.append(graph)
    for _ in range(4):
        for i in (0, 1, 0):
            B, T, S = sizes[i]
            n = torch.randint(1, S + 1, (B,), generator=g)
            masks[i].copy_((torch.arange(S)[None] < n[:, None]).float())
            qs[i].copy_(rand(B, T, 1024))
            M = rows[i][0]
            src[i].copy_(torch.randint(0, M, (M,), generator=g).int())
            len_in[i].copy_(torch.randint(1, 25, (M,), generator=g).int().clamp(max=8))
            want = [torch.full_like(x, 3) for x in outs[i]]
            call(i, want)
            for x in outs[i]:
                x.fill_(7)
            graphs[i].replay()
            torch.cuda.synchronize()
            for x, y in zip(outs[i], want):
                assert torch.equal(x, y), i
    assert mt.mt_attn_device_errors(a) == 0


@pytest.mark.parametrize("add", [None, [9, 9, 9, 9]])
def test_a_step_without_room_is_taken_back(add):
    """A pool that runs out under a beam: check() tells, gives the rows before back, and the beam goes on with fewer rows."""
    attn = mt.mt_attn_load(mt.make_attn_config(2, 1, 64, page=8))
    cache = PagedCache(attn, 2, 9, 6)
    cache.advance(i32([-1, -1]), i32([16, 11]))  # 2 + 2 pages
    cache.k.normal_(), cache.v.normal_()
    cache.advance(i32([0, 0, 1, 1]))             # two blocks and a copy: 7 in use
    assert cache.check() == 0
    cache.advance(i32([0, 1, 2, 3]))             # inside their pages
    assert cache.check() == 0 and int(cache.free) == 2
    table, lens, k, v = cache.table.clone(), cache.lens.clone(), cache.k.clone(), cache.v.clone()
    many = [m % 4 for m in range(12)] if add is None else [0, 1, 2, 3]
    for _ in range(2):
        cache.advance(i32(many), None if add is None else i32(add))  # more than two copies, or blocks
        assert cache.check() == 8
        assert torch.equal(cache.table, table) and torch.equal(cache.lens, lens) and int(cache.free) == 2
        assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
        assert cache.check() == 0 and torch.equal(cache.lens, lens)  # once
    hist = [cached(cache, layer, m) for layer in range(2) for m in (0, 2)]
    cache.advance(i32([0, 2]), i32([5, 9]))      # the two others' pages are free again
    assert cache.check() == 0 and cache.lens.tolist() == [23, 22] and int(cache.free) == 9 - 3 - 3
    for (layer, m), (hk, hv) in zip([(l, m) for l in range(2) for m in (0, 1)], hist):
        n, (gk, gv) = len(hk), cached(cache, layer, m)
        assert torch.equal(gk[:n], hk) and torch.equal(gv[:n], hv)
    # rows that are given back are no loss: nothing to go back to, whatever another cache of the layer has reported
    cache.advance(i32([-1, -1]), i32([0, 0]))
    assert cache.check() == 0 and cache.lens.tolist() == [0, 0] and int(cache.free) == 9


def test_a_shrinking_beam_stays_in_its_buffers():
    """From 16 hypotheses to 9, and back: no new buffers, no wait for the device, every row what it continues."""
    attn = mt.mt_attn_load(mt.make_attn_config(1, 1, 8, page=8))
    cache = PagedCache(attn, 1, 60, 4)
    cache.advance(i32([-1] * 16), i32([1 + m % 3 for m in range(16)]))
    lens = [1 + m % 3 for m in range(16)]
    g = gen(9)
    cache._wait = lambda: pytest.fail("waits for the device")
    for n in [15, 14, 13, 12, 11, 10, 9, 12, 16]:
        src = torch.randint(0, len(lens), (n,), generator=g).tolist()
        before, pages = cache.table.tolist(), cache.table.data_ptr()
        cache.advance(i32(src))
        lens = [lens[r] + 1 for r in src]
        assert cache.lens.tolist() == lens and cache.table.shape == (n, 4) and cache.table.data_ptr() != pages
        table = cache.table.tolist()
        written = [t[(ln - 1) // 8] for t, ln in zip(table, lens)]
        assert len(set(written)) == n  # a page of its own to go on writing
        for t, r, ln in zip(table, src, lens):
            assert t[:(ln - 1) // 8] == before[r][:(ln - 1) // 8]
    assert mt.mt_attn_device_errors(attn) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tables_follow_a_beam_search(dtype):
    """Prompts, then steps whose hypotheses mt_beam_topk chooses: its row_out is mt_pages_advance's src_row as it stands."""
    from paper_1804_00344_amd import synth
    from paper_1804_00344_amd.runner import Decoder
    B, S, K, V, n_blocks = 3, 13, 4, 500, 4
    w, l = make(3, dtype)
    cache = PagedCache(l.attn, 1, 50, n_blocks)
    l.set_batch(B, S, K, n_blocks * PAGE)
    g = gen(10)
    new = [13, 1, 7]
    cache.advance(i32([-1] * B), i32(new))
    l.prompt(torch.randn(B, S, E, generator=g).to(l.io_dtype).to(DEV), cache, 0, i32(new))
    hist = [cached(cache, 0, m) for m in range(B)]
    p = synth.with_sizes(synth.PRESETS["tiny_f32"], V=V, B=B, K=K)
    dec = Decoder.from_preset(p, synth.make_weights(p))
    M = B * K
    ws = torch.empty(mt.mt_workspace_bytes(dec.model, B, K, 8), dtype=torch.uint8, device=DEV)
    emb, wo = (torch.randn(V, E, generator=g).to(DEV) for _ in range(2))
    score = torch.tensor([0.0] + [-1e30] * (K - 1), device=DEV).repeat(B)  # one live hypothesis each
    tok, bp = torch.ones(M, dtype=torch.int32, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV)
    row = i32([m // K for m in range(M)])  # the first step continues the prompts
    forked = False
    for t in range(8):
        cache.advance(row)
        parents = row.tolist()
        forked = forked or (t > 0 and len(set(parents)) < M)
        out = l.step(emb[tok.long()].to(l.io_dtype), cache, 0)
        v_new = l.sb["qkv"][:, 0, QD + KD:]
        kv = [cached(cache, 0, m) for m in range(M)]
        for m, r in enumerate(parents):  # its parent's positions, and its own
            (k, v), (ok, ov) = kv[m], hist[r]
            assert len(k) == len(ok) + 1 and torch.equal(k[:-1], ok) and torch.equal(v[:-1], ov), (t, m)
            assert torch.equal(v[-1], v_new[m].cpu())
        hist = kv
        logp = torch.log_softmax(out.float() @ wo.T, 1)
        mt.mt_beam_topk(dec.model, B, K, score, logp, score, tok, bp, row, ws)
    assert forked and cache.check() == 0
