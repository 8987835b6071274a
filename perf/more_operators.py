"""Performance cases of the attention layer's operators for serving: heads' norms and rotation with the
store into a paged cache, attention over that cache, cross attention to an encoder's states, and the page
tables that follow a beam.

Each kind is one call of the binding (mtstep) on buffers that a program holds:

  append   queries and keys of new tokens normalised per head and rotated by position, keys and values stored
           into their pages (mt_attn_append)
  paged    attention of the new tokens (a prompt, a piece of one, one token of each hypothesis) over the cache
           (mt_attn_paged)
  cross    attention of hypotheses or of whole targets to encoder states under a mask (mt_attn_cross)
  advance  the page tables of the next step: forked along the beam, shared pages that are written next copied, room
           for the new tokens (mt_pages_advance)
  pack     the pages in use copied to the front of another cache (mt_pages_pack)

`own` chooses between these calls and the plain form of the same mathematics in torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
IO = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---- cases --------------------------------------------------------------------------------------

def _append(dt, B, S, Hq, Hk, Dh, page, norm, rot, pairs, past, ragged):
    return dict(kind="append", dt=dt, B=B, S=S, Hq=Hq, Hk=Hk, Dh=Dh, page=page, norm=norm, rot=rot, pairs=pairs,
                past=past, ragged=ragged)


def _paged(dt, B, S, Hq, Hk, Dh, page, window, past, K, ragged):
    return dict(kind="paged", dt=dt, B=B, S=S, Hq=Hq, Hk=Hk, Dh=Dh, page=page, window=window, past=past, K=K,
                ragged=ragged)


def _cross(dt, B, T, S, Hq, Hk, Dh, ragged):
    return dict(kind="cross", dt=dt, B=B, T=T, S=S, Hq=Hq, Hk=Hk, Dh=Dh, ragged=ragged)


def _advance(dt, B, K, layers, Hk, Dh, page, past, ragged):
    return dict(kind="advance", dt=dt, B=B, K=K, layers=layers, Hk=Hk, Dh=Dh, page=page, past=past, ragged=ragged)


def _pack(dt, B, layers, Hk, Dh, page, past, ragged):
    return dict(kind="pack", dt=dt, B=B, K=1, layers=layers, Hk=Hk, Dh=Dh, page=page, past=past, ragged=ragged)


def listed():
    return [
        # one token of each of 64 sentences' 12 hypotheses, as the benchmark's decoder step (8 heads of 64: 512 features)
        dict(_append("f32", 768, 1, 8, 8, 64, 16, False, 64, False, 79, True), name="append_beams_f32"),
        # prompts of long documents, queries that share key heads, normalised, in pieces
        dict(_append("bf16", 8, 4096, 32, 8, 128, 16, True, 128, False, 4096, False), name="append_prompts_bf16"),
        # odd sizes: short pieces of prompts with a window, heads that fill no tile
        dict(_paged("f32", 5, 61, 6, 3, 40, 8, 50, 272, 1, True), name="paged_odd_f32"),
        # one token of each of 64 sentences' 12 hypotheses, which share their older pages
        dict(_paged("bf16", 768, 1, 8, 8, 64, 16, 0, 511, 12, True), name="paged_beams_bf16"),
        # one token of each of 16 long documents
        dict(_paged("bf16", 16, 1, 32, 8, 128, 64, 0, 32767, 1, False), name="paged_long_bf16"),
        # a piece of 2048 positions of each of two long documents
        dict(_paged("bf16", 2, 2048, 32, 8, 128, 16, 0, 6144, 1, False), name="paged_chunk_bf16"),
        # 12 hypotheses of each of 64 sentences over source sentences of the benchmark's lengths
        dict(_cross("f32", 64, 12, 80, 8, 8, 64, True), name="cross_beams_f32"),
        # whole targets scored against whole source documents
        dict(_cross("bf16", 8, 2048, 2048, 16, 16, 64, True), name="cross_documents_bf16"),
        # a step of a beam of 5 over one sentence: latency
        dict(_advance("bf16", 1, 5, 6, 8, 64, 16, 37, False), name="advance_one_bf16"),
        # a step of 64 sentences with 12 hypotheses each through six layers' caches
        dict(_advance("bf16", 64, 12, 6, 8, 64, 16, 80, True), name="advance_beams_bf16"),
        # a few odd sentences into a smaller cache
        dict(_pack("f32", 7, 3, 3, 40, 8, 150, True), name="pack_odd_f32"),
        # what is left of a batch of long documents into a new cache
        dict(_pack("bf16", 16, 4, 8, 128, 64, 4096, True), name="pack_long_bf16"),
    ]


def draw(rng):
    def logu(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    yes = lambda p=0.5: rng.random() < p
    kind = rng.choice(["append", "paged", "paged", "paged", "cross", "cross", "advance", "pack"])
    dt = rng.choice(["f32", "bf16", "bf16"])
    Hk = rng.choice([1, 2, 3, 4, 8, 8, 16])
    Hq = Hk * rng.choice([1, 1, 2, 3, 4, 8])
    Dh = rng.choice([64, 64, 128, 128, 8 * rng.randint(1, 32)])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    flops = 2e10 if dt == "f32" else 1.2e11
    if kind == "append":
        S = logu(1, 4096)
        B = logu(1, max(1, min(768, 2 ** 27 // (S * (Hq + 2 * Hk) * Dh))))
        rot = rng.choice([0, Dh, Dh, Dh, 2 * rng.randint(1, Dh // 2)])
        return _append(dt, B, S, Hq, Hk, Dh, page, yes(), rot, yes(0.3), logu(1, 100000), yes())
    if kind == "paged":
        S = 1 if yes(0.4) else logu(1, 2048)
        past = logu(1, 32768)
        keys = past + S
        while 4.0 * Dh * Hq * S * keys > flops or Hk * Dh * keys > 2 ** 28 or 4.0 * Hq * S * keys > 2 ** 31:
            S, past = max(1, S // 2), max(1, past // 2)
            keys = past + S
        most = min(768, flops / (4.0 * Dh * Hq * S * keys), 2 ** 28 / (Hk * Dh * keys), 2 ** 27 / (Hq * Dh * S))
        K = rng.choice([1, 4, 5, 12]) if S == 1 else 1
        B = K * logu(1, max(1, int(most) // K))
        return _paged(dt, B, S, Hq, Hk, Dh, page, logu(1, 4096) if yes(0.3) else 0, past, K, yes())
    if kind == "cross":
        T = rng.choice([1, 4, 5, 12, logu(1, 2048), logu(1, 2048)])
        S = logu(1, 4096)
        while 4.0 * Dh * Hq * T * S > flops:
            T, S = max(1, T // 2), max(1, S // 2)
        most = min(256, flops / (4.0 * Dh * Hq * T * S), 2 ** 27 / (Hk * Dh * S), 2 ** 27 / (Hq * Dh * T))
        return _cross(dt, logu(1, max(1, int(most))), T, S, Hq, Hk, Dh, yes(0.7))
    layers = rng.randint(1, 6)
    past = logu(1, 4096)
    per = layers * Hk * Dh * (past + 2 * page)
    if kind == "advance":
        K = rng.choice([1, 4, 5, 8, 12, 16])
        B = logu(1, max(1, min(64, 2 ** 28 // (per * K))))
        while per * K > 2 ** 28:
            layers, past = 1, max(1, past // 2)
            per = layers * Hk * Dh * (past + 2 * page)
        return _advance(dt, B, K, layers, Hk, Dh, page, past, yes())
    return _pack(dt, logu(1, max(1, min(64, 2 ** 28 // per))), layers, Hk, Dh, page, past, yes())


# ---- inputs -------------------------------------------------------------------------------------

def _sizes(n, most, ragged, order):
    """n lengths: all `most`, or quantiles of a lognormal (sigma 0.5, mean about a third of `most`), the longest
    one `most`, in a given order: the same work for every seed."""
    if not ragged:
        return np.full(n, most, np.int64)
    q = (np.arange(n) + 0.5) / n
    z = torch.special.ndtri(torch.from_numpy(q)).numpy()
    v = np.clip(np.rint(np.exp(math.log(max(1.0, most / 3)) - 0.125 + 0.5 * z)), 1, most).astype(np.int64)
    v[-1] = most
    return v[order]


def _lengths(c, seed):
    """(positions before the call, new positions) of each sequence.  The hypotheses of a sentence are equally long;
    a piece's new positions are longer where those before it are."""
    B, K = c["B"], c.get("K", 1)
    n = B // K if c["kind"] == "paged" else B
    order = np.random.default_rng(seed).permutation(n)
    past = _sizes(n, c["past"], c["ragged"], order)
    S = c.get("S", 1)
    new = _sizes(n, S, c["ragged"] and S > 1, order)
    if c["kind"] in ("append", "paged") and S > 1 and c["ragged"] and n > 1:
        new[order.argmin()] = 0  # a sequence that takes no part
    if c["kind"] == "paged":
        past, new = past.repeat(K), new.repeat(K)
    return past, new


def _tables(lens, shared, K, page, n_blocks, rng, spare):
    """Page tables of rows in groups of K that hold their first `shared` blocks in common, pages in random order
    in a pool with some spare ones; -1 behind a row's blocks.  (table, pages of the pool)"""
    M = len(lens)
    blocks = (lens + page - 1) // page
    need = sum(int(blocks[m]) - (0 if m % K == 0 else min(int(shared[m]), int(blocks[m]))) for m in range(M))
    n_pages = need + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((M, n_blocks), -1, np.int32)
    at = 0
    for m in range(M):
        nb, sh = int(blocks[m]), 0
        if m % K:
            sh = min(int(shared[m]), nb)
            table[m, :sh] = table[m - m % K, :sh]
        table[m, sh:nb] = order[at:at + nb - sh]
        at += nb - sh
    return table, n_pages


def _far_table(lens, new, page, n_blocks, rng):
    """The same for calls that only touch the blocks of the new positions: the others hold page 0."""
    table = np.zeros((len(lens), n_blocks), np.int32)
    first = (lens - new) // page
    count = np.where(new > 0, (lens + page - 1) // page - first, 0)
    order = rng.permutation(max(1, int(count.sum()))).astype(np.int32)
    at = 0
    for m in range(len(lens)):
        table[m, first[m]:first[m] + count[m]] = order[at:at + count[m]]
        at += count[m]
    return table, len(order)


def _shared(c, lens):
    """Blocks that the hypotheses of a sentence hold in common: half of the full ones."""
    return lens // c["page"] // 2


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed + 1)
    io, kind, Hk, Dh = IO[c["dt"]], c["kind"], c["Hk"], c["Dh"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, dtype=torch.float32, device=DEV)

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)

    def cache(*lead):  # drawn in pieces: no second cache in 32 bits
        t = torch.empty(*lead, Hk, c["page"], Dh, dtype=io, device=DEV)
        flat = t.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            flat[i:i + (1 << 26)] = normal(min(1 << 26, flat.numel() - i))
        return t

    x = {}
    if kind == "cross":
        B, T, S, Hq = c["B"], c["T"], c["S"], c["Hq"]
        x["q"] = normal(B, T, Hq * Dh).to(io)
        x["kv"] = normal(B, S, 2 * Hk * Dh).to(io)  # one projection makes both
        n = _sizes(B, S, c["ragged"], np.random.default_rng(seed).permutation(B))
        x["mask"] = (torch.arange(S, device=DEV)[None, :] < torch.from_numpy(n).to(DEV)[:, None]).float()
        return x
    page = c["page"]
    past, new = _lengths(c, seed)
    if kind in ("append", "paged"):
        B, S, Hq = c["B"], c["S"], c["Hq"]
        lens = past + new
        n_blocks = -(-(c["past"] + S) // page)
        if kind == "append":
            table, n_pages = _far_table(lens, new, page, n_blocks, rng)
            x["qkv"] = (normal(B, S, (Hq + 2 * Hk) * Dh) * 1.5).to(io)  # one projection makes all three
            x["gq"], x["gk"] = (1 + 0.1 * normal(Dh) for _ in range(2))
        else:
            table, n_pages = _tables(lens, _shared(c, lens), c["K"], page, n_blocks, rng, 16)
            x["q"] = (normal(B, S, Hq * Dh) * 1.5).to(io)
        x["lens"], x["new"], x["table"] = ints(lens), ints(new), ints(table)
        x["k"], x["v"] = cache(n_pages), cache(n_pages)
        return x
    layers = c["layers"]
    if kind == "pack":
        n_blocks = -(-c["past"] // page)
        table, n_pages = _tables(past, past, 1, page, n_blocks, rng, int(sum(-(-past // page))))  # half of it is free
        x["lens"], x["table"] = ints(past), ints(table)
        x["k"], x["v"] = cache(layers, n_pages), cache(layers, n_pages)
        return x
    B, K = c["B"], c["K"]
    n_blocks = -(-c["past"] // page) + 1
    lens = past.repeat(K)
    table, n_pages = _tables(lens, _shared(c, lens), K, page, n_blocks, rng, 2 * B * K)
    x["lens"], x["table"] = ints(lens), ints(table)
    x["row"] = ints(np.concatenate([b * K + rng.permutation(K)[_parents(K)] for b in range(B)]))
    x["add"] = ints(np.ones(B * K))
    x["k"], x["v"] = cache(layers, n_pages), cache(layers, n_pages)
    return x


def _parents(K):
    """Which of its sentence's K hypotheses each of the next ones continues: the better ones several times."""
    return np.array([i * i // (2 * K) for i in range(K)])


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    st, kind, io = dict(c=c, x=x), c["kind"], IO[c["dt"]]
    if kind == "append":
        st["q"] = torch.zeros(c["B"], c["S"], c["Hq"] * c["Dh"], dtype=io, device=DEV)
    elif kind in ("paged", "cross"):
        st["y"] = torch.zeros_like(x["q"])
    elif kind == "advance":
        st["table"], st["lens"] = torch.empty_like(x["table"]), torch.empty_like(x["lens"])
        st["free"] = torch.empty(1, dtype=torch.int32, device=DEV)
    else:
        n = int((-(-x["lens"].long() // c["page"])).sum())
        st["table"], st["lens"] = torch.empty_like(x["table"]), torch.empty_like(x["lens"])
        st["used"] = torch.empty(1, dtype=torch.int32, device=DEV)
        st["k"], st["v"] = (torch.zeros(c["layers"], n, *x["k"].shape[2:], dtype=io, device=DEV) for _ in range(2))
    if not own:
        return st
    from paper_1804_00344_amd import mtstep as mt
    kw = {}
    if kind == "append":
        kw = dict(qk_norm=c["norm"], norm_eps=EPS, rot=c["rot"], rot_pairs=c["pairs"])
    if kind == "paged":
        kw = dict(window=c["window"])
    cfg = mt.make_attn_config(c.get("Hq", c["Hk"]), c["Hk"], c["Dh"], page=c.get("page", 16), dtype=c["dt"], **kw)
    st["layer"] = mt.mt_attn_load(cfg, {k: x[k] for k in ("gq", "gk") if k in x})
    n = 0
    if kind == "paged":
        n = mt.mt_attn_workspace_bytes(st["layer"], c["B"], c["S"], x["table"].shape[1] * c["page"])
    elif kind == "cross":
        n = mt.mt_attn_workspace_bytes(st["layer"], c["B"], c["T"], c["S"])
    elif kind != "append":
        n = mt.mt_pages_workspace_bytes(st["layer"], len(x["lens"]), x["k"].shape[1])
    if n:
        st["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return st


# ---- one pass -----------------------------------------------------------------------------------

def _split(c, qkv):
    a, b = c["Hq"] * c["Dh"], (c["Hq"] + c["Hk"]) * c["Dh"]
    return qkv[..., :a], qkv[..., a:b], qkv[..., b:]


def _run_own(st):
    from paper_1804_00344_amd import mtstep as mt
    c, x, kind = st["c"], st["x"], st["c"]["kind"]
    if kind == "append":
        q, k, v = _split(c, x["qkv"])
        mt.mt_attn_append(st["layer"], q, k, v, st["q"], x["lens"], x["table"], x["k"], x["v"], n_new=x["new"])
        return dict(q=st["q"], k=x["k"], v=x["v"])
    if kind == "paged":
        mt.mt_attn_paged(st["layer"], x["q"], x["lens"], x["table"], x["k"], x["v"], st["y"], n_new=x["new"], ws=st["ws"])
        return st["y"]
    if kind == "cross":
        w = c["Hk"] * c["Dh"]
        mt.mt_attn_cross(st["layer"], x["q"], x["kv"][..., :w], x["kv"][..., w:], st["y"], mask=x["mask"], ws=st["ws"])
        return st["y"]
    if kind == "advance":
        mt.mt_pages_advance(st["layer"], x["row"], x["add"], x["table"], x["lens"], st["table"], st["lens"], x["k"], x["v"],
                            free_out=st["free"], ws=st["ws"])
        return dict(table=st["table"], lens=st["lens"], free=st["free"], k=x["k"], v=x["v"])
    mt.mt_pages_pack(st["layer"], x["table"], x["lens"], x["k"], x["v"], st["table"], st["lens"], st["k"], st["v"],
                     st["used"], ws=st["ws"])
    return dict(table=st["table"], lens=st["lens"], used=st["used"], k=st["k"], v=st["v"])


def _softmax_rows(s, seen):
    """Weights over the last dimension where `seen`; zeros where nothing is."""
    s = torch.where(seen, s, float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), 0.0, m))
    return p / torch.clamp(p.sum(-1, keepdim=True), min=1e-38)


def _attend(c, q, k, v, seen):
    """q [n, T, Hq, Dh], k, v [n, L, Hk, Dh], seen [n, T, L]: [n, T, Hq * Dh], in 32 bits."""
    n, T, Hq, Dh = q.shape
    L, Hk = k.shape[1], c["Hk"]
    G = Hq // Hk
    qh = q.float().reshape(n, T, Hk, G, Dh).permute(0, 2, 3, 1, 4).reshape(n, Hk, G * T, Dh) / math.sqrt(Dh)
    s = qh @ k.float().permute(0, 2, 3, 1).contiguous()
    p = _softmax_rows(s.reshape(n, Hk, G, T, L), seen[:, None, None])
    y = p.reshape(n, Hk, G * T, L) @ v.float().permute(0, 2, 1, 3).contiguous()
    return y.reshape(n, Hk, G, T, Dh).permute(0, 3, 1, 2, 4).reshape(n, T, Hq * Dh)


def _pairs(c):
    """Features that turn together: (first, second) of each pair."""
    i = torch.arange(c["rot"] // 2, device=DEV)
    return (2 * i, 2 * i + 1) if c["pairs"] else (i, i + c["rot"] // 2)


def _plain_append(st):
    c, x, page = st["c"], st["x"], st["c"]["page"]
    B, S, Hq, Hk, Dh = (c[n] for n in ("B", "S", "Hq", "Hk", "Dh"))
    lens, new = x["lens"].long(), x["new"].long()
    i = torch.arange(S, device=DEV)
    pos = (lens - new)[:, None] + i
    live = i[None, :] < new[:, None]
    q, k, v = (t.reshape(B, S, -1, Dh) for t in _split(c, x["qkv"]))

    def turn(t, gain):
        t = t.float()
        if c["norm"]:
            t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS) * gain
        if c["rot"]:
            f = torch.exp(torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV) * (-2.0 * math.log(10000.0) / c["rot"]))
            a = pos.double()[:, :, None, None] * f
            co, si = torch.cos(a).float(), torch.sin(a).float()
            lo, hi = _pairs(c)
            u, w = t[..., lo], t[..., hi]
            t = t.clone()
            t[..., lo], t[..., hi] = u * co - w * si, w * co + u * si
        return t.to(IO[c["dt"]])

    st["q"].copy_(torch.where(live[:, :, None], turn(q, x["gq"]).reshape(B, S, Hq * Dh), st["q"]))
    at = torch.where(live, pos, 0)
    pg = x["table"].gather(1, at // page).long()
    keep = live.reshape(-1)
    pg, off = pg.reshape(-1)[keep], (at % page).reshape(-1)[keep]
    x["k"][pg, :, off] = turn(k, x["gk"]).reshape(B * S, Hk, Dh)[keep]
    x["v"][pg, :, off] = v.reshape(B * S, Hk, Dh)[keep]
    return dict(q=st["q"], k=x["k"], v=x["v"])


def _plain_paged(st):
    c, x, page = st["c"], st["x"], st["c"]["page"]
    B, S, Hq, Hk, Dh = (c[n] for n in ("B", "S", "Hq", "Hk", "Dh"))
    L = x["table"].shape[1] * page
    per = max(1, min(B, int(2 ** 30 // (L * Hk * Dh + L * S * Hq))))  # sequences at a time
    j, i = torch.arange(L, device=DEV), torch.arange(S, device=DEV)
    for b in range(0, B, per):
        sl = slice(b, b + per)
        pg = x["table"][sl].long().clamp(min=0)
        k, v = (t[pg].permute(0, 1, 3, 2, 4).reshape(-1, L, Hk, Dh) for t in (x["k"], x["v"]))
        lens, new = x["lens"][sl].long(), x["new"][sl].long()
        pos = ((lens - new)[:, None] + i)[:, :, None]
        live = (i[None, :] < new[:, None])[:, :, None]
        seen = (j <= pos) & live
        if c["window"]:
            seen &= j > pos - c["window"]
        y = _attend(c, x["q"][sl].reshape(-1, S, Hq, Dh), k, v, seen)
        st["y"][sl] = y.to(st["y"].dtype)
    return st["y"]


def _plain_refs(table, blocks, n_pages):
    """References of each page from the rows' blocks."""
    n_blocks = table.shape[1]
    valid = torch.arange(n_blocks, device=DEV)[None, :] < blocks[:, None]
    one = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV)
    one.index_add_(0, torch.where(valid, table.long(), n_pages).reshape(-1), torch.ones(table.numel(), dtype=torch.int64, device=DEV))
    return one[:n_pages], valid


def _plain_advance(st):
    c, x, page = st["c"], st["x"], st["c"]["page"]
    n_pages, n_blocks = x["k"].shape[1], x["table"].shape[1]
    row, add = x["row"].long(), x["add"].long()
    M = len(row)
    L = x["lens"].long()[row]
    blocks = -(-L // page)
    table = x["table"][row]
    refs, valid = _plain_refs(table, blocks, n_pages)
    table = torch.where(valid, table, -1)
    m = torch.arange(M, device=DEV)
    last = table.gather(1, (blocks - 1).clamp(min=0)[:, None])[:, 0].long()
    grows = (add > 0) & (L % page != 0)
    at = torch.where(grows, last, n_pages)  # the partial page that a row goes on writing
    count = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV).index_add_(0, at, grows.long())
    final = torch.full((n_pages + 1,), -1, dtype=torch.int64, device=DEV).scatter_reduce(0, at, m, "amax")
    refs1 = torch.cat([refs, refs.new_zeros(1)])
    keeps = (final[at] == m) & (count[at] == refs1[at])
    copy = grows & (refs1[at] > 1) & ~keeps
    full = -(-(L + add) // page)
    need = full - blocks + copy
    first = torch.cumsum(need, 0) - need
    order = torch.argsort((refs > 0).long(), stable=True)  # the free pages first, ascending
    col = torch.arange(n_blocks, device=DEV)[None, :]
    fresh = (col >= blocks[:, None]) & (col < full[:, None])
    fresh |= copy[:, None] & (col == blocks[:, None] - 1)
    take = first[:, None] + col - (blocks - copy.long())[:, None]
    table = torch.where(fresh, order[take.clamp(0, n_pages - 1)].to(torch.int32), table)
    to = table.gather(1, (blocks - 1).clamp(min=0)[:, None])[:, 0].long()
    src, dst, n = last[copy], to[copy], (L % page)[copy]
    write = (torch.arange(page, device=DEV)[None, :] < n[:, None])[None, :, None, :, None]
    for t in (x["k"], x["v"]):
        t[:, dst] = torch.where(write, t[:, src], t[:, dst])
    st["table"].copy_(table)
    st["lens"].copy_(L + add)
    st["free"].copy_((refs == 0).sum() - need.sum())
    return dict(table=st["table"], lens=st["lens"], free=st["free"], k=x["k"], v=x["v"])


def _plain_pack(st):
    c, x = st["c"], st["x"]
    lens = x["lens"].long()
    refs, valid = _plain_refs(x["table"], -(-lens // c["page"]), x["k"].shape[1])
    live = refs > 0
    rank = torch.cumsum(live, 0) - 1
    st["table"].copy_(torch.where(valid, rank[x["table"].long().clamp(min=0)], -1))
    st["lens"].copy_(x["lens"])
    n = live.sum()
    st["used"].copy_(n)
    src = torch.argsort((~live).long(), stable=True)[:st["k"].shape[1]]  # the new cache is as large as they are
    st["k"].copy_(x["k"][:, src])
    st["v"].copy_(x["v"][:, src])
    return dict(table=st["table"], lens=st["lens"], used=st["used"], k=st["k"], v=st["v"])


def run(st):
    if own:
        return _run_own(st)
    c, x, kind = st["c"], st["x"], st["c"]["kind"]
    if kind == "append":
        return _plain_append(st)
    if kind == "paged":
        return _plain_paged(st)
    if kind == "advance":
        return _plain_advance(st)
    if kind == "pack":
        return _plain_pack(st)
    B, T, S, Hq, Hk, Dh = (c[n] for n in ("B", "T", "S", "Hq", "Hk", "Dh"))
    w = Hk * Dh
    per = max(1, min(B, int(2 ** 30 // (S * T * Hq))))
    for b in range(0, B, per):
        sl = slice(b, b + per)
        kv = x["kv"][sl]
        y = _attend(c, x["q"][sl].reshape(-1, T, Hq, Dh), kv[..., :w].reshape(-1, S, Hk, Dh), kv[..., w:].reshape(-1, S, Hk, Dh),
                    (x["mask"][sl] != 0)[:, None, :].expand(-1, T, -1))
        st["y"][sl] = y.to(st["y"].dtype)
    return st["y"]


# ---- the work of a pass -------------------------------------------------------------------------

def _seen_pairs(past, new, window):
    """Visible (query, key) pairs, and keys that some query sees, of one sequence."""
    p = np.arange(past, past + new, dtype=np.float64)
    n = np.minimum(p + 1, window) if window else p + 1
    first = max(0, past - window + 1) if window else 0
    return float(n.sum()), float(past + new - first) if new else 0.0


def work(case):
    """Each input read once (the positions that are seen, a shared page once), each output written once."""
    c, kind = case, case["kind"]
    e, Hk, Dh = (4 if c["dt"] == "f32" else 2), c["Hk"], c["Dh"]
    if kind == "cross":
        n = _sizes(c["B"], c["S"], c["ragged"], np.arange(c["B"]))
        return {"flops": 4.0 * Dh * c["Hq"] * c["T"] * float(n.sum()),
                "bytes": e * Dh * (2.0 * c["Hq"] * c["B"] * c["T"] + 2.0 * Hk * float(n.sum())) + 4.0 * c["B"] * c["S"]}
    past, new = _lengths(c, 0)
    if kind == "append":
        toks = float(new.sum())
        turned = (c["Hq"] + Hk) * toks
        return {"bytes": e * Dh * toks * (2.0 * c["Hq"] + 4.0 * Hk), "flops": turned * (4.0 * Dh * c["norm"] + 3.0 * c["rot"])}
    if kind == "paged":
        K, page = c["K"], c["page"]
        seen = [_seen_pairs(int(p), int(n), c["window"]) for p, n in zip(past, new)]
        lens = past + new
        again = sum(min(s[1], float(_shared(c, lens)[m] * page)) for m, s in enumerate(seen) if m % K and not c["window"])
        keys = sum(s[1] for s in seen) - again
        return {"flops": 4.0 * Dh * c["Hq"] * sum(s[0] for s in seen),
                "bytes": e * Dh * (2.0 * c["Hq"] * float(new.sum()) + 2.0 * Hk * keys)}
    page, layers = c["page"], c["layers"]
    blocks = float((-(-past // page)).sum())
    if kind == "pack":
        return {"bytes": 4.0 * e * layers * Hk * Dh * page * blocks + 8.0 * blocks, "flops": blocks}
    K = c["K"]
    again = K - len(set(_parents(K).tolist()))  # hypotheses that continue the same one write their own copy
    return {"bytes": 4.0 * e * layers * Hk * Dh * again * float((past % page).sum()) + 8.0 * K * blocks, "flops": K * blocks}


# ---- the same in 64 bits ------------------------------------------------------------------------

def _exact_rows(q, k, v):
    """One key head: q [R, Dh] with the keys k, v [L, Dh] that all of its rows see: softmax as the exponential of
    differences from the logarithm of the sum."""
    s = torch.mm(q, k.t()) / math.sqrt(q.shape[1])
    return torch.mm(torch.exp(s - torch.logsumexp(s, 1, keepdim=True)), v)


def _exact_paged(c, x):
    page, Hq, Hk, Dh, S = c["page"], c["Hq"], c["Hk"], c["Dh"], c["S"]
    G, table = Hq // Hk, x["table"].cpu().numpy()
    y = torch.zeros(c["B"], S, Hk, G, Dh, dtype=torch.float64, device=DEV)
    for b, (n, new) in enumerate(zip(x["lens"].tolist(), x["new"].tolist())):
        if not new:
            continue
        at = torch.from_numpy(table[b, :-(-n // page)].astype(np.int64)).to(DEV)
        for h in range(Hk):
            k, v = (t[at, h].reshape(-1, Dh)[:n].double() for t in (x["k"], x["v"]))
            q = x["q"][b, :new].reshape(new, Hk, G, Dh)[:, h].double()
            if new == 1:
                lo = max(0, n - c["window"]) if c["window"] else 0
                y[b, 0, h] = _exact_rows(q[0], k[lo:], v[lo:])
                continue
            pos = torch.arange(n - new, n, device=DEV)[:, None]
            key = torch.arange(n, device=DEV)[None, :]
            hide = key > pos
            if c["window"]:
                hide |= key <= pos - c["window"]
            for g in range(G):
                s = torch.mm(q[:, g].contiguous(), k.t()) / math.sqrt(Dh)
                s.masked_fill_(hide, float("-inf"))
                y[b, :new, h, g] = torch.mm(torch.exp(s - torch.logsumexp(s, 1, keepdim=True)), v)
    return y.reshape(c["B"], S, Hq * Dh)


def _exact_append(c, x):
    page, Hq, Hk, Dh = c["page"], c["Hq"], c["Hk"], c["Dh"]
    out = dict(q=torch.zeros(c["B"], c["S"], Hq * Dh, dtype=torch.float64, device=DEV), k=x["k"].double(), v=x["v"].double())
    table = x["table"].cpu().numpy()
    f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / max(1, c["rot"]))
    for b, (n, new) in enumerate(zip(x["lens"].tolist(), x["new"].tolist())):
        if not new:
            continue
        pos = np.arange(n - new, n)
        angle = torch.from_numpy(pos).to(DEV).double()[:, None] * f
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        rows = x["qkv"][b, :new].double().reshape(new, Hq + 2 * Hk, Dh)
        qk = rows[:, :Hq + Hk].clone()
        if c["norm"]:
            qk = qk / torch.sqrt(qk.square().sum(-1, keepdim=True) / Dh + EPS)
            qk[:, :Hq] *= x["gq"].double()
            qk[:, Hq:] *= x["gk"].double()
        if c["rot"]:  # pairs as complex numbers
            r = qk[..., :c["rot"]]
            r = r.reshape(new, Hq + Hk, -1, 2) if c["pairs"] else r.reshape(new, Hq + Hk, 2, -1).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(r.contiguous()) * turn)
            qk[..., :c["rot"]] = (z if c["pairs"] else z.transpose(2, 3)).reshape(new, Hq + Hk, -1)
        out["q"][b, :new] = qk[:, :Hq].reshape(new, -1)
        pg, off = (torch.from_numpy(a.astype(np.int64)).to(DEV) for a in (table[b, pos // page], pos % page))
        out["k"][pg, :, off] = qk[:, Hq:]
        out["v"][pg, :, off] = rows[:, Hq + Hk:]
    return out


def _exact_advance(c, x):
    """Row by row, as the definition says it."""
    page, n_pages = c["page"], x["k"].shape[1]
    told, lens = x["table"].tolist(), x["lens"].tolist()
    row, add = x["row"].tolist(), x["add"].tolist()
    rows = [told[r][:-(-lens[r] // page)] for r in row]
    refs = np.zeros(n_pages, np.int64)
    for r in rows:
        for p in r:
            refs[p] += 1
    free = iter([p for p in range(n_pages) if refs[p] == 0])
    taken, copies = 0, []
    table = np.full((len(row), len(told[0])), -1, np.int32)
    for m, r in enumerate(rows):
        n = lens[row[m]]
        if add[m] > 0 and n % page and refs[r[-1]] > 1:  # others hold the page that is written next
            p = next(free)
            taken += 1
            refs[r[-1]] -= 1
            copies.append((r[-1], p, n % page))
            r[-1] = p
        while len(r) * page < n + add[m]:
            r.append(next(free))
            taken += 1
        table[m, :len(r)] = r
    left = sum(1 for _ in free)
    k, v = x["k"].double(), x["v"].double()
    for t in (k, v):
        for s, d, n in copies:
            t[:, d, :, :n] = t[:, s, :, :n]
    ints = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(DEV)
    return dict(table=ints(table), lens=ints([lens[r] + a for r, a in zip(row, add)]), free=ints([left]), k=k, v=v)


def _exact_pack(c, x):
    told = x["table"].cpu().numpy()
    used = sorted({int(p) for r in told for p in r if p >= 0})
    new = np.full(x["k"].shape[1] + 1, -1, np.int32)  # -1 stays -1
    new[used] = np.arange(len(used))
    at = torch.tensor(used, device=DEV)
    ints = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(DEV)
    return dict(table=ints(new[told]), lens=x["lens"].clone(), used=ints([len(used)]), k=x["k"][:, at].double(), v=x["v"][:, at].double())


def exact(case, seed):
    """What run returns, in 64 bits: attention one key head of one sequence at a time, rotations as products of
    complex numbers, page tables row by row on the host."""
    c, x = case, _inputs(case, seed)
    if c["kind"] != "cross":
        return dict(append=_exact_append, paged=_exact_paged, advance=_exact_advance, pack=_exact_pack)[c["kind"]](c, x)
    B, T, Hq, Hk, Dh = (c[n] for n in ("B", "T", "Hq", "Hk", "Dh"))
    G, w = Hq // Hk, Hk * Dh
    y = torch.zeros(B, T, Hk, G, Dh, dtype=torch.float64, device=DEV)
    for b in range(B):
        at = x["mask"][b].nonzero()[:, 0]
        if not len(at):
            continue
        kv = x["kv"][b, at].double()
        for h in range(Hk):
            q = x["q"][b].reshape(T, Hk, G, Dh)[:, h].double().reshape(T * G, Dh)
            r = _exact_rows(q, kv[:, h * Dh:(h + 1) * Dh].contiguous(), kv[:, w + h * Dh:w + (h + 1) * Dh].contiguous())
            y[b, :, h] = r.reshape(T, G, Dh)
    return y.reshape(B, T, Hq * Dh)
