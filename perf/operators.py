"""Performance cases of the recurrent layer's operators: the selective state space scan with its short
causal convolution, for whole prompts and for single tokens of hypotheses, and the matrix products in
8-bit integers that feed them and the output layer.

Each kind is one call of the binding (mtstep) on buffers that a program holds:

  conv       the causal convolution over a padded batch of prompts (mt_ssm_conv)
  conv_step  the same for one token of each hypothesis, states gathered along the beam (mt_ssm_conv_step)
  scan       the selective scan over a padded batch of prompts (mt_ssm_scan)
  step       the same for one token of each hypothesis (mt_ssm_step)
  i8         rows times a weight matrix, both in 8 bits with a scale per row and per column (mt_i8_product)

`own` chooses between these calls and the plain form of the same mathematics in torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------

def _conv(dt, B, S, D, W, silu, ragged, state):
    return dict(kind="conv", dt=dt, B=B, S=S, D=D, W=W, silu=silu, ragged=ragged, state=state)


def _conv_step(dt, M, D, W, K):
    return dict(kind="conv_step", dt=dt, M=M, D=D, W=W, K=K, silu=True)


def _scan(dt, B, S, D, N, G, ragged, state, gate):
    return dict(kind="scan", dt=dt, B=B, S=S, D=D, N=N, G=G, ragged=ragged, state=state, gate=gate)


def _step(dt, M, D, N, G, K, gate):
    return dict(kind="step", dt=dt, M=M, D=D, N=N, G=G, K=K, gate=gate)


def _i8(xdt, ydt, M, K, N, bias, pad):
    return dict(kind="i8", xdt=xdt, ydt=ydt, M=M, K=K, N=N, bias=bias, pad=pad)


def listed():
    return [
        # a few short pieces of longer inputs, odd channel count: the convolution continues from its state
        dict(_conv("f32", 3, 61, 333, 3, True, True, True), name="conv_odd_f32"),
        # long documents, all of one length, in the layer's ordinary width
        dict(_conv("bf16", 4, 8192, 2048, 4, True, False, False), name="conv_long_bf16"),
        # interactive decoding: one hypothesis
        dict(_conv_step("bf16", 1, 2048, 4, 1), name="conv_step_one_bf16"),
        # 64 sentences with 12 hypotheses each, as the benchmark's decoder step
        dict(_conv_step("bf16", 768, 2048, 4, 12), name="conv_step_beams_bf16"),
        # odd sizes: three groups of state inputs, 24 states, a piece of a longer input each
        dict(_scan("f32", 7, 97, 330, 24, 3, True, True, True), name="scan_odd_f32"),
        # a batch of 64 source sentences of the benchmark's lengths
        dict(_scan("bf16", 64, 80, 2048, 16, 1, True, False, True), name="scan_batch_bf16"),
        # one long document: few rows, a long axis
        dict(_scan("bf16", 1, 8192, 2048, 16, 1, False, False, True), name="scan_long_bf16"),
        # interactive decoding: one hypothesis
        dict(_step("bf16", 1, 2048, 16, 1, 1, True), name="step_one_bf16"),
        # 64 sentences with 12 hypotheses each
        dict(_step("bf16", 768, 2048, 16, 1, 12, True), name="step_beams_bf16"),
        # the output layer for one hypothesis: all weight traffic
        dict(_i8("f32", "f32", 1, 512, 50000, True, 0), name="i8_vocab_one_f32"),
        # the output layer of the benchmark's decoder step
        dict(_i8("f32", "f32", 768, 512, 50000, True, 0), name="i8_vocab_beams_f32"),
        # a projection over the positions of long documents
        dict(_i8("bf16", "bf16", 8192, 4096, 8192, False, 0), name="i8_prompts_bf16"),
    ]


def draw(rng):
    def logu(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def even(n, to=16):  # model widths are mostly multiples of 16
        return max(to, n // to * to) if rng.random() < 0.7 else n

    kind = rng.choice(["conv", "conv_step", "scan", "scan", "step", "i8", "i8"])
    dt = rng.choice(["f32", "bf16", "bf16"])
    yes = lambda p=0.5: rng.random() < p
    if kind == "conv":
        D, S = even(logu(1, 4096)), logu(1, 8192)
        B = logu(1, max(1, min(64, 2 ** 25 // (D * S))))
        return _conv(dt, B, S, D, rng.randint(1, 8), yes(0.8), yes(), yes())
    if kind == "scan":
        D, N = even(logu(1, 4096)), rng.choice([1, 4, 8, 16, 16, 16, 24, 32, 64, 100, 128])
        S = logu(1, 8192)
        cells = 2 ** 27 if N >= 16 else 2 ** 24 * N // 2
        while D * N * S > cells:
            S = max(1, S // 2)
        B = logu(1, max(1, min(64, cells // (D * N * S))))
        G = rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if D % g == 0])
        return _scan(dt, B, S, D, N, G, yes(), yes(), yes(0.7))
    K = rng.choice([1, 4, 5, 8, 12, 16])
    if kind == "conv_step":
        return _conv_step(dt, K * logu(1, 1024 // K), even(logu(1, 2048)), rng.randint(2, 8), K)
    if kind == "step":
        D, N = even(logu(1, 2048)), rng.choice([1, 4, 8, 16, 16, 16, 24, 64, 128])
        M = K * logu(1, max(1, min(1024, 2 ** 24 // (D * N)) // K))
        G = rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if D % g == 0])
        return _step(dt, M, D, N, G, K, yes(0.7))
    Kd, N = even(logu(16, 4096)), even(logu(16, 50000))
    M = logu(1, max(1, min(8192, 2 ** 29 // max(Kd, N), 2 ** 37 // (Kd * N))))
    return _i8(rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]), M, Kd, N, yes(), rng.choice([0, 0, 0, 8, 5]))


# ---- inputs -------------------------------------------------------------------------------------

def _lens(c, seed):
    """Lengths of the case's prompts: all S, or quantiles of a lognormal mix (sigma 0.5, mean about a
    third of S) in an order drawn from the seed, the longest one S: the same work for every seed."""
    B, S = c["B"], c["S"]
    if not c["ragged"]:
        return np.full(B, S, np.int64)
    q = (np.arange(B) + 0.5) / B
    z = torch.special.ndtri(torch.from_numpy(q)).numpy()
    n = np.clip(np.rint(np.exp(math.log(max(1.0, S / 3)) - 0.125 + 0.5 * z)), 1, S).astype(np.int64)
    n[-1] = S
    return n[np.random.default_rng(seed).permutation(B)]


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    f32 = dict(dtype=torch.float32, device=DEV)

    def normal(*shape):
        return torch.randn(*shape, generator=g, **f32)

    x = {}
    if c["kind"] == "i8":
        M, K, N = c["M"], c["K"], c["N"]
        lim = math.sqrt(6.0 / (K + N))
        x["W"] = (torch.rand(K, N, generator=g, **f32) * 2 - 1) * lim
        x["bias"] = normal(N) if c["bias"] else None
        # rows of different sizes, as the states of different positions
        x["x"] = torch.zeros(M, K + c["pad"], dtype=IO[c["xdt"]], device=DEV)
        x["x"][:, :K] = normal(M, K) * torch.exp(normal(M, 1))
        return x
    io, D = IO[c["dt"]], c["D"]
    steps = c["kind"] in ("conv_step", "step")
    lead = (c["M"],) if steps else (c["B"], c["S"])
    if steps:  # each hypothesis continues one of its sentence's
        M, K = c["M"], c["K"]
        x["row"] = (torch.arange(M) // K * K).to(DEV).to(torch.int32)
        x["row"] += torch.randint(0, K, (M,), generator=g, device=DEV, dtype=torch.int32)
    else:
        x["lens"] = torch.from_numpy(_lens(c, seed)).to(torch.int32).to(DEV)
    if c["kind"].startswith("conv"):
        W = c["W"]
        # the two halves of an input projection stand side by side: the convolution takes the first
        x["xz"] = normal(*lead, 2 * D).to(io)
        x["w"], x["b"] = normal(D, W) / math.sqrt(W), 0.1 * normal(D)
        rows = c["M"] if steps else c["B"]
        x["state"] = normal(rows, W - 1, D).to(io) if steps or c["state"] else None
        return x
    N, G = c["N"], c["G"]
    x["x"] = torch.nn.functional.silu(normal(*lead, D)).to(io)
    x["dtr"] = normal(*lead, D).to(io)
    R = 16  # the product that makes B and C has other columns before them
    x["bc"] = normal(*lead, R + 2 * G * N).to(io)
    x["z"] = normal(*lead, D).to(io) if c["gate"] else None
    x["A"] = -torch.arange(1, N + 1, **f32).expand(D, N) * torch.exp(0.1 * normal(D, N))
    step = torch.exp(torch.rand(D, generator=g, **f32) * math.log(100.0) + math.log(1e-3))  # 0.001 to 0.1
    x["dt_bias"] = step + torch.log(-torch.expm1(-step))
    x["skip"] = 1 + 0.1 * normal(D)
    rows = c["M"] if steps else c["B"]
    x["state"] = normal(rows, D, N) if steps or c["state"] else None
    return x


def _quantise(w, dim):
    """q = rint(w * (127 / a)), s = a / 127 with a the largest magnitude along dim, in 32 bits."""
    a = w.float().abs().amax(dim, keepdim=True)
    live = a >= 2.0 ** -100
    r = torch.where(live, torch.full_like(a, 127.0) / torch.where(live, a, 1.0), 0.0)
    return torch.round(w.float() * r), a / torch.full_like(a, 127.0) * live


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    st = dict(c=c, x=x)
    kind = c["kind"]
    if kind == "i8":
        M, N = c["M"], c["N"]
        if not own:
            st["qw"], st["sw"] = _quantise(x["W"], 0)  # whole numbers
        else:
            from paper_1804_00344_amd import mtstep as mt
            st["mat"] = mt.mt_i8_load(x["W"], x["bias"])
            st["ws"] = torch.empty(mt.mt_i8_workspace_bytes(st["mat"], M), dtype=torch.uint8, device=DEV)
            st["y"] = torch.empty(M, N, dtype=IO[c["ydt"]], device=DEV)
        del x["W"]
        return st
    if not own:
        return st
    from paper_1804_00344_amd import mtstep as mt
    D, io = c["D"], IO[c["dt"]]
    steps = kind in ("conv_step", "step")
    lead = (c["M"],) if steps else (c["B"], c["S"])
    if kind.startswith("conv"):
        cfg = mt.make_ssm_config(D, 1, conv=c["W"], conv_silu=c["silu"], dtype=c["dt"])
        st["cell"] = mt.mt_ssm_load(cfg, dict(A=torch.full((D, 1), -1.0), conv_w=x["w"], conv_b=x["b"]))
        st["state"] = torch.empty(lead[0], c["W"] - 1, D, dtype=io, device=DEV)
    else:
        cfg = mt.make_ssm_config(D, c["N"], groups=c["G"], dtype=c["dt"])
        st["cell"] = mt.mt_ssm_load(cfg, {k: x[k] for k in ("A", "dt_bias", "skip")})
        st["state"] = torch.empty(lead[0], D, c["N"], dtype=torch.float32, device=DEV)
        if not steps:
            st["ws"] = torch.empty(mt.mt_ssm_workspace_bytes(st["cell"], c["B"], c["S"]), dtype=torch.uint8,
                                   device=DEV)
    st["y"] = torch.zeros(*lead, D, dtype=io, device=DEV)
    return st


# ---- one pass -----------------------------------------------------------------------------------

def _run_own(st):
    from paper_1804_00344_amd import mtstep as mt
    c, x, kind = st["c"], st["x"], st["c"]["kind"]
    if kind == "i8":
        mt.mt_i8_product(st["mat"], x["x"][:, :c["K"]], st["y"], st["ws"])
        return st["y"]
    y, state = st["y"], st["state"]
    if kind == "conv":
        mt.mt_ssm_conv(st["cell"], x["xz"][..., :c["D"]], y, lens=x["lens"], state_in=x["state"], state_out=state)
    elif kind == "conv_step":
        mt.mt_ssm_conv_step(st["cell"], x["xz"][..., :c["D"]], y, x["state"], state, src_row=x["row"])
    else:
        GN = c["G"] * c["N"]
        bm, cm = x["bc"][..., -2 * GN:-GN], x["bc"][..., -GN:]
        if kind == "scan":
            mt.mt_ssm_scan(st["cell"], x["x"], x["dtr"], bm, cm, y, z=x["z"], lens=x["lens"], state_in=x["state"],
                           state_out=state, ws=st["ws"])
        else:
            mt.mt_ssm_step(st["cell"], x["x"], x["dtr"], bm, cm, y, x["state"], state, z=x["z"], src_row=x["row"])
    return dict(y=y, state=state)


def _silu(v):
    return v / (1 + torch.exp(-v))


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def run(st):
    if own:
        return _run_own(st)
    c, x, kind = st["c"], st["x"], st["c"]["kind"]
    if kind == "i8":
        q, s = _quantise(x["x"][:, :c["K"]], 1)
        y = (q @ st["qw"]) * st["sw"] * s
        if c["bias"]:
            y = y + x["bias"]
        return y.to(IO[c["ydt"]])
    io, D = IO[c["dt"]], c["D"]
    if kind in ("conv", "conv_step"):
        W = c["W"]
        v = x["xz"][..., :D].float()
        if kind == "conv_step":
            v = v[:, None]
            old = x["state"][x["row"].long()].float()
        else:
            old = x["state"].float() if x["state"] is not None else v.new_zeros(v.shape[0], W - 1, D)
        S = v.shape[1]
        v = torch.cat([old, v], 1)
        y = x["b"].expand(v.shape[0], S, D).clone()
        for j in range(W):
            y += v[:, j:j + S] * x["w"][:, j]
        if c["silu"]:
            y = _silu(y)
        if kind == "conv_step":
            return dict(y=y[:, 0].to(io), state=v[:, 1:].to(io))
        n = x["lens"].long()
        y = torch.where(torch.arange(S, device=DEV)[None, :, None] < n[:, None, None], y, 0.0)
        keep = n[:, None] + torch.arange(W - 1, device=DEV)  # the last W - 1 inputs of each prompt
        return dict(y=y.to(io), state=v.gather(1, keep[:, :, None].expand(-1, -1, D)).to(io))
    N, G = c["N"], c["G"]
    xv, delta = x["x"].float(), _softplus(x["dtr"].float() + x["dt_bias"])
    lead = xv.shape[:-1]
    bm = x["bc"][..., -2 * G * N:-G * N].float().reshape(*lead, G, 1, N)
    cm = x["bc"][..., -G * N:].float().reshape(*lead, G, 1, N)
    A = x["A"].reshape(G, D // G, N)
    if kind == "step":
        h = x["state"][x["row"].long()].reshape(-1, G, D // G, N)
        dv, dx = (t.reshape(-1, G, D // G, 1) for t in (delta, delta * xv))
        h = torch.exp(dv * A) * h + dx * bm
        y = (h * cm).sum(-1).reshape(*lead, D)
        h = h.reshape(-1, D, N)
    else:
        B, S = lead
        live = (torch.arange(S, device=DEV)[None, :] < x["lens"][:, None])[:, :, None]
        delta = torch.where(live, delta, 0.0)  # a position behind the prompt keeps the state as it is
        dv, dx = (t.reshape(B, S, G, D // G, 1) for t in (delta, delta * xv))
        h = xv.new_zeros(B, G, D // G, N) if x["state"] is None else x["state"].reshape(B, G, D // G, N)
        y = torch.empty(B, S, G, D // G, device=DEV)
        for t in range(S):
            h = torch.exp(dv[:, t] * A) * h + dx[:, t] * bm[:, t]
            y[:, t] = (h * cm[:, t]).sum(-1)
        y, h = y.reshape(B, S, D), h.reshape(B, D, N)
    y = y + x["skip"] * xv
    if c["gate"]:
        y = y * _silu(x["z"].float())
    if kind == "scan":
        y = torch.where(live, y, 0.0)
    return dict(y=y.to(io), state=h)


# ---- the work of a pass -------------------------------------------------------------------------

def work(case):
    """Each input read once (the positions of the prompts only), each output written once."""
    c, kind = case, case["kind"]
    es = {"f32": 4, "bf16": 2}
    if kind == "i8":
        M, K, N = c["M"], c["K"], c["N"]
        return {"flops": 2.0 * M * K * N,
                "bytes": es[c["xdt"]] * M * K + K * N + (8.0 if c["bias"] else 4.0) * N + es[c["ydt"]] * M * N}
    e, D = es[c["dt"]], c["D"]
    rows = c["M"] if "M" in c else c["B"]
    toks = c["M"] if "M" in c else int(_lens(c, 0).sum())
    if kind.startswith("conv"):
        W = c["W"]
        old = rows if kind == "conv_step" or c["state"] else 0
        return {"flops": 2.0 * toks * D * W, "bytes": e * D * (2.0 * toks + (W - 1) * (old + rows)) + 4.0 * D * (W + 1)}
    N, G = c["N"], c["G"]
    old = rows if kind == "step" or c["state"] else 0
    return {"flops": 6.0 * toks * D * N,
            "bytes": e * toks * ((4.0 if c["gate"] else 3.0) * D + 2 * G * N) + 4.0 * D * N * (rows + old + 1) + 8.0 * D}


# ---- the same in 64 bits ------------------------------------------------------------------------

def _whole(w, dim):
    """The 8-bit whole numbers and scales of w: they are defined in 32-bit arithmetic (quotient and product
    of 32-bit numbers formed in 64 bits and rounded once are the correctly rounded ones)."""
    w = w.double()
    a = w.abs().max(dim, keepdim=True).values
    r = torch.where(a >= 2.0 ** -100, 127.0 / a, torch.zeros_like(a)).float().double()
    q = (w * r).float().double().round()
    return q, torch.where(a >= 2.0 ** -100, a / 127.0, torch.zeros_like(a)).float().double()


def exact(case, seed):
    """What run returns, in 64 bits: the convolution from its definition as a correlation, the scan as
    compositions of affine maps over doubling spans, the products of the 8-bit numbers."""
    c, x, kind = case, _inputs(case, seed), case["kind"]
    if kind == "i8":
        qx, sx = _whole(x["x"][:, :c["K"]], 1)
        qw, sw = _whole(x["W"], 0)
        y = torch.empty(c["M"], c["N"], dtype=torch.float64, device=DEV)
        for i in range(0, c["M"], 1024):
            y[i:i + 1024] = qx[i:i + 1024] @ qw * (sx[i:i + 1024] * sw)
        return y if x["bias"] is None else y + x["bias"].double()
    D = c["D"]
    if kind.startswith("conv"):
        W = c["W"]
        v = x["xz"][..., :D].double()
        if kind == "conv_step":
            seqs = torch.cat([x["state"].double()[x["row"].long()], v[:, None]], 1)
        else:
            first = torch.zeros(c["B"], W - 1, D, dtype=torch.float64, device=DEV)
            seqs = torch.cat([first if x["state"] is None else x["state"].double(), v], 1)
        y = seqs.unfold(1, W, 1).mul(x["w"].double()).sum(-1) + x["b"].double()
        if c["silu"]:
            y = y * torch.sigmoid(y)
        if kind == "conv_step":
            return dict(y=y[:, 0], state=seqs[:, 1:])
        state = torch.empty(c["B"], W - 1, D, dtype=torch.float64, device=DEV)
        for b, n in enumerate(x["lens"].tolist()):
            y[b, n:] = 0
            state[b] = seqs[b, n:n + W - 1]
        return dict(y=y, state=state)
    N, G = c["N"], c["G"]
    scan = kind == "scan"
    lift = (lambda t: t) if scan else (lambda t: t[:, None])  # a single token is a prompt of one
    xv, raw, bc = lift(x["x"]).double(), lift(x["dtr"]).double(), lift(x["bc"]).double()
    B, S = xv.shape[:2]
    n = x["lens"].tolist() if scan else [1] * B
    if not scan:
        h0 = x["state"].double()[x["row"].long()]
    else:
        h0 = torch.zeros(B, D, N, dtype=torch.float64, device=DEV) if x["state"] is None else x["state"].double()
    delta = torch.nn.functional.softplus(raw + x["dt_bias"].double(), threshold=40)
    y = torch.zeros(B, S, D, dtype=torch.float64, device=DEV)
    state = h0.clone()
    per = max(1, min(D, 2 ** 27 // (S * N)))  # channels at a time
    for b in range(B):
        L = n[b]
        if L == 0:
            continue
        for d0 in range(0, D, per):
            d1 = min(D, d0 + per)
            grp = torch.arange(d0, d1, device=DEV) // (D // G)
            bm = bc[b, :L, -2 * G * N:-G * N].reshape(L, G, N)[:, grp]
            cm = bc[b, :L, -G * N:].reshape(L, G, N)[:, grp]
            dl = delta[b, :L, d0:d1]
            mul = torch.exp(dl[:, :, None] * x["A"][d0:d1].double())
            add = (dl * xv[b, :L, d0:d1])[:, :, None] * bm
            add[0] += mul[0] * h0[b, d0:d1]
            span = 1
            while span < L:  # the map of the last 2 * span positions from those of span
                add[span:] = add[span:] + mul[span:] * add[:-span].clone()
                mul[span:] = mul[span:] * mul[:-span].clone()
                span *= 2
            y[b, :L, d0:d1] = (add * cm).sum(-1)
            state[b, d0:d1] = add[-1]
        y[b, :L] += x["skip"].double() * xv[b, :L]
        if c["gate"]:
            zz = lift(x["z"])[b, :L].double()
            y[b, :L] *= zz * torch.sigmoid(zz)
    return dict(y=y if scan else y[:, 0], state=state)
