"""Device-buffer harness around the libmtstep calls (allocation and call order only).

Holds a loaded model, one batch's device inputs (context, mask, attention keys,
start state), a workspace and ping-pong state/beam buffers, and issues
mt_precompute_ctx / mt_decoder_step / mt_beam_topk in decode order.  torch
provides device memory and the stream; all arithmetic runs in libmtstep.
"""
from __future__ import annotations

import contextlib
from typing import Dict, Optional

import numpy as np
import torch

from . import mtstep as mt


class Decoder:
    def __init__(self, E: int, H: int, A: int, V: int, weights: Dict[str, np.ndarray], *, gemm: str = "f32",
                 layer_norm: bool = False, tied_output: bool = False, k_max: int = 16, ln_eps: float = 1e-5,
                 transitions: int = 0, src_V: int = 0, dual_source: bool = False, enc_transitions: int = 0,
                 enc_layer_norm: bool = False, device: str = "cuda:0"):
        self.E, self.H, self.A, self.V, self.C = E, H, A, V, 2 * H
        self.gemm = gemm
        self.device = torch.device(device)
        self.cfg = mt.make_config(E, H, A, V, layer_norm=layer_norm, tied_output=tied_output, k_max=k_max,
                                  gemm=gemm, ln_eps=ln_eps, transitions=transitions, src_V=src_V,
                                  dual_source=dual_source, enc_transitions=enc_transitions,
                                  enc_layer_norm=enc_layer_norm)
        self.dual = bool(dual_source)
        self.S2 = 0
        with torch.cuda.device(self.device):
            self.model = mt.mt_load_weights(self.cfg, weights)
        self.io_dtype = torch.bfloat16 if gemm == "bf16" else torch.float32
        self.reuse_state = True  # the decode loop's steps reuse the previous step's bf16 state copy

    @classmethod
    def from_preset(cls, p, weights, **kw):
        return cls(p.E, p.H, p.A, p.V, weights, gemm=p.gemm, layer_norm=p.layer_norm, k_max=max(p.K, 1),
                   transitions=p.transitions, **kw)

    # ---- batch ------------------------------------------------------------------------
    def set_batch(self, ctx: np.ndarray, mask: np.ndarray, K: int):
        B, S, Cd = ctx.shape
        assert Cd == self.C and mask.shape == (B, S)
        d = self.device
        self.B, self.S, self.K, self.M = B, S, K, B * K
        self.ctx = torch.from_numpy(np.ascontiguousarray(ctx, np.float32)).to(d).to(self.io_dtype).contiguous()
        self.mask = torch.from_numpy(np.ascontiguousarray(mask, np.float32)).to(d)
        self.pctx = torch.empty((B, S, self.A), dtype=self.io_dtype, device=d)
        self.s0 = torch.empty((B, self.H), dtype=torch.float32, device=d)
        nbytes = mt.mt_workspace_bytes(self.model, B, K, S)
        assert nbytes > 0
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=d)
        M = self.M
        self.state = [torch.empty((M, self.H), dtype=torch.float32, device=d) for _ in range(2)]
        self.tok = torch.empty(M, dtype=torch.int32, device=d)
        self.row = torch.empty(M, dtype=torch.int32, device=d)
        self.bp = torch.empty(M, dtype=torch.int32, device=d)
        self.score = torch.empty(M, dtype=torch.float32, device=d)
        self.cur = 0

    def set_source(self, src_tok: np.ndarray, mask: np.ndarray, K: int, stream=None):
        """Batch from source tokens: the context comes from the model's encoder (mt_encode)."""
        B, S = src_tok.shape
        self.set_batch(np.zeros((1, 1, self.C), np.float32), np.ones((1, 1), np.float32), K)  # buffers of the right kind
        d = self.device
        self.B, self.S, self.K, self.M = B, S, K, B * K
        self.src_tok = torch.from_numpy(np.ascontiguousarray(src_tok, np.int32)).to(d)
        self.mask = torch.from_numpy(np.ascontiguousarray(mask, np.float32)).to(d)
        self.ctx = torch.empty((B, S, self.C), dtype=self.io_dtype, device=d)
        self.pctx = torch.empty((B, S, self.A), dtype=self.io_dtype, device=d)
        self.s0 = torch.empty((B, self.H), dtype=torch.float32, device=d)
        nbytes = mt.mt_workspace_bytes(self.model, B, K, S)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=d)
        self.ews = torch.empty(mt.mt_encode_workspace_bytes(self.model, B, S), dtype=torch.uint8, device=d)
        M = self.M
        self.state = [torch.empty((M, self.H), dtype=torch.float32, device=d) for _ in range(2)]
        self.tok = torch.empty(M, dtype=torch.int32, device=d)
        self.row = torch.empty(M, dtype=torch.int32, device=d)
        self.bp = torch.empty(M, dtype=torch.int32, device=d)
        self.score = torch.empty(M, dtype=torch.float32, device=d)
        self.cur = 0
        self.encode(stream=stream)

    def encode(self, stream=None):
        mt.mt_encode(self.model, self.B, self.S, self.src_tok, self.mask, self.ctx, self.ews, stream=stream)

    def set_second_source(self, ctx2: np.ndarray, mask2: np.ndarray):
        """The second source of a dual-source model (after set_batch / set_source)."""
        B, S2, Cd = ctx2.shape
        assert self.dual and B == self.B and Cd == self.C and mask2.shape == (B, S2)
        d = self.device
        self.S2 = S2
        self.ctx2 = torch.from_numpy(np.ascontiguousarray(ctx2, np.float32)).to(d).to(self.io_dtype).contiguous()
        self.mask2 = torch.from_numpy(np.ascontiguousarray(mask2, np.float32)).to(d)
        self.pctx2 = torch.empty((B, S2, self.A), dtype=self.io_dtype, device=d)
        need = mt.mt_workspace_bytes(self.model, B, self.K, S2)
        if need > self.ws.numel():
            self.ws = torch.empty(need, dtype=torch.uint8, device=d)

    def precompute(self, stream=None):
        mt.mt_precompute_ctx(self.model, self.B, self.S, self.ctx, self.mask, self.pctx, self.s0, self.ws,
                             stream=stream)
        if self.dual:
            mt.mt_precompute_keys2(self.model, self.B, self.S2, self.ctx2, self.mask2, self.pctx2, self.ws,
                                   stream=stream)

    def step(self, prev_tok, src_row, state_in, n_state_rows: int, state_out, *, logp=None, attn=None,
             taps=None, stream=None):
        if self.dual:
            mt.mt_decoder_step_dual(self.model, self.B, self.K, self.S, prev_tok, src_row, n_state_rows, state_in,
                                    self.ctx, self.pctx, self.mask, self.S2, self.ctx2, self.pctx2, self.mask2,
                                    state_out, logp_out=logp, attn_out=attn, taps=taps, ws=self.ws, stream=stream)
            return
        mt.mt_decoder_step(self.model, self.B, self.K, self.S, prev_tok, src_row, n_state_rows, state_in, self.ctx,
                           self.pctx, self.mask, state_out, logp_out=logp, attn_out=attn, taps=taps, ws=self.ws,
                           stream=stream)

    def topk(self, prev_score, logp=None, *, score_out=None, tok_out=None, bp_out=None, row_out=None,
             stream=None):
        score_out = self.score if score_out is None else score_out
        tok_out = self.tok if tok_out is None else tok_out
        bp_out = self.bp if bp_out is None else bp_out
        row_out = self.row if row_out is None else row_out
        mt.mt_beam_topk(self.model, self.B, self.K, prev_score, logp, score_out, tok_out, bp_out, row_out,
                        ws=self.ws, stream=stream)
        return score_out, tok_out, bp_out, row_out

    # ---- decode loop ------------------------------------------------------------------
    def start(self, tok0: np.ndarray, score0: np.ndarray):
        """Beam start: every row reads its sentence's start state (src_row = m // K).

        The start beam is staged on the device once per (tok0, score0) pair; later starts
        are device-to-device copies on the stream, so a new decode does not synchronise."""
        d = self.device
        tok0 = np.ascontiguousarray(tok0, np.int32)
        score0 = np.ascontiguousarray(score0, np.float32)
        key = (self.M, tok0.tobytes(), score0.tobytes())
        if getattr(self, "_start_key", None) != key:
            self._start_tok = torch.from_numpy(tok0).to(d)
            self._start_score = torch.from_numpy(score0).to(d)
            self._start_row = torch.arange(self.M, dtype=torch.int32, device=d) // self.K
            self._start_key = key
        self.tok.copy_(self._start_tok)
        self.row.copy_(self._start_row)
        self.score.copy_(self._start_score)
        self.first = True

    @contextlib.contextmanager
    def _reuse(self):
        """Within the decode loop the state a step reads is the previous step's output, which
        nothing else writes: a bf16 model's step may take the copy of it the previous step
        left in the workspace (mt_set_state_reuse), for that call only."""
        on = self.reuse_state and self.gemm == "bf16" and not self.first
        if on:
            mt.mt_set_state_reuse(self.model, True)
        try:
            yield
        finally:
            if on:
                mt.mt_set_state_reuse(self.model, False)

    def advance(self, *, logp=None, attn=None, stream=None):
        """One beam-search step: decoder step on the current beam, then top-K in place."""
        if self.first:
            state_in, nrows = self.s0, self.B
        else:
            state_in, nrows = self.state[self.cur], self.M
        out = self.state[1 - self.cur] if not self.first else self.state[self.cur]
        with self._reuse():
            self.step(self.tok, self.row, state_in, nrows, out, logp=logp, attn=attn, stream=stream)
        self.topk(self.score, None, stream=stream)
        if not self.first:
            self.cur = 1 - self.cur
        self.first = False
        return self.state[self.cur]


def translate(dec: "Decoder", tok0, score0, max_steps: int, eos: int, alpha: float, check_every: int = 4,
              stream=None):
    """Batched beam search to finished translations: steps, selections and the device-side
    bookkeeping (mt_beam_finish) until every sentence has finished its K hypotheses or
    max_steps is reached (the last step finishes every live one).  The host looks at the
    beams every `check_every` steps (one synchronisation) to stop early.  Returns
    (n-best lists per sentence [(normalised score, score, tokens)], steps run)."""
    d, B, K, M = dec.device, dec.B, dec.K, dec.M
    dec.precompute(stream=stream)
    dec.start(tok0, score0)
    beam = torch.full((B,), K, dtype=torch.int32, device=d)
    fcount = torch.zeros(B, dtype=torch.int32, device=d)
    hist_tok = torch.empty((max_steps, M), dtype=torch.int32, device=d)
    hist_bp = torch.empty((max_steps, M), dtype=torch.int32, device=d)
    fs = torch.empty(M, dtype=torch.float32, device=d)
    fn = torch.empty(M, dtype=torch.float32, device=d)
    fst, fpa, fto = [torch.empty(M, dtype=torch.int32, device=d) for _ in range(3)]
    steps = 0
    for t in range(max_steps):
        dec.advance(stream=stream)
        mt.mt_beam_finish(dec.model, B, K, t, eos, alpha, t == max_steps - 1, dec.tok, dec.bp, dec.row, dec.score,
                          beam, fcount, hist_tok[t], hist_bp[t], fs, fn, fst, fpa, fto, stream=stream)
        steps = t + 1
        if (t + 1) % check_every == 0 and int(beam.sum().item()) == 0:
            break
    # the n-best lists ranked and backtracked on the device (mt_beam_nbest); the host only
    # unpacks them
    order = torch.empty(M, dtype=torch.int32, device=d)
    seq = torch.empty((M, max(steps, 1)), dtype=torch.int32, device=d)
    mt.mt_beam_nbest(dec.model, B, K, steps, hist_tok, hist_bp, fcount, fn, fst, fpa, fto, order, seq, stream=stream)
    fc, od, sq = fcount.cpu().numpy(), order.cpu().numpy(), seq.cpu().numpy()
    fs, fn, fst = fs.cpu().numpy(), fn.cpu().numpy(), fst.cpu().numpy()
    nbest = []
    for b in range(B):
        lst = []
        for r in range(min(int(fc[b]), K)):
            f = b * K + int(od[b * K + r])
            lst.append((float(fn[f]), float(fs[f]), sq[b * K + r, :int(fst[f]) + 1].tolist()))
        nbest.append(lst)
    return nbest, steps


class Ensemble:
    """Members decoding one beam (ensembling, a meta-algorithm of batched beam search), each
    with its own states.  Fused (the default): every member's step adds its weighted logits
    into one buffer (mt_ensemble_step) and one selection subtracts the per-row constant
    sum_i w_i LSE_i (mt_ensemble_topk), selecting from the beam candidates the last member
    collected on the combined values; where the library supports it (joint) the members' steps
    stop after the readout and one vocabulary pass serves them all.  Materialised (fused=False): every member writes its
    log-probabilities, mt_ensemble_logp combines them and mt_beam_topk selects.  Either way the
    first member's beam buffers hold the beam that all members read next."""

    def __init__(self, members, weights, fused=True, joint=None, concurrent=True):
        assert len(members) == len(weights) >= 1
        self.members, self.weights = list(members), [float(x) for x in weights]
        self.lead = self.members[0]
        self.fused = fused
        # fused: one vocabulary pass for all members where the library supports it (no combined
        # buffer), else each member adds its weighted logits into the combined buffer
        ok = fused and mt.mt_ensemble_joint_ok([d.model for d in self.members])
        self.joint = ok if joint is None else bool(joint)
        if self.joint and not ok:
            raise ValueError("the joint vocabulary pass does not support these members")
        # Members whose steps are independent (the joint pass, or materialised log-probabilities)
        # run on streams of their own, so that one member's latency-bound kernels overlap the
        # other's; the per-member fused pass adds into one buffer in member order and stays on
        # the caller's stream.  The streams keep the default priority.
        self.concurrent = concurrent and len(self.members) > 1 and (self.joint or not self.fused)
        dev = self.lead.device
        self.streams = [torch.cuda.Stream(device=dev) for _ in self.members] if self.concurrent else None
        self._ev = [torch.cuda.Event() for _ in range(len(self.members) + 1)] if self.concurrent else None

    def set_batch(self, ctx: np.ndarray, mask: np.ndarray, K: int):
        if self.concurrent:  # the members' old buffers may still be in use on their streams
            torch.cuda.synchronize(self.lead.device)
        for d in self.members:
            d.set_batch(ctx, mask, K)
        self._alloc_logp()

    def _alloc_logp(self):
        lead = self.lead
        if self.concurrent:  # no member stream may still use buffers that are about to be replaced
            torch.cuda.synchronize(lead.device)
        # the fused path needs only the combined buffer, the joint pass not even that
        self.logp = [None if self.fused else torch.empty((lead.M, lead.V), dtype=torch.float32, device=lead.device)
                     for _ in self.members]
        self.comb = None if self.joint else torch.empty((lead.M, lead.V), dtype=torch.float32, device=lead.device)

    def set_source(self, src_tok: np.ndarray, mask: np.ndarray, K: int, stream=None):
        """Batch from source tokens: every member encodes them with its own encoder (mt_encode)
        into its own context, as each member of an ensemble has its own encoder."""
        if self.concurrent:
            torch.cuda.synchronize(self.lead.device)
        for d in self.members:
            d.set_source(src_tok, mask, K, stream=stream)
        self._alloc_logp()

    def encode(self, stream=None):
        for d in self.members:
            d.encode(stream=stream)

    def precompute(self, stream=None):
        for d in self.members:
            d.precompute(stream=stream)

    def start(self, tok0: np.ndarray, score0: np.ndarray):
        for d in self.members:
            d.start(tok0, score0)

    def advance(self, stream=None, row_const=None):
        lead = self.lead
        base = stream if stream is not None else torch.cuda.current_stream(lead.device)
        if self.concurrent:  # the members' streams start after what the caller queued
            self._ev[-1].record(base)
        for i, (d, lp) in enumerate(zip(self.members, self.logp)):
            if d.first:
                state_in, nrows = d.s0, d.B
            else:
                state_in, nrows = d.state[d.cur], d.M
            out = d.state[1 - d.cur] if not d.first else d.state[d.cur]
            st = base
            if self.concurrent:
                st = self.streams[i]
                st.wait_event(self._ev[-1])
            with d._reuse():
                if self.fused:
                    mt.mt_ensemble_step(d.model, i, len(self.members), self.weights[i], d.B, d.K, d.S, lead.tok,
                                        lead.row, nrows, state_in, d.ctx, d.pctx, d.mask, out, self.comb, d.ws,
                                        stream=st)
                else:
                    d.step(lead.tok, lead.row, state_in, nrows, out, logp=lp, stream=st)
            if self.concurrent:
                self._ev[i].record(st)
        if self.concurrent:  # the selection waits for every member
            for i in range(len(self.members)):
                base.wait_event(self._ev[i])
        stream = base
        if self.fused:
            mt.mt_ensemble_topk([d.model for d in self.members], self.weights, [d.ws for d in self.members], lead.B,
                                lead.K, lead.score, self.comb, lead.score, lead.tok, lead.bp, lead.row,
                                row_const_out=row_const, stream=stream)
        else:
            mt.mt_ensemble_logp(lead.model, self.logp, self.weights, lead.M, self.comb, stream=stream)
            lead.topk(lead.score, self.comb, stream=stream)
        for d in self.members:
            if not d.first:
                d.cur = 1 - d.cur
            d.first = False
        return [d.state[d.cur] for d in self.members]


class SsmLayer:
    """A recurrent layer of the state space kind for serving: over a padded batch of prompts, then
    token by token for hypotheses whose states are gathered along the beam, as the Decoder's are.  Its calls run on
    its own device, whichever is current.

        [x' | z] = u Win,  x = conv(x'),  [r | B | C] = x Wx,  dt = r Wdt,  y = scan(x, dt, B, C; z),  out = y Wout

    weights: Win [E, 2D], Wx [D, R + 2GN], Wdt [R, D], Wout [D, E], optional biases bin [2D], bout [E]
    (products in 8 bits), and the cell's A, dt_bias, skip, conv_w, conv_b (see mt_ssm_weights)."""

    def __init__(self, weights, *, groups: int = 1, conv_silu: bool = True, dtype: str = "bf16", device: str = "cuda:0"):
        w = weights
        self.E, self.D, self.R = w["Win"].shape[0], w["Wout"].shape[0], w["Wdt"].shape[0]
        self.N, self.GN, self.W = w["A"].shape[1], groups * w["A"].shape[1], w["conv_w"].shape[1]
        self.device = torch.device(device)
        if self.device.index is None:  # the device that is current now, for good
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.io_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        cfg = mt.make_ssm_config(self.D, self.N, groups=groups, conv=self.W, conv_silu=conv_silu, dtype=dtype)
        with torch.cuda.device(self.device):
            self.cell = mt.mt_ssm_load(cfg, {k: w.get(k) for k in mt.SSM_WEIGHT_FIELDS})
            self.win = mt.mt_i8_load(w["Win"], w.get("bin"))
            self.wx, self.wdt = mt.mt_i8_load(w["Wx"]), mt.mt_i8_load(w["Wdt"])
            self.wout = mt.mt_i8_load(w["Wout"], w.get("bout"))

    def _buffers(self, lead):
        """Activations and workspace of a call over rows of shape lead."""
        io = dict(dtype=self.io_dtype, device=self.device)
        M = int(np.prod(lead))
        # one product at a time uses the workspace, the scan after them
        n = max([mt.mt_i8_workspace_bytes(w, M) for w in (self.win, self.wx, self.wdt, self.wout)] +
                ([mt.mt_ssm_workspace_bytes(self.cell, *lead)] if len(lead) == 2 else []))
        return dict(xz=torch.zeros(*lead, 2 * self.D, **io), x=torch.zeros(*lead, self.D, **io),
                    rbc=torch.zeros(*lead, self.R + 2 * self.GN, **io), dt=torch.zeros(*lead, self.D, **io),
                    y=torch.zeros(*lead, self.D, **io), out=torch.zeros(*lead, self.E, **io),
                    ws=torch.empty(n, dtype=torch.uint8, device=self.device))

    def _states(self, rows):
        return (torch.zeros(rows, self.W - 1, self.D, dtype=self.io_dtype, device=self.device),
                torch.zeros(rows, self.D, self.N, dtype=torch.float32, device=self.device))

    def set_batch(self, B: int, S: int, K: int):
        """Buffers for B prompts of padded length S and K hypotheses of each.  Waits for the device (unless it is
        captured into a graph): prompt and step may then run on any stream, and the last batch's work, wherever it
        ran, has ended when its buffers are given back."""
        with torch.cuda.device(self.device):
            pb, sb = self._buffers((B, S)), self._buffers((B * K,))
            prompt_state, beam_state = self._states(B), [self._states(B * K) for _ in range(2)]
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.synchronize(self.device)
        self.B, self.S, self.K, self.M = B, S, K, B * K
        self.pb, self.sb, self.prompt_state, self.beam_state = pb, sb, prompt_state, beam_state
        self.cur = -1  # the states a step reads: the prompts' (-1), or those of the last step

    def _project(self, u, f, stream):
        mt.mt_i8_product(self.win, u, f["xz"], f["ws"], stream=stream)
        return f["xz"][..., :self.D], f["xz"][..., self.D:]

    def _inputs(self, f, stream):
        mt.mt_i8_product(self.wx, f["x"], f["rbc"], f["ws"], stream=stream)
        mt.mt_i8_product(self.wdt, f["rbc"][..., :self.R], f["dt"], f["ws"], stream=stream)
        return f["x"], f["dt"], f["rbc"][..., self.R:self.R + self.GN], f["rbc"][..., self.R + self.GN:]

    def prompt(self, u, lens=None, stream=None):
        """u [B, S, E] in the io type, lens [B] int32: out [B, S, E] (valid positions); keeps the states."""
        f, (cs, hs) = self.pb, self.prompt_state
        with torch.cuda.device(self.device):
            xp, z = self._project(u, f, stream)
            mt.mt_ssm_conv(self.cell, xp, f["x"], lens=lens, state_out=cs, stream=stream)
            x, dt, bm, cm = self._inputs(f, stream)
            mt.mt_ssm_scan(self.cell, x, dt, bm, cm, f["y"], z=z, lens=lens, state_out=hs, ws=f["ws"], stream=stream)
            mt.mt_i8_product(self.wout, f["y"], f["out"], f["ws"], stream=stream)
        self.cur = -1
        return f["out"]

    def step(self, u, src_row, stream=None):
        """u [M, E]: out [M, E].  src_row [M] int32: the state row each hypothesis continues, of the prompts
        (m // K) in the first step and of the previous step afterwards (row_out of mt_beam_topk)."""
        f = self.sb
        ci, hi = self.prompt_state if self.cur < 0 else self.beam_state[self.cur]
        nxt = 0 if self.cur != 0 else 1
        co, ho = self.beam_state[nxt]
        with torch.cuda.device(self.device):
            xp, z = self._project(u, f, stream)
            mt.mt_ssm_conv_step(self.cell, xp, f["x"], ci, co, src_row=src_row, stream=stream)
            x, dt, bm, cm = self._inputs(f, stream)
            mt.mt_ssm_step(self.cell, x, dt, bm, cm, f["y"], hi, ho, z=z, src_row=src_row, stream=stream)
            mt.mt_i8_product(self.wout, f["y"], f["out"], f["ws"], stream=stream)
        self.cur = nxt
        return f["out"]


class PagedCache:
    """The keys and values of a program's attention layers in pages, k, v [layers, n_pages, Hk, page, Dh], and the table and
    lengths of its current rows: prompts first, then hypotheses that continue one another's.  Making one, and the first
    advance to a number of rows from one power of two to the next, wait for the device (unless captured into a graph): any
    stream may follow.

    An advance that finds too few pages writes none and leaves rows of no positions, over which a layer's calls give zeros;
    check() says so and goes back.  Where the pool may run out it has to be called before the next advance, which
    would take the pages of the rows that were lost for free ones."""

    def __init__(self, attn: mt.Attn, layers: int, n_pages: int, n_blocks: int):
        self.attn, self.n_blocks = attn, n_blocks
        shape = (layers, n_pages) + tuple(attn.page_shape)
        self.k, self.v = (torch.zeros(shape, dtype=attn.dtype, device=attn.device) for _ in range(2))
        self.free = torch.full((1,), n_pages, dtype=torch.int32, device=attn.device)
        self._spare, self._before = {}, None
        self.table, self.lens, _ = self._rows(1)  # one empty row, for new ones to begin with
        self.lens.zero_()
        self._wait()

    def _wait(self):
        with torch.cuda.device(self.attn.device):
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.synchronize(self.attn.device)

    def _rows(self, n):
        """A table and lengths of n rows that are not the current ones, and a workspace: of two each for up to a power of two."""
        i32, most = dict(dtype=torch.int32, device=self.attn.device), 1 << (n - 1).bit_length()
        if most not in self._spare:
            ws = mt.mt_pages_workspace_bytes(self.attn, most, self.k.shape[1])
            self._spare[most] = [(torch.empty(most, self.n_blocks, **i32), torch.empty(most, **i32)) for _ in range(2)] + [
                torch.empty(ws, dtype=torch.uint8, device=self.attn.device)]
            self._wait()
        one, other, ws = self._spare[most]
        current = getattr(self, "table", None)
        table, lens = other if current is not None and current.data_ptr() == one[0].data_ptr() else one
        return table[:n], lens[:n], ws

    def advance(self, src_row, add=None, stream=None):
        """Rows that continue src_row [M] int32 (below 0: new ones) of the current ones, with room for add [M] (None: 1 each)
        more positions."""
        n = src_row.numel()
        table, lens, ws = self._rows(n)
        with torch.cuda.device(self.attn.device):
            mt.mt_pages_advance(self.attn, src_row, add, self.table, self.lens, table, lens, self.k, self.v, free_out=self.free,
                                ws=ws, stream=stream)
        self._before = self.table, self.lens  # as they were until the next advance
        self.table, self.lens = table, lens

    def check(self) -> int:
        """Waits for the device and gives the layer's device-side error bits (mt_attn_device_errors, which clears them).  Where
        the last advance found no room (bit 8), the rows before it are the current ones again."""
        with torch.cuda.device(self.attn.device):
            flags = mt.mt_attn_device_errors(self.attn)
            if flags & 8 and self._before and int(self.free) == self.k.shape[1] and not bool(self.lens.any()):
                (self.table, self.lens), self._before = self._before, None
                n = self.lens.numel()  # the free pages beside these rows: that of a step in which none grows
                table, lens, ws = self._rows(n)
                mt.mt_pages_advance(self.attn, None, torch.zeros_like(self.lens), self.table, self.lens, table, lens, self.k, self.v,
                                    free_out=self.free, ws=ws)
                self._wait()
        return flags

    def pack(self, n_pages: int, stream=None) -> "PagedCache":
        """A cache of n_pages that holds the current rows, their pages at its front (rows of no positions where n_pages do not
        suffice, which check() tells; this cache stays as it is)."""
        out = PagedCache(self.attn, self.k.shape[0], n_pages, self.n_blocks)
        n = self.lens.numel()
        table, lens, _ = out._rows(n)
        ws = torch.empty(mt.mt_pages_workspace_bytes(self.attn, n, self.k.shape[1]), dtype=torch.uint8, device=self.attn.device)
        self._wait()
        with torch.cuda.device(self.attn.device):
            mt.mt_pages_pack(self.attn, self.table, self.lens, self.k, self.v, table, lens, out.k, out.v, out.free, ws=ws,
                             stream=stream)
        self._wait()  # the workspace is given back
        out.free.neg_().add_(n_pages)  # the used pages, until here
        out._wait()
        out.table, out.lens = table, lens
        return out


class AttnLayer:
    """The attention of a decoder's layer for serving: over the positions before (a PagedCache that layers share), for pieces
    of prompts and for single tokens of hypotheses, and over an encoder's states (mt_encode's context).  Its calls run on
    its own device, whichever is current.

        [q | k | v] = u Wqkv,  out = attention(q, cache) Wo;   q' = u Wcq,  [k' | v'] = ctx Wckv,  out' = attention(q', k', v') Wco

    weights: Wqkv [E, (Hq + 2Hk) Dh], Wo [Hq Dh, E], optional biases bqkv, bo; with cross attention Wcq [E, Hq Dh],
    Wckv [C, 2 Hk Dh], Wco [Hq Dh, E], biases bcq, bckv, bco (products in 8 bits); gq, gk, freq (see mt_attn_weights)."""

    def __init__(self, weights, Hq: int, Hk: int, *, page: int = 16, dtype: str = "bf16", device: str = "cuda:0", **heads):
        w = weights
        self.E = w["Wqkv"].shape[0]
        self.Dh = w["Wqkv"].shape[1] // (Hq + 2 * Hk)
        self.QD, self.KD = Hq * self.Dh, Hk * self.Dh
        self.device = torch.device(device)
        if self.device.index is None:  # the device that is current now, for good
            self.device = torch.device("cuda", torch.cuda.current_device())
        cfg = mt.make_attn_config(Hq, Hk, self.Dh, page=page, dtype=dtype, **heads)
        with torch.cuda.device(self.device):
            self.attn = mt.mt_attn_load(cfg, {k: w.get(k) for k in mt.ATTN_WEIGHT_FIELDS})
            self.wqkv, self.wo = mt.mt_i8_load(w["Wqkv"], w.get("bqkv")), mt.mt_i8_load(w["Wo"], w.get("bo"))
            self.cross_w = [mt.mt_i8_load(w["W" + n], w.get("b" + n)) for n in ("cq", "ckv", "co")] if "Wcq" in w else None
        self.io_dtype = self.attn.dtype

    def _buffers(self, B, S, n_keys, S_src):
        io = dict(dtype=self.io_dtype, device=self.device)
        mats = [self.wqkv, self.wo] + (self.cross_w[::2] if S_src else [])
        n = [mt.mt_i8_workspace_bytes(m, B * S) for m in mats] + [mt.mt_attn_workspace_bytes(self.attn, B, S, n_keys)]
        return dict(qkv=torch.zeros(B, S, self.QD + 2 * self.KD, **io), y=torch.zeros(B, S, self.QD, **io),
                    out=torch.zeros(B, S, self.E, **io), ws=torch.empty(max(n), dtype=torch.uint8, device=self.device))

    def set_batch(self, B: int, S: int, K: int, n_keys: int, S_src: int = 0):
        """Buffers for pieces of S positions of B prompts, single tokens of K hypotheses of each, over n_keys positions (the
        cache's n_blocks * page), and S_src encoder states a sentence.  Waits for the device (unless captured)."""
        with torch.cuda.device(self.device):
            pb, sb = self._buffers(B, S, n_keys, 0), self._buffers(B * K, 1, n_keys, 0)
            xb = kv = None
            if S_src:
                io = dict(dtype=self.io_dtype, device=self.device)
                xb, kv = self._buffers(B, K, S_src, S_src), torch.zeros(B, S_src, 2 * self.KD, **io)
                kws = torch.empty(mt.mt_i8_workspace_bytes(self.cross_w[1], B * S_src), dtype=torch.uint8, device=self.device)
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.synchronize(self.device)
        self.B, self.S, self.K, self.M = B, S, K, B * K
        self.pb, self.sb, self.xb, self.src_kv, self.src_ws = pb, sb, xb, kv, kws if S_src else None

    def _self(self, f, u, cache, layer, n_new, stream):
        B, S = u.shape[:2]
        q, k, v = (f["qkv"][..., a:b] for a, b in ((0, self.QD), (self.QD, self.QD + self.KD), (self.QD + self.KD, None)))
        with torch.cuda.device(self.device):
            mt.mt_i8_product(self.wqkv, u, f["qkv"], f["ws"], stream=stream)
            mt.mt_attn_append(self.attn, q, k, v, q, cache.lens, cache.table, cache.k[layer], cache.v[layer], n_new=n_new,
                              stream=stream)
            mt.mt_attn_paged(self.attn, q, cache.lens, cache.table, cache.k[layer], cache.v[layer], f["y"], n_new=n_new,
                             ws=f["ws"], stream=stream)
            mt.mt_i8_product(self.wo, f["y"], f["out"], f["ws"], stream=stream)
        return f["out"]

    def prompt(self, u, cache: PagedCache, layer: int = 0, n_new=None, stream=None):
        """u [B, S, E]: the new positions of the cache's rows (its advance has made room), n_new [B] int32 of them: out
        [B, S, E]."""
        return self._self(self.pb, u, cache, layer, n_new, stream)

    def step(self, u, cache: PagedCache, layer: int = 0, stream=None):
        """u [M, E], a token of each row: out [M, E]."""
        return self._self(self.sb, u[:, None], cache, layer, None, stream)[:, 0]

    def set_source(self, ctx, mask, stream=None):
        """ctx [B, S_src, C] in the io type, mask [B, S_src] fp32: the keys and values of the cross attention."""
        self.mask = mask
        with torch.cuda.device(self.device):
            mt.mt_i8_product(self.cross_w[1], ctx, self.src_kv, self.src_ws, stream=stream)

    def cross(self, u, stream=None):
        """u [M, E], hypotheses m of sentence m // K: out [M, E]."""
        f = self.xb
        q = f["qkv"].view(-1)[:self.M * self.QD].view(self.B, self.K, self.QD)
        with torch.cuda.device(self.device):
            mt.mt_i8_product(self.cross_w[0], u.view(self.B, self.K, self.E), q, f["ws"], stream=stream)
            mt.mt_attn_cross(self.attn, q, self.src_kv[..., :self.KD], self.src_kv[..., self.KD:], f["y"], mask=self.mask,
                             ws=f["ws"], stream=stream)
            mt.mt_i8_product(self.cross_w[2], f["y"], f["out"], f["ws"], stream=stream)
        return f["out"].view(self.M, self.E)
