"""The recurrent layer's operators together, as runner.SsmLayer calls them: ragged prompts, then beam
search over the layer's outputs with an output layer in 8 bits and mt_beam_topk, whose row_out gathers the
next step's states.  Every stage is checked in 64 bits from the inputs that the GPU's stage read."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref
from paper_1804_00344_amd import mtstep as mt
from paper_1804_00344_amd import synth
from test_gpu_layer import DEV, check, gen, per_channel

if torch.cuda.is_available():
    from paper_1804_00344_amd.runner import Decoder, SsmLayer

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

E, D, N, R, G, W = 32, 72, 16, 6, 2, 4


def weights(seed):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    return dict(Win=r(E, 2 * D) / 4, bin=r(2 * D) / 4, Wx=r(D, R + 2 * G * N) / 6, Wdt=r(R, D) / 2, Wout=r(D, E) / 6, bout=r(E),
                A=-torch.exp(r(D, N)), dt_bias=r(D) - 3, skip=r(D), conv_w=r(D, W) / 2, conv_b=r(D))


def cpu64(t):
    return t.detach().cpu().double()


def check_product(x, wname, bname, w, y, what):
    want, err = ref.product(x.detach().float().cpu().reshape(-1, x.shape[-1]).numpy(), w[wname].numpy(),
                            w[bname].numpy() if bname else None)
    check(y.reshape(-1, y.shape[-1]), torch.from_numpy(want), torch.from_numpy(err), what)


def check_stages(f, u, w, states_in, states_out, lens):
    """One pass over rows [B, S, ..] (a step: S = 1) from the states each row starts from."""
    c = lambda t: cpu64(t).reshape(len(lens), -1, t.shape[-1])
    check_product(u, "Win", "bin", w, f["xz"], "in")
    check_product(f["x"], "Wx", None, w, f["rbc"], "x")
    check_product(f["rbc"][..., :R], "Wdt", None, w, f["dt"], "dt")
    check_product(f["y"], "Wout", "bout", w, f["out"], "out")
    p = {k: v.double() for k, v in w.items()}
    for b, n in enumerate(lens):
        got = lambda t: t.reshape(len(lens), -1, t.shape[-1])[b, :n]
        y, cs, err = ref.conv(c(f["xz"])[b, :n, :D], p["conv_w"], p["conv_b"], True, states_in[0][b])
        check(got(f["x"]), y, err, "conv")
        assert torch.equal(cpu64(states_out[0][b]), cs)
        bc = c(f["rbc"])[b, :n, R:]
        y, h, ye, he = ref.scan(c(f["x"])[b, :n], c(f["dt"])[b, :n], per_channel(bc, D, N, G, False), per_channel(bc, D, N, G, True),
                                c(f["xz"])[b, :n, D:], p["A"], p["dt_bias"], p["skip"], states_in[1][b])
        check(got(f["y"]), y, ye, "scan")
        check(states_out[1][b], h, he, "state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_then_beam(dtype):
    B, S, K, V, steps = 3, 21, 4, 1000, 4
    lens = [21, 0, 9]
    w = weights(3)
    layer = SsmLayer(w, groups=G, dtype=dtype)
    layer.set_batch(B, S, K)
    g = gen(5)
    u = torch.randn(B, S, E, generator=g).to(layer.io_dtype).to(DEV)
    layer.prompt(u, torch.tensor(lens, dtype=torch.int32, device=DEV))
    zeros = (torch.zeros(B, W - 1, D, dtype=torch.float64), torch.zeros(B, D, N, dtype=torch.float64))
    check_stages(layer.pb, u, w, zeros, layer.prompt_state, lens)

    emb = torch.randn(V, E, generator=g).to(layer.io_dtype).to(DEV)
    wo, bo = torch.randn(E, V, generator=g) / 2, torch.randn(V, generator=g)
    out_layer = mt.mt_i8_load(wo, bo)
    p = synth.with_sizes(synth.PRESETS["tiny_f32"], V=V, B=B, K=K)
    dec = Decoder.from_preset(p, synth.make_weights(p))
    M = B * K
    ws = torch.empty(mt.mt_workspace_bytes(dec.model, B, K, 8), dtype=torch.uint8, device=DEV)
    lws = torch.empty(mt.mt_i8_workspace_bytes(out_layer, M), dtype=torch.uint8, device=DEV)
    logits = torch.empty(M, V, device=DEV)
    score = torch.tensor([0.0] + [-1e30] * (K - 1), device=DEV).repeat(B)  # one live hypothesis each
    tok, bp, row = (torch.empty(M, dtype=torch.int32, device=DEV) for _ in range(3))
    rows = (torch.arange(M, device=DEV) // K).to(torch.int32)  # the first step continues the prompts
    tok.fill_(1)
    moved = False
    for t in range(steps):
        before = [cpu64(s)[rows.cpu().long()] for s in (layer.prompt_state if layer.cur < 0 else layer.beam_state[layer.cur])]
        x = emb[tok.long()]
        out = layer.step(x, rows)
        check_stages(layer.sb, x, w, before, layer.beam_state[layer.cur], [1] * M)
        mt.mt_i8_product(out_layer, out, logits, lws)
        check_product(out, "wo", "bo", dict(wo=wo, bo=bo), logits, "logits")
        prev = score.clone()
        logp = torch.log_softmax(logits, 1)
        mt.mt_beam_topk(dec.model, B, K, score, logp, score, tok, bp, row, ws)
        flat = (prev[:, None] + logp).reshape(B, K * V)
        assert torch.equal(score.reshape(B, K), flat.topk(K, 1)[0])
        rows = row.clone()
        moved = moved or not torch.equal(rows, torch.arange(M, dtype=torch.int32, device=DEV))
    assert moved  # hypotheses changed their places: the states were gathered
    assert mt.mt_ssm_device_errors(layer.cell) == 0
