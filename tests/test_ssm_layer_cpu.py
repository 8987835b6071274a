"""runner.SsmLayer's order of calls without a GPU: the binding's calls are recorded, not made."""
import types

import numpy as np
import torch

from paper_1804_00344_amd import mtstep as mt
from paper_1804_00344_amd.runner import SsmLayer

E, D, N, R, W = 8, 12, 4, 2, 3


class Current:
    """In place of torch.cuda.device: the devices made current, innermost last."""
    stack = [torch.device("cuda", 0)]

    def __init__(self, device):
        self.device = torch.device(device)

    def __enter__(self):
        self.stack.append(self.device)

    def __exit__(self, *_):
        self.stack.pop()


def test_every_call_is_made_on_the_layers_device(monkeypatch):
    """A layer of another device than the current one: each call finds its device current, as its handle needs."""
    seen = []

    def call(name, result=None):
        def f(*a, **kw):
            seen.append((name, Current.stack[-1]))
            return result
        return f

    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", call("capturing", False))
    monkeypatch.setattr(torch.cuda, "synchronize", lambda d: None)
    monkeypatch.setattr(SsmLayer, "_buffers", lambda self, lead: {
        k: torch.zeros(*lead, n) for k, n in dict(xz=2 * D, x=D, rbc=R + 2 * N, dt=D, y=D, out=E, ws=1).items()})
    monkeypatch.setattr(SsmLayer, "_states", lambda self, rows: (torch.zeros(rows, W - 1, D), torch.zeros(rows, D, N)))
    handle = types.SimpleNamespace(device=torch.device("cuda", 1))
    for name in ("mt_ssm_load", "mt_i8_load"):
        monkeypatch.setattr(mt, name, call(name, handle))
    for name in ("mt_i8_product", "mt_ssm_conv", "mt_ssm_scan", "mt_ssm_conv_step", "mt_ssm_step"):
        monkeypatch.setattr(mt, name, call(name))
    z = lambda *s: np.zeros(s, np.float32)
    layer = SsmLayer(dict(Win=z(E, 2 * D), Wx=z(D, R + 2 * N), Wdt=z(R, D), Wout=z(D, E), A=z(D, N), conv_w=z(D, W)),
                     device="cuda:1")
    layer.set_batch(2, 5, 3)
    layer.prompt(torch.zeros(2, 5, E))
    layer.step(torch.zeros(6, E), torch.zeros(6, dtype=torch.int32))
    layer.step(torch.zeros(6, E), torch.zeros(6, dtype=torch.int32))
    names = [n for n, _ in seen]
    assert names.count("mt_i8_product") == 12 and {"mt_ssm_scan", "mt_ssm_conv", "mt_ssm_step", "mt_ssm_conv_step"} <= set(names)
    assert all(d == torch.device("cuda", 1) for _, d in seen), seen
    assert Current.stack == [torch.device("cuda", 0)]


def test_a_device_without_a_number_is_the_current_one_for_good(monkeypatch):
    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for name in ("mt_ssm_load", "mt_i8_load"):
        monkeypatch.setattr(mt, name, lambda *a: None)
    z = lambda *s: np.zeros(s, np.float32)
    layer = SsmLayer(dict(Win=z(E, 2 * D), Wx=z(D, R + 2 * N), Wdt=z(R, D), Wout=z(D, E), A=z(D, N), conv_w=z(D, W)), device="cuda")
    assert layer.device == torch.device("cuda", 1)
