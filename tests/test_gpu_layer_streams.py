"""The recurrent layer on streams other than the current one."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_layer import DEV, gen
from test_gpu_ssm_layer import E, G, weights

if torch.cuda.is_available():
    from paper_1804_00344_amd.runner import SsmLayer

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BUSY = 200_000_000  # cycles: the current stream is behind by about 0.1 s


def batch(layer, B, S, K):
    u = torch.randn(B, S, E, generator=gen(5)).to(layer.io_dtype).to(DEV)
    v = torch.randn(B * K, E, generator=gen(6)).to(layer.io_dtype).to(DEV)
    rows = (torch.arange(B * K, device=DEV) // K).to(torch.int32)
    return u, v, rows


def run(layer, u, v, rows, stream):
    a = layer.prompt(u, stream=stream)
    b = layer.step(v, rows, stream=stream)
    return a, b, *layer.prompt_state, *layer.beam_state[layer.cur]


def test_a_side_stream_right_after_set_batch():
    """The buffers are ready for any stream: what the current stream still has to do does not reach them."""
    B, S, K = 3, 21, 4
    layer = SsmLayer(weights(3), groups=G, dtype="f32")
    layer.set_batch(B, S, K)
    u, v, rows = batch(layer, B, S, K)
    want = [t.clone() for t in run(layer, u, v, rows, None)]
    torch.cuda.synchronize()
    for use in ("argument", "current"):
        side = torch.cuda.Stream()
        torch.cuda._sleep(BUSY)
        layer.set_batch(B, S, K)
        if use == "argument":
            got = run(layer, u, v, rows, side)
        else:
            with torch.cuda.stream(side):
                got = run(layer, u, v, rows, None)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), use


def test_set_batch_waits_for_the_last_batch():
    """Work of the last batch on a side stream does not write into memory that is given back and used again."""
    B, S, K = 3, 50, 4
    layer = SsmLayer(weights(3), groups=G, dtype="f32")
    layer.set_batch(B, S, K)
    u, v, rows = batch(layer, B, S, K)
    sizes = [t.shape for t in layer.pb.values()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    run(layer, u, v, rows, side)
    layer.set_batch(B, S, K)
    mine = [torch.full(s, 7.0, device=DEV) for s in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(bool((t == 7.0).all()) for t in mine)


def test_set_batch_within_a_capture():
    """A batch set up, run and replayed as one graph; it cannot wait for the device and need not."""
    B, S, K = 2, 19, 3
    layer = SsmLayer(weights(4), groups=G, dtype="f32")
    layer.set_batch(B, S, K)
    u, v, rows = batch(layer, B, S, K)
    want = [t.clone() for t in run(layer, u, v, rows, None)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.set_batch(B, S, K)
        got = run(layer, u, v, rows, None)
    for i in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i
