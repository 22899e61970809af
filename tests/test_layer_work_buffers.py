"""Work buffers of LinearW4A4: calls that may overlap never share them.  CPU: which buffers a call takes, with the library replaced by
recorders.  GPU: two streams with different inputs of one size give what single calls give."""
import contextlib
import threading
import types

import pytest
import torch

from paper_2607_21446_b200 import binding as kb


@pytest.fixture
def calls(monkeypatch):
    """A layer on CPU tensors; the list of (codes, scales) that its calls hand to the library, kept alive as a running call would."""
    seen = []
    layer = kb.LinearW4A4(types.SimpleNamespace(_h=None), torch.zeros(64, 80, dtype=torch.uint8), torch.zeros(kb.tiled_scale_bytes(64, 160), dtype=torch.uint8))
    allocated = []

    def recorded(make):
        def f(*a, **kw):
            t = make(*a, **kw)
            allocated.append(t)
            return t
        return f

    monkeypatch.setattr(kb.torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(kb.torch, "zeros", recorded(torch.zeros))
    monkeypatch.setattr(kb, "_x_shape", lambda X: tuple(X.shape))
    monkeypatch.setattr(kb, "_stream", lambda s: 0 if s is None else s)
    monkeypatch.setattr(kb, "_allocating", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(kb, "_capturing", lambda: calls_state["capturing"], raising=False)
    monkeypatch.setattr(kb, "kroquant_quantize", lambda X, f, q, s, **kw: seen.append((q.data_ptr(), s.data_ptr())))
    monkeypatch.setattr(kb, "kroquant_linear_mxfp4", lambda q, s, *a, **kw: torch.zeros(q.shape[0], 64))
    monkeypatch.setattr(kb, "load_library", lambda: types.SimpleNamespace(
        kroquant_linear_w4a4=lambda *a: seen.append((_value(a[8]), _value(a[9]))) or 0))
    calls_state = {"capturing": False}
    return types.SimpleNamespace(layer=layer, seen=seen, state=calls_state, allocated=allocated)


def _value(p):
    return p.value if hasattr(p, "value") else p


@pytest.mark.parametrize("fused", [True, False])
def test_one_pair_for_each_stream_thread_and_captured_call(calls, fused):
    X, longer = torch.zeros(10, 160, dtype=torch.bfloat16), torch.zeros(300, 160, dtype=torch.bfloat16)
    call, seen = calls.layer.fused if fused else calls.layer, calls.seen
    call(X, stream=1), call(X, stream=2), call(X, stream=1)
    assert seen[0] == seen[2] and seen[0][0] != seen[1][0] and seen[0][1] != seen[1][1]
    call(longer, stream=1), call(X, stream=1)                   # grown once, then enough for both
    assert seen[3] == seen[4] and seen[3] != seen[0]
    call(X, stream=2)
    assert seen[5] == seen[1]
    calls.state["capturing"] = True                             # a graph runs next to later calls
    call(X, stream=1), call(X, stream=1)
    assert len({seen[4], seen[6], seen[7]}) == 3
    calls.state["capturing"] = False
    call(X, stream=1)
    assert seen[8] == seen[4]
    other = threading.Thread(target=call, args=(X,), kwargs={"stream": 1})
    other.start(), other.join()
    assert seen[9] not in seen[:9]


def test_both_forms_of_the_layer_share_a_pair_on_one_stream(calls):
    X = torch.zeros(10, 160, dtype=torch.bfloat16)
    calls.layer.fused(X, stream=1), calls.layer(X, stream=1)
    assert calls.seen[0] == calls.seen[1]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1152, 2240])
@pytest.mark.parametrize("tokens", [40, 1000])
@pytest.mark.parametrize("fused", [True, False])
def test_two_streams_with_equal_token_counts(d, tokens, fused):
    from examples.quantized_block import dense_layer, randn
    g = torch.Generator(device="cuda")
    g.manual_seed(d + tokens)
    layer = dense_layer(randn(g, 4096, d, gain=d ** -0.5))
    xs = [randn(g, tokens, d) for _ in range(2)]
    call = layer.fused if fused else layer
    want = []
    for x in xs:
        want.append(call(x).clone())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs.append((i, call(xs[i])))
    for _ in range(4):                                          # and with the stream as an argument, into buffers made before
        for i, s in enumerate(streams):
            out = torch.empty(tokens, 4096, device="cuda", dtype=torch.bfloat16)
            s.wait_stream(torch.cuda.current_stream())
            outs.append((i, call(xs[i], out=out, stream=s)))
    torch.cuda.synchronize()
    for i, o in outs:
        assert torch.equal(o, want[i])
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("fused", [True, False])
def test_captured_calls_next_to_later_ones(fused):
    from examples.quantized_block import dense_layer, randn
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    layer = dense_layer(randn(g, 1024, 2240, gain=0.02))
    a, b = randn(g, 500, 2240), randn(g, 500, 2240)
    call = layer.fused if fused else layer
    want_a, want_b = call(a).clone(), call(b).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = []
    for _ in range(4):
        graph.replay()
        with torch.cuda.stream(side):
            eager.append(call(b))
    torch.cuda.synchronize()
    assert torch.equal(out, want_a) and all(torch.equal(e, want_b) for e in eager)
