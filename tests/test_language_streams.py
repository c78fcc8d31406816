"""Calls of the operators for language models on a stream that is not the current one: where their memory comes from, and how long it stays.
What was wrong is shown on the CPU, with stand-ins for the streams; the GPU tests run the calls themselves."""
import contextlib

import pytest
import torch

import paper_2010_08679_amd as P
from paper_2010_08679_amd import language

DEV = "cuda:0"


class Stream:
    """Keeps what it was told."""

    def __init__(self):
        self.waited_for = []

    def wait_stream(self, other):
        self.waited_for.append(other)


class Allocations:
    """Which stream was current at each torch.empty, and which streams tensors were recorded on."""

    def __init__(self, monkeypatch, capturing=False):
        self.current, self.made, self.recorded = None, [], []
        empty = torch.empty

        def recorded_empty(*args, **kwargs):
            self.made.append(self.current)
            return empty(*args, **kwargs)

        @contextlib.contextmanager
        def on(stream):
            before, self.current = self.current, stream
            yield
            self.current = before

        monkeypatch.setattr(torch, "empty", recorded_empty)
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.recorded.append((t.data_ptr(), s)))
        for name in ("cnr_quantize_blocks", "cnr_block_product", "cnr_count_tokens", "cnr_adjust_logits"):
            monkeypatch.setattr(language.L, name, lambda *args: None)

    def of(self, call):
        self.made.clear()
        result = call()
        assert self.current is None
        return result, set(self.made)


def test_results_are_allocated_on_the_stream_of_the_call(monkeypatch):
    a, b = P.BlockMatrix.empty(4, 100, device="cpu"), P.BlockMatrix.empty(6, 100, device="cpu")
    seen, side = Allocations(monkeypatch), Stream()
    for stream in (None, side):
        assert seen.of(lambda: P.quantize_blocks(None, torch.zeros(4, 100), stream=stream))[1] == {stream}
        assert seen.of(lambda: P.block_product(None, a, b, stream=stream))[1] == {stream}


@pytest.mark.parametrize("capturing", [False, True])
def test_a_layer_allocates_on_the_stream_of_the_call_and_keeps_its_memory_for_it(monkeypatch, capturing):
    layer = P.BlockLinear(None, 6, 4, 300, device="cpu")
    made_on, side, other = Stream(), Stream(), Stream()
    layer._made_on = made_on  # as on a GPU
    space = iter(range(1 << 12, 1 << 20, 1 << 12))
    monkeypatch.setattr(language.L, "cnr_block_product_workspace_bytes", lambda *args: next(space))
    seen = Allocations(monkeypatch, capturing)
    buffers = {t.data_ptr() for t in (layer.weight.codes, layer.weight.scale, layer.weight_t.codes, layer.weight_t.scale, *layer._x, *layer._x_t, *layer._dy,
                                      *layer._dy_t)}
    layer.load(torch.zeros(6, 4), stream=side)
    assert side.waited_for == ([] if capturing else [made_on])
    assert {p for p, s in seen.recorded if s is side} == buffers
    for stream in (side, other):
        assert seen.of(lambda: layer.forward(torch.zeros(3 + 40 * (stream is other), 4), stream=stream))[1] == {stream}  # the result and the workspace
        assert seen.of(lambda: layer.backward(torch.zeros(3 + 40 * (stream is other), 6), stream=stream))[1] == {stream}
    assert side.waited_for == other.waited_for == ([] if capturing else [made_on])
    for stream in (side, other):
        assert {p for p, s in seen.recorded if s is stream} >= buffers | {layer._spaces[-1].data_ptr()}
    assert (layer._spaces[0].data_ptr(), side) in seen.recorded
    seen.recorded.clear()
    assert seen.of(lambda: layer.forward(torch.zeros(9, 4)))[1] == {None}


def test_a_ledger_waits_for_the_state_that_it_made(monkeypatch):
    given = torch.zeros(2, 2, dtype=torch.int32)
    for ledger, own in ((P.TokenLedger(None, 2, 40, device="cpu"), 2), (P.TokenLedger(None, 2, 40, given, device="cpu"), 0)):
        ledger._made_on, side = Stream(), Stream()
        with monkeypatch.context() as patched:
            seen = Allocations(patched)
            ledger.count(torch.zeros(2, dtype=torch.int64), stream=side)
            ledger.adjust(torch.zeros(2, 40), stream=side)
        assert side.waited_for == [ledger._made_on] and len(seen.recorded) == own


def test_a_ledger_of_given_state_has_no_stream_of_its_own():
    given = torch.zeros(2, 2, dtype=torch.int32)
    ledger = P.TokenLedger(None, 2, 40, given)  # wherever it is, without a GPU too
    assert ledger.seen is given and ledger.counts is None and ledger._made_on is None


@pytest.mark.gpu
def test_results_on_another_stream_while_the_current_one_is_busy():
    # memory that work on the current stream still uses is free to that stream's next allocations only
    ctx = P.cnr_create(0)
    g = torch.Generator(device=DEV).manual_seed(1)
    m, n, k = 512, 768, 640
    x, w = torch.randn(m, k, generator=g, device=DEV).bfloat16(), torch.randn(n, k, generator=g, device=DEV)
    layer, again = P.BlockLinear(ctx, n, k, m), P.BlockLinear(ctx, n, k, m)
    layer.load(w)
    want = layer.forward(x)
    want_x, want_w = layer.backward(want)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, generator=g, device=DEV)
    torch.cuda.synchronize()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        old = [torch.empty(t.numel(), dtype=t.dtype, device=DEV) for t in (want, want_x, want_w, layer._x[0], layer._x_t[0])]
        for _ in range(20):
            busy = (busy @ busy).clamp_(-1, 1)
        for t in old:
            t.fill_(7)
        del old, t
        again.load(w, stream=side)
        y = again.forward(x, stream=side)
        dx, dw = again.backward(y, stream=side)
        q = P.quantize_blocks(ctx, x, stream=side)
        p = P.block_product(ctx, q, again.weight, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, want_x) and torch.equal(dw, want_w) and torch.equal(p, want)
    P.cnr_destroy(ctx)


@pytest.mark.gpu
def test_a_layers_first_calls_on_a_stream_are_captured():
    ctx = P.cnr_create(0)
    g = torch.Generator(device=DEV).manual_seed(2)
    n_in, n_out, tokens = 16384, 1024, 64
    layer, w = P.BlockLinear(ctx, n_out, n_in, tokens), torch.randn(n_out, n_in, generator=g, device=DEV)
    x = torch.randn(tokens, n_in, generator=g, device=DEV).bfloat16()
    layer.load(w)
    want = layer.forward(x)
    want_x, want_w = layer.backward(want)
    fresh, side, graph = P.BlockLinear(ctx, n_out, n_in, tokens), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fresh.load(w, stream=side)
        y = fresh.forward(x, stream=side)
        dx, dw = fresh.backward(y, stream=side)
    for _ in range(4):
        for t in (y, dx, dw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, want_x) and torch.equal(dw, want_w)
    assert fresh._spaces
    P.cnr_destroy(ctx)
