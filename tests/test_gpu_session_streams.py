"""Sessions whose launches run on another stream than the one they were built on."""
import pytest
import torch

import decoder_util as D

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Busy:
    """Some tens of milliseconds of work for a stream."""

    def __init__(self):
        self.a = torch.ones(8192, 8192, dtype=torch.float16, device=DEV)
        self.c = torch.empty_like(self.a)
        self.on(torch.cuda.current_stream())
        torch.cuda.synchronize()

    def on(self, stream):
        with torch.cuda.stream(stream):
            for _ in range(60):
                torch.mm(self.a, self.a, out=self.c)


def attention(seed, n=6000):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (D.normal(g, (r, 8 * 64), "f16").to(DEV) for r in (1, n, n))
    return [q, k, v], D.attention(q, k, v, "f16", heads=8, width=64)


def bound(tensors):
    return D.bind(lambda b, e: b.attention(*e, heads=8, width=64), tensors)


def test_a_session_is_ready_for_any_stream_when_it_is_built():
    """Its results and counters are cleared on the building stream, which has other work to do first."""
    busy, building, side = Busy(), torch.cuda.Stream(), torch.cuda.Stream()
    for seed in range(3):
        tensors, want = attention(seed)
        torch.cuda.synchronize()
        busy.on(building)
        with torch.cuda.stream(building):
            s = bound(tensors)
        s.launch(side)
        with torch.cuda.stream(side):
            got = s.result(0).clone()
        torch.cuda.synchronize()
        D.within(got, *want, "f16")
        assert torch.equal(s.result(0), got)                   # nothing cleared it afterwards
        s.run_eager()
        assert torch.equal(s.result(0), got)                   # the counters are as the first launch needs them
        s.close()


def test_a_session_built_inside_a_capture():
    """Clearing and launch are both in the graph."""
    tensors, want = attention(5)
    table = [bound(tensors)]                                   # what a first use loads is loaded before
    table[0].launch()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = bound(tensors)
        s.launch()
        got = s.result(0) * 1
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        D.within(got, *want, "f16")
    s.close()


def test_a_dropped_sessions_memory_waits_for_its_launches():
    """Tensors made after a session has gone do not take its memory from a stream that still works on it."""
    busy, side = Busy(), torch.cuda.Stream()
    for seed in range(3):
        tensors, want = attention(seed, 60000)
        torch.cuda.synchronize()
        s = bound(tensors)
        addresses = {t.data_ptr() for t in [*s.ext_dev, *s.out_dev]}
        sizes = [t.numel() for t in s.ext_dev]
        busy.on(side)
        s.launch(side)
        with torch.cuda.stream(side):
            got = s.result(0).clone()
        s.close()
        del s, tensors
        fresh = [torch.full((n,), float("nan"), dtype=torch.float16, device=DEV) for n in sizes * 2]
        assert not addresses & {t.data_ptr() for t in fresh}
        torch.cuda.synchronize()
        D.within(got, *want, "f16")


def test_streams_of_another_device_are_refused():
    tensors, _ = attention(1)
    s = bound(tensors)

    class Elsewhere:
        cuda_stream, device = 0x1234, torch.device("cuda", 7)

    for _ in range(2):
        with pytest.raises(ValueError):
            s.launch(Elsewhere())
    s.close()


def test_streams_that_end_before_the_session():
    """The allocator is not told of streams that their owner destroys, the session's own among them."""
    tensors, want = attention(2)
    torch.cuda.synchronize()
    for foreign in (lambda s: s.make_streams(1).torch_streams[0], lambda s: torch.cuda.ExternalStream(s.make_streams(2).handles[1])):
        s = bound(tensors)
        stream = foreign(s)
        assert stream.stream_id == stream.cuda_stream != 0
        s.launch(stream)
        with torch.cuda.stream(stream):                        # as the current stream it is another object
            assert torch.cuda.current_stream().stream_id == stream.stream_id
            s.launch()
        torch.cuda.synchronize()
        D.within(s.result(0), *want, "f16")
        s.close()
        del s, stream
        fresh = [torch.empty(n, device=DEV) for n in (64, 1 << 20, 1 << 24)]
        del fresh
        torch.cuda.empty_cache()
    pool, default = torch.cuda.Stream(), torch.cuda.default_stream()
    assert pool.stream_id != pool.cuda_stream and default.stream_id == 0
