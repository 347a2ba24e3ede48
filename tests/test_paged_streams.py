"""Streams of the paged cache's binding: whose memory a workspace is that the call takes for itself."""
import contextlib
import types

import pytest

import paper_2608_02901_gb300 as akv
from paper_2608_02901_gb300 import paged

torch = pytest.importorskip("torch")


class FakeTorch:
    """What the binding uses of torch to make a workspace: notes the stream that is current when memory is asked for."""
    uint8 = "uint8"

    def __init__(self):
        self.current, self.asked = "current", []
        self.cuda = types.SimpleNamespace(stream=self.stream, ExternalStream=lambda ptr, device=None: types.SimpleNamespace(cuda_stream=ptr))

    @contextlib.contextmanager
    def stream(self, s):
        was, self.current = self.current, s.cuda_stream
        yield
        self.current = was

    def empty(self, n, dtype, device):
        self.asked.append((n, self.current, device))
        return types.SimpleNamespace(data_ptr=lambda: 4096, nbytes=n, record_stream=lambda s: None)


@pytest.mark.parametrize("stream,owner", [(None, "current"), (types.SimpleNamespace(cuda_stream=77), 77), (91, 91), (0, 0)])
def test_a_workspace_belongs_to_the_stream_that_uses_it(monkeypatch, stream, owner):
    """Blocks that torch's allocator gets back go to later calls of the stream they were asked for on, and of no other."""
    fake = FakeTorch()
    monkeypatch.setattr(paged, "_torch", fake)
    pages = types.SimpleNamespace(index=0, device="cuda:0")
    _, at, n = paged._workspace(None, pages, stream, lambda x: x + 1, 300)
    assert (at, n) == (4096, 301) and fake.asked == [(301, owner, "cuda:0")]
    assert fake.current == "current"


@pytest.mark.gpu
def test_calls_on_streams_that_run_together():
    """Attention, selection and reservation without a workspace of the caller's, on the current and two other streams in turn
    and with nothing between them: what they give one after another, they give together."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from test_paged_cache import Cache, params, queries, selection
    from test_pages import Gpu, filled, ints

    p = params(4, 8, 64, 64, False, True, bounds=True)
    c = Cache(p, [20000, 9001, 777], seed=31)
    c.fill()
    side = [torch.cuda.Stream() for _ in range(2)]
    streams = [None, side[0], side[1].cuda_stream]  # (a handle will do)
    n = 30
    qs = [queries(c, 1) for _ in range(n)]
    sels = [selection(c, 1, 40) for _ in range(n)]
    sims = [filled(6, 40, 300, 16, 1, [16 * (5 + i), 100, 3 * i + 1], seed=i) for i in range(n)]
    for s in sims:
        s.fork([(0, 3), (1, 4), (2, 5)])

    def calls(which):
        states = [Gpu(s) for s in sims]
        new = ints([1, 40, 5, 17, 2, 1])
        outs = [torch.zeros_like(q) for q in qs]
        lses = [torch.zeros(q.shape[:3], device="cuda") for q in qs]
        kept = [torch.zeros_like(q) for q in qs]
        torch.cuda.synchronize()
        for i in range(n):
            at = which(i)
            akv.akv_paged_attn(p, c.pages, qs[i], outs[i], lse=lses[i], sm_scale=0.1, stream=at)
            akv.akv_paged_select(p, c.pages, qs[i], sels[i], stream=at)
            akv.akv_paged_attn(p, c.pages, qs[i], kept[i], sel=sels[i], sm_scale=0.1, stream=at)
            akv.akv_pages_reserve(states[i].p, states[i].pages, new, states[i].one, stream=at)
        torch.cuda.synchronize()
        return [t.clone() for g in states for t in (g.table, g.refs, g.pool, g.one)], outs, lses, kept, [t.clone() for s in sels for t in (s.pages, s.count)]

    want = calls(lambda i: None)
    for _ in range(3):
        got = calls(lambda i: streams[i % 3])
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
