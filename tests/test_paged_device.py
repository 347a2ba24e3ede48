"""The device that the paged cache's calls launch on: the pool's, whichever is current.  Two devices made up on the host."""
import contextlib
import types

import pytest

import paper_2608_02901_gb300 as akv
from paper_2608_02901_gb300 import paged

torch = pytest.importorskip("torch")

POOLS = 1  # the pool's device; device 0 is the current one


class Tensor:
    """What the binding asks of a CUDA tensor on the pool's device."""
    device = types.SimpleNamespace(index=POOLS)
    nbytes = 1 << 40

    def __init__(self, *shape, dtype=torch.int32):
        self.shape, self.dtype = shape, dtype

    def get_device(self):
        return POOLS

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def stride(self):
        out = [1]
        for x in self.shape[:0:-1]:
            out.insert(0, out[0] * x)
        return out


@pytest.fixture
def devices(monkeypatch):
    """A library that notes the current device of each entry, and torch's calls that change it."""
    state = types.SimpleNamespace(current=0, calls=[])

    @contextlib.contextmanager
    def device(i):
        was, state.current = state.current, i
        yield
        state.current = was

    def raw_stream(i):
        return 1000 + i

    class Lib:
        def __getattr__(self, name):
            def entry(*args):
                state.calls.append((name, state.current, args[-1]))
                return 0
            return entry

    monkeypatch.setattr(paged, "_loaded", Lib())
    monkeypatch.setattr(paged, "_torch", types.SimpleNamespace(cuda=types.SimpleNamespace(device=device), float32=torch.float32))
    monkeypatch.setattr(paged, "_raw_stream", raw_stream)
    monkeypatch.setattr(paged, "_device", lambda: state.current, raising=False)
    monkeypatch.setattr(paged, "_int32", torch.int32)
    monkeypatch.setattr(paged, "_bf16", torch.bfloat16)
    return state


def calls(stream=None):
    """Every entry point that launches, on a pool of the second device."""
    p = akv.PagedParams(2, 8, 32, bounds=True)
    params, ref = p.c(), object()
    pages = types.SimpleNamespace(p=p, index=POOLS, device="cuda:1", rows=3, pref=params, ref=ref)
    kv, q = (Tensor(3, 2, h, 128, dtype=torch.bfloat16) for h in (2, 8))
    ints, one, ws = Tensor(3), Tensor(1), Tensor(4096)
    sel = types.SimpleNamespace(pages=types.SimpleNamespace(device="cuda:1"), count=Tensor(3, 2, 2), top=4, ref=ref)
    return [
        lambda: akv.akv_paged_append(p, pages, kv, kv, n_new=ints, stream=stream),
        lambda: akv.akv_paged_read(p, pages, kv, kv, start=ints, stream=stream),
        lambda: akv.akv_paged_attn(p, pages, q, q, lse=Tensor(3, 2, 8, dtype=torch.float32), ws=ws, stream=stream),
        lambda: akv.akv_paged_select(p, pages, q, sel, ws=ws, stream=stream),
        lambda: akv.akv_pages_copy(p, pages, ints, ints, stream=stream),
        lambda: akv.akv_pages_fork(p, pages, ints, ints, stream=stream),
        lambda: akv.akv_pages_reserve(p, pages, ints, one, ws=ws, stream=stream),
        lambda: akv.akv_pages_free(p, pages, ints, stream=stream),
        lambda: akv.akv_pages_compact(p, pages, one, ws=ws, stream=stream),
    ]


@pytest.mark.parametrize("i", range(9))
def test_calls_launch_on_the_pools_device(devices, i):
    for stream, handle in ((None, 1000 + POOLS), (77, 77), (types.SimpleNamespace(cuda_stream=78, device_index=POOLS), 78)):
        calls(stream)[i]()
        assert devices.calls[-1][1:] == (POOLS, handle), devices.calls
    assert devices.current == 0
    devices.current = POOLS
    calls()[i]()
    assert devices.calls[-1][1:] == (POOLS, 1000 + POOLS) and devices.current == POOLS


@pytest.mark.parametrize("i", range(9))
def test_streams_of_another_device_are_refused(devices, i):
    with pytest.raises(ValueError, match="stream"):
        calls(types.SimpleNamespace(cuda_stream=78, device_index=0))[i]()
    assert not devices.calls


@pytest.mark.gpu
def test_streams_have_a_device():
    """What the refusal looks at, of torch's own streams."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    side = torch.cuda.Stream()
    assert side.device_index == 0
    assert torch.cuda.ExternalStream(side.cuda_stream).device_index == 0
    assert torch.cuda.current_stream().device_index == 0
