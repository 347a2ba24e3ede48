"""Shared-prefix attention, weights, eviction and trimming launch on the pool's device, on the stream that they are given."""
import types

import pytest

import paper_2608_02901_gb300 as akv
from test_paged_device import POOLS, Tensor, devices  # noqa: F401 - the fixture

torch = pytest.importorskip("torch")


def calls(stream=None):
    p = akv.PagedParams(2, 8, 32)
    params, ref = p.c(), object()
    pages = types.SimpleNamespace(p=p, index=POOLS, device="cuda:1", rows=3, pref=params, ref=ref)
    q, lse, ints, ws = Tensor(3, 2, 8, 128, dtype=torch.bfloat16), Tensor(3, 2, 8, dtype=torch.float32), Tensor(3), Tensor(4096)
    scores = Tensor(3, 2, 64, dtype=torch.float32)
    share = types.SimpleNamespace(index=POOLS, ref=ref, rows=3)
    kept = types.SimpleNamespace(tokens=types.SimpleNamespace(device="cuda:1", shape=(3, 2, 4)), count=Tensor(3), top=4, ref=ref)
    return [
        lambda: akv.akv_pages_share(p, pages, share, ws=ws, stream=stream),
        lambda: akv.akv_paged_attn_shared(p, pages, q, q, share, lse=lse, ws=ws, stream=stream),
        lambda: akv.akv_paged_weights(p, pages, q, lse, scores, was=scores, ws=ws, stream=stream),
        lambda: akv.akv_paged_evict(p, pages, ints, ints, scores, kept, keep=ints, stream=stream),
        lambda: akv.akv_pages_trim(p, pages, ints, stream=stream),
    ]


@pytest.mark.parametrize("i", range(5))
def test_calls_launch_on_the_pools_device(devices, i):  # noqa: F811
    for stream, handle in ((None, 1000 + POOLS), (77, 77), (types.SimpleNamespace(cuda_stream=78, device_index=POOLS), 78)):
        calls(stream)[i]()
        assert devices.calls[-1][1:] == (POOLS, handle), devices.calls
    assert devices.current == 0


@pytest.mark.parametrize("i", range(5))
def test_streams_of_another_device_are_refused(devices, i):  # noqa: F811
    with pytest.raises(ValueError, match="stream"):
        calls(types.SimpleNamespace(cuda_stream=78, device_index=0))[i]()
    assert not devices.calls
