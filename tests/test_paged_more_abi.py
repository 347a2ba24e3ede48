"""Refusals and sizes of shared attention, accumulated weights, eviction and trimming through the C ABI: no GPU, no launch is reached."""
import ctypes

import pytest

import paper_2608_02901_gb300 as akv
from paper_2608_02901_gb300 import paged
from test_paged_abi import AT, INVALID, OK, PAGES, PARAMS, TOO_SMALL, UNSUPPORTED, call, pages, params, refused, rows

WS = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2608_02901_gb300 import build
    build.build()


def share(**kw):
    c = paged._Share(AT, AT, AT, AT)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def scores(**kw):
    c = paged._Scores(AT, 2 * 160, 160, 160)  # 5 rows of 5 pages of 32 tokens, 2 heads
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def kept(**kw):
    c = paged._Kept(AT, AT, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def plain(**kw):
    return params(flags=akv.AKV_FLAG_ROTATE, **kw)


def pages_(**kw):
    size = akv.akv_paged_page_bytes(akv.PagedParams(2, 8, 32))
    return pages(**{"pool_bytes": 2 * 10 * size, "layer_stride": 10 * size, **kw})


def attn(p=None, g=None, layer=0, q=None, out=None, lse=None, T=1, sm=1.0, sh=share, ws=AT, n=WS):
    return ("akv_paged_attn_shared", p or params(), g or pages(), layer, q or rows(), out or rows(), lse, T, sm, sh() if sh else None, ws, n, None)


def weights(p=None, g=None, layer=0, q=None, lse=AT, T=1, sm=1.0, decay=1.0, was=None, now=scores, ws=AT, n=WS):
    return ("akv_paged_weights", p or params(), g or pages(), layer, q or rows(), lse, T, sm, decay, was() if was else None, now() if now else None,
            ws, n, None)


def evict(p=None, g=None, layer=0, src=AT, dst=AT, n=2, sc=scores, keep=None, sink=1, recent=1, k=kept):
    return ("akv_paged_evict", p or plain(), g or pages_(), layer, src, dst, n, sc() if sc else None, keep, sink, recent, k() if k else None, None)


@pytest.mark.parametrize("change,status,text", PARAMS)
def test_parameters(change, status, text):
    for make in (attn, weights, evict):
        refused(status, text, *make(p=params(**change)))
    refused(status, text, "akv_pages_trim", params(**change), pages(), AT, 1, None)
    refused(status, text, "akv_pages_share", params(**change), pages(), share(), AT, WS, None)


@pytest.mark.parametrize("change,status,text", PAGES)
def test_pages(change, status, text):
    for make in (attn, weights):
        refused(status, text, *make(g=pages(**change)))
    refused(status, text, "akv_pages_trim", params(), pages(**change), AT, 1, None)
    refused(status, text, "akv_pages_share", params(), pages(**change), share(), AT, WS, None)


def test_layers():
    for layer in (-1, 2):
        for make in (attn, weights, evict):
            refused(INVALID, "layer", *make(layer=layer))


def test_share():
    for field in ("leader", "pages", "size", "order"):
        for at, text in ((None, "null share"), (AT + 2, "4-byte")):
            refused(INVALID, text, "akv_pages_share", params(), pages(), share(**{field: at}), AT, WS, None)
            refused(INVALID, text, *attn(sh=lambda: share(**{field: at})))
    refused(INVALID, "null share", "akv_pages_share", params(), pages(), None, AT, WS, None)
    refused(INVALID, "null share", *attn(sh=None))
    many = pages(rows=(1 << 16) + 1)
    refused(UNSUPPORTED, "2^16 rows", "akv_pages_share", params(), many, share(), AT, WS, None)
    refused(UNSUPPORTED, "2^16 rows", *attn(g=many, out=rows(stride_b=1 << 20)))
    size = ctypes.c_size_t()
    assert call("akv_pages_workspace_size", params(), pages(), ctypes.byref(size)) == OK
    refused(TOO_SMALL, "workspace", "akv_pages_share", params(), pages(), share(), AT, size.value - 1, None)
    for ws in (None, AT + 16):
        refused(INVALID, "workspace", "akv_pages_share", params(), pages(), share(), ws, WS, None)


def test_shared_attention():
    for T in (0, 65, -1):
        refused(UNSUPPORTED, "query tokens", *attn(T=T))
        refused(UNSUPPORTED, "query tokens", "akv_paged_attn_shared_workspace_size", params(), pages(), T, ctypes.byref(ctypes.c_size_t()))
    refused(INVALID, "null ws_bytes", "akv_paged_attn_shared_workspace_size", params(), pages(), 1, None)
    refused(INVALID, "null q", *attn(q=rows(ptr=None)))
    refused(INVALID, "q must be 2-byte", *attn(q=rows(ptr=AT + 1)))
    refused(INVALID, "out: rows overlap", *attn(out=rows(stride_h=64)))
    refused(INVALID, "lse", *attn(lse=AT + 2))
    for sm in (float("nan"), float("inf")):
        refused(INVALID, "sm_scale", *attn(sm=sm))
    size = ctypes.c_size_t()
    assert call("akv_paged_attn_shared_workspace_size", params(), pages(), 3, ctypes.byref(size)) == OK
    refused(TOO_SMALL, "workspace", *attn(T=3, n=size.value - 1))
    for ws in (None, AT + 8):
        refused(INVALID, "workspace", *attn(ws=ws))


def test_weights():
    for T in (0, 65):
        refused(UNSUPPORTED, "query tokens", *weights(T=T))
    refused(INVALID, "null lse", *weights(lse=None))
    refused(INVALID, "lse must be", *weights(lse=AT + 1))
    refused(INVALID, "null now", *weights(now=None))
    for bad in (float("nan"), float("-inf")):
        refused(INVALID, "sm_scale", *weights(sm=bad))
        refused(INVALID, "decay", *weights(decay=bad))
    for who in ("was", "now"):
        given = lambda **kw: {who: lambda: scores(**kw)}  # noqa: E731
        refused(INVALID, "null " + who, *weights(**given(ptr=None)))
        refused(INVALID, who + " must be 4-byte", *weights(**given(ptr=AT + 2)))
        refused(TOO_SMALL, who + ": room", *weights(**given(cap=159)))
        refused(INVALID, who + ": negative", *weights(**given(stride_b=-1)))
    for kw in (dict(stride_h=159), dict(stride_b=319), dict(stride_b=0), dict(stride_h=0)):
        refused(INVALID, "now: heads' numbers overlap", *weights(now=lambda: scores(**kw)))
    refused(INVALID, "out of range", *weights(now=lambda: scores(stride_b=2**61)))
    size = ctypes.c_size_t()
    for T in (1, 9):
        assert call("akv_paged_weights_workspace_size", params(), pages(), T, ctypes.byref(size)) == OK
        refused(TOO_SMALL, "workspace", *weights(T=T, n=size.value - 1))
    for ws in (None, AT + 8):
        refused(INVALID, "workspace", *weights(ws=ws))
    refused(UNSUPPORTED, "query tokens", "akv_paged_weights_workspace_size", params(), pages(), 0, ctypes.byref(size))
    refused(INVALID, "null ws_bytes", "akv_paged_weights_workspace_size", params(), pages(), 1, None)


def test_evict():
    refused(UNSUPPORTED, "bounds", *evict(p=params(), g=pages()))
    refused(INVALID, "null list", *evict(src=None))
    refused(INVALID, "null list", *evict(dst=None))
    refused(INVALID, "lists must be", *evict(src=AT + 2))
    refused(INVALID, "negative count", *evict(n=-1))
    refused(UNSUPPORTED, "too many", *evict(n=1 << 22))
    refused(INVALID, "null scores", *evict(sc=None))
    refused(TOO_SMALL, "scores: room", *evict(sc=lambda: scores(cap=100)))
    refused(INVALID, "overlap", *evict(sc=lambda: scores(stride_h=1)))
    refused(INVALID, "keep must be", *evict(keep=AT + 1))
    for kw in (dict(sink=-1), dict(recent=-1)):
        refused(INVALID, "sink and recent", *evict(**kw))
    refused(INVALID, "null kept", *evict(k=None))
    for kw, text in ((dict(tokens=None), "null kept"), (dict(count=None), "null kept"), (dict(tokens=AT + 2), "kept must be"),
                     (dict(top=0), "top"), (dict(top=2**30 + 1), "top")):
        refused(INVALID, text, *evict(k=lambda: kept(**kw)))
    name, *args = evict(src=None, dst=None, n=0, k=lambda: kept(tokens=None, count=None))
    assert call(name, *args) == OK


def test_trim():
    refused(INVALID, "null refs", "akv_pages_trim", params(), pages(refs=None), AT, 1, None)
    refused(INVALID, "null list", "akv_pages_trim", params(), pages(), None, 1, None)
    refused(INVALID, "negative", "akv_pages_trim", params(), pages(), AT, -1, None)
    refused(INVALID, "4-byte", "akv_pages_trim", params(), pages(), AT + 2, 1, None)
    assert call("akv_pages_trim", params(), pages(), None, 0, None) == OK


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for arrays in (i32(4), i32(3, 5), i32(4, 5, 1)):
        with pytest.raises(ValueError, match="share"):
            akv.PageShare(arrays)
    with pytest.raises(ValueError, match="device"):
        akv.PageShare(i32(4, 5))
    with pytest.raises(ValueError, match="int32"):
        akv.PageShare(torch.zeros((4, 5)))
    for tokens, count in ((i32(2, 3), i32(2)), (i32(2, 3, 4), i32(3)), (i32(2, 3, 4), i32(2, 3))):
        with pytest.raises(ValueError, match="kept"):
            akv.KeptTokens(tokens, count)
    with pytest.raises(ValueError, match="contiguous"):
        akv.KeptTokens(i32(2, 4, 3).transpose(1, 2), i32(2))


def test_share_flags():
    for flags in (2, 1 << 31, 3):
        refused(INVALID, "flags", "akv_pages_share", params(), pages(), share(flags=flags), AT, WS, None)
        refused(INVALID, "flags", *attn(sh=lambda: share(flags=flags)))
