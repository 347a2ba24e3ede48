"""Refusals and sizes of the paged cache's entry points, through the C ABI: no GPU is needed, no launch is reached."""
import ctypes
import os

import pytest

import paged_ref as ref
import paper_2608_02901_gb300 as akv
from paper_2608_02901_gb300 import paged

OK, INVALID, UNSUPPORTED, TOO_SMALL = akv.AKV_OK, akv.AKV_ERR_INVALID, akv.AKV_ERR_UNSUPPORTED, akv.AKV_ERR_TOO_SMALL
AT = 1 << 20  # an address that nothing reads


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2608_02901_gb300 import build
    build.build()


def params(**kw):
    c = akv.PagedParams(n_kv_heads=2, n_q_heads=8, page_tokens=32, group=64, rotate=True, bounds=True).c()
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def pages(p=None, **kw):
    size = akv.akv_paged_page_bytes(akv.PagedParams(2, 8, 32, bounds=True))
    c = paged._Pages(AT, 2 * 10 * size, 10 * size, 2, 10, AT, 5, 3, 5, AT, AT)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    c = paged._Rows(AT, 4096, 1024, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def sel(**kw):
    c = paged._Selection(AT, AT, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def ref_(x):
    return None if x is None else ctypes.byref(x)


def call(name, *args):
    return getattr(akv.lib(), name)(*[ref_(a) if isinstance(a, ctypes.Structure) else a for a in args])


def refused(status, text, name, *args):
    assert call(name, *args) == status
    assert text in akv.akv_last_error(), akv.akv_last_error()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("bounds", [False, True])
def test_page_bytes(page, group, bounds):
    p = akv.PagedParams(n_kv_heads=3, n_q_heads=3, page_tokens=page, group=group, bounds=bounds)
    assert akv.akv_paged_page_bytes(p) == 3 * ref.block_bytes(p)


PARAMS = [
    (dict(head_dim=64), UNSUPPORTED, "head_dim"), (dict(n_kv_heads=0), INVALID, "n_kv_heads"), (dict(n_q_heads=0), INVALID, "n_q_heads"),
    (dict(n_q_heads=7), INVALID, "multiple"), (dict(n_kv_heads=257, n_q_heads=257), UNSUPPORTED, "256"),
    (dict(n_q_heads=130), UNSUPPORTED, "64 query heads"), (dict(page_tokens=48), UNSUPPORTED, "page_tokens"),
    (dict(page_tokens=0), UNSUPPORTED, "page_tokens"), (dict(page_tokens=256), UNSUPPORTED, "page_tokens"),
    (dict(group=32), UNSUPPORTED, "group"), (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(flags=2), INVALID, "flags"),
    (dict(reserved=1), INVALID, "reserved"),
]


@pytest.mark.parametrize("change,status,text", PARAMS)
def test_parameters(change, status, text):
    size = ctypes.c_size_t()
    refused(status, text, "akv_paged_page_bytes", params(**change), ctypes.byref(size))
    refused(status, text, "akv_paged_attn", params(**change), pages(), 0, rows(), rows(), None, 1, 1.0, None, AT, 1 << 40, None)
    refused(status, text, "akv_pages_free", params(**change), pages(), AT, 1, None)


PAGES = [
    (dict(pool=None), INVALID, "null pool"), (dict(table=None), INVALID, "table"), (dict(lens=None), INVALID, "lens"),
    (dict(pool=AT + 8), INVALID, "16-byte"), (dict(table=AT + 2), INVALID, "4-byte"), (dict(lens=AT + 1), INVALID, "4-byte"),
    (dict(refs=AT + 1), INVALID, "4-byte"), (dict(n_layers=0), INVALID, "n_layers"), (dict(n_pages=0), INVALID, "n_pages"),
    (dict(rows=0), INVALID, "rows"), (dict(max_pages=0), INVALID, "max_pages"), (dict(table_stride=4), INVALID, "table_stride"),
    (dict(pool_bytes=100), TOO_SMALL, "pool"), (dict(layer_stride=8), INVALID, "layer_stride"),
    (dict(n_layers=2**31 - 1, layer_stride=2**62), INVALID, "layer_stride"),
    (dict(max_pages=1 << 26, table_stride=1 << 26), UNSUPPORTED, "2^30"), (dict(rows=1 << 22), UNSUPPORTED, "requests"),
    (dict(rows=1 << 20, max_pages=1 << 12, table_stride=1 << 12), UNSUPPORTED, "2^31"),
]


@pytest.mark.parametrize("change,status,text", PAGES)
def test_pages(change, status, text):
    refused(status, text, "akv_paged_append", params(), pages(**change), 0, rows(), rows(), 1, None, None)
    refused(status, text, "akv_pages_copy", params(), pages(**change), AT, AT, 1, None)


def test_null_structures():
    size = ctypes.c_size_t()
    refused(INVALID, "null params", "akv_paged_page_bytes", None, ctypes.byref(size))
    refused(INVALID, "null bytes", "akv_paged_page_bytes", params(), None)
    refused(INVALID, "null pages", "akv_paged_read", params(), None, 0, None, rows(), rows(), 1, None)
    refused(INVALID, "null K", "akv_paged_append", params(), pages(), 0, None, rows(), 1, None, None)
    refused(INVALID, "null V", "akv_paged_append", params(), pages(), 0, rows(), rows(ptr=None), 1, None, None)
    refused(INVALID, "null ws_bytes", "akv_pages_workspace_size", params(), pages(), None)


def test_append_and_read():
    for layer in (-1, 2):
        refused(INVALID, "layer", "akv_paged_append", params(), pages(), layer, rows(), rows(), 1, None, None)
    refused(INVALID, "negative T", "akv_paged_append", params(), pages(), 0, rows(), rows(), -1, None, None)
    refused(INVALID, "2-byte", "akv_paged_append", params(), pages(), 0, rows(ptr=AT + 1), rows(), 1, None, None)
    refused(INVALID, "negative stride", "akv_paged_append", params(), pages(), 0, rows(), rows(stride_h=-128), 1, None, None)
    refused(INVALID, "n_new", "akv_paged_append", params(), pages(), 0, rows(), rows(), 1, AT + 2, None)
    refused(INVALID, "overlap", "akv_paged_read", params(), pages(), 0, None, rows(), rows(stride_t=0), 2, None)
    refused(INVALID, "overlap", "akv_paged_read", params(), pages(), 0, None, rows(stride_b=64), rows(), 1, None)
    refused(INVALID, "start", "akv_paged_read", params(), pages(), 0, AT + 1, rows(), rows(), 1, None)
    assert call("akv_paged_append", params(), pages(), 0, rows(), rows(), 0, None, None) == OK
    assert call("akv_paged_read", params(), pages(), 1, None, rows(), rows(), 0, None) == OK
    assert call("akv_paged_append", params(), pages(), 0, rows(ptr=None), rows(ptr=None), 0, None, None) == OK
    assert call("akv_paged_read", params(), pages(), 0, None, rows(ptr=None), rows(ptr=None), 0, None) == OK


def test_attention():
    size = ctypes.c_size_t()
    assert call("akv_paged_attn_workspace_size", params(), pages(), 1, 0, ctypes.byref(size)) == OK and size.value > 0

    def attn(p=None, g=None, q=None, out=None, lse=None, T=1, sm=1.0, s=None, ws=AT, n=1 << 40):
        return "akv_paged_attn", p or params(), g or pages(), 0, q or rows(), out or rows(), lse, T, sm, s, ws, n, None

    refused(UNSUPPORTED, "query tokens", *attn(T=0))
    refused(UNSUPPORTED, "query tokens", *attn(T=65))
    refused(INVALID, "finite", *attn(sm=float("nan")))
    refused(INVALID, "finite", *attn(sm=float("inf")))
    refused(INVALID, "null q", *attn(q=rows(ptr=None)))
    refused(INVALID, "null out", *attn(out=rows(ptr=None)))
    refused(INVALID, "overlap", *attn(out=rows(stride_h=0)))
    refused(INVALID, "lse", *attn(lse=AT + 2))
    refused(INVALID, "workspace", *attn(ws=None))
    refused(INVALID, "workspace", *attn(ws=AT + 16))
    refused(TOO_SMALL, "workspace", *attn(n=size.value - 1))
    refused(INVALID, "selection", *attn(s=sel(pages=None)))
    refused(INVALID, "selection", *attn(s=sel(count=AT + 1)))
    refused(INVALID, "top", *attn(s=sel(top=0)))
    refused(UNSUPPORTED, "query tokens", "akv_paged_attn_workspace_size", params(), pages(), 0, 0, ctypes.byref(size))
    refused(INVALID, "top", "akv_paged_attn_workspace_size", params(), pages(), 1, -1, ctypes.byref(size))


def test_selection():
    size = ctypes.c_size_t()
    assert call("akv_paged_select_workspace_size", params(), pages(), 3, ctypes.byref(size)) == OK and size.value > 0

    def select(p=None, g=None, q=None, T=3, sink=1, recent=1, s=None, ws=AT, n=1 << 40):
        return "akv_paged_select", p or params(), g or pages(), 0, q or rows(), T, sink, recent, s or sel(), ws, n, None

    plain = params(flags=1)
    refused(INVALID, "bounds", *select(p=plain))
    refused(INVALID, "sink", *select(sink=-1))
    refused(INVALID, "sink", *select(recent=-1))
    refused(INVALID, "sink", *select(sink=3, recent=2))
    refused(INVALID, "sink", *select(sink=2**31 - 1, recent=2**31 - 1))
    refused(INVALID, "top", *select(s=sel(top=0)))
    refused(INVALID, "null q", *select(q=rows(ptr=None)))
    refused(TOO_SMALL, "workspace", *select(n=size.value - 1))
    refused(INVALID, "null selection", "akv_paged_select", params(), pages(), 0, rows(), 1, 1, 1, None, AT, 1 << 40, None)


def test_page_operations():
    size = ctypes.c_size_t()
    assert call("akv_pages_workspace_size", params(), pages(), ctypes.byref(size)) == OK and size.value > 0
    none = pages(refs=None)
    refused(INVALID, "null refs", "akv_pages_fork", params(), none, AT, AT, 1, None)
    refused(INVALID, "null refs", "akv_pages_free", params(), none, AT, 1, None)
    refused(INVALID, "null refs", "akv_pages_reserve", params(), none, AT, AT, AT, 1 << 40, None)
    refused(INVALID, "null refs", "akv_pages_compact", params(), none, AT, AT, 1 << 40, None)
    refused(INVALID, "negative", "akv_pages_copy", params(), none, AT, AT, -1, None)
    refused(INVALID, "null list", "akv_pages_fork", params(), pages(), None, AT, 1, None)
    refused(INVALID, "aligned", "akv_pages_free", params(), pages(), AT + 2, 1, None)
    refused(INVALID, "n_new", "akv_pages_reserve", params(), pages(), None, AT, AT, 1 << 40, None)
    refused(INVALID, "missing", "akv_pages_reserve", params(), pages(), AT, None, AT, 1 << 40, None)
    refused(INVALID, "n_live", "akv_pages_compact", params(), pages(), None, AT, 1 << 40, None)
    refused(TOO_SMALL, "workspace", "akv_pages_reserve", params(), pages(), AT, AT, AT, size.value - 1, None)
    refused(TOO_SMALL, "workspace", "akv_pages_compact", params(), pages(), AT, AT, size.value - 1, None)
    for name, args in (("akv_pages_copy", (AT, AT, 0)), ("akv_pages_fork", (AT, AT, 0)), ("akv_pages_free", (AT, 0))):
        assert call(name, params(), pages(), *args, None) == OK


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    p = akv.PagedParams(2, 8, 32)
    pool = torch.zeros((1, 4, akv.akv_paged_page_bytes(p)), dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        akv.Pages(p, pool, torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_every_entry_point_is_in_the_package():
    for name in paged.EXPORTED:
        assert callable(getattr(akv, name)) and hasattr(akv.lib(), name)
    assert os.path.exists(akv.LIB_PATH)


def test_written_rows_may_lie_in_any_order_but_not_on_top_of_one_another():
    """[rows][T][heads] = 3 x 4 x 2 rows of 128, T = 4."""
    def read(K, T=4):
        return "akv_paged_read", params(), pages(), 0, None, K, rows(), T, None

    # two heads 128 apart step over 256 values, four tokens of them over 1024
    for b, t, h in ((1024, 256, 64), (1024, 192, 128), (960, 256, 128), (128, 128, 128), (512, 256, 128), (256, 700, 128),
                    (256, 128, 512), (128, 4096, 300), (0, 256, 128), (2**62, 2**62, 2**61)):
        assert call(*read(rows(stride_b=b, stride_t=t, stride_h=h))) == INVALID, (b, t, h)
    refused(INVALID, "overlap", *read(rows(stride_b=896, stride_t=256, stride_h=128)))
    refused(INVALID, "out of range", *read(rows(stride_b=2**62, stride_t=256, stride_h=128)))
    refused(UNSUPPORTED, "2^30", *read(rows(), T=2**30 + 1))
