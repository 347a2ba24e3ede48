"""A NaN key in a page's bounds, and in the choice of pages."""
import math

import pytest

import paged_ref as ref
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, attend, bounds_of, check_selection, f64, params, queries, selection, wanted

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("page,half,rotate,at_once", [(16, False, False, True), (64, True, True, True), (128, False, True, False), (32, True, False, False)])
def test_bounds_take_a_nan_key_in(page, half, rotate, at_once):
    """The dimensions in which a key is NaN have NaN bounds, the others the smallest and largest key, however the tokens came."""
    p = params(2, 1, page, 64, half, rotate, bounds=True)
    c = Cache(p, [0], seed=page, room=3 * page)
    n = 2 * page + 5
    k, v = c.rows(n)
    k[0, 3, 0, 7] = math.nan  # one key of the first page
    k[0, page - 1, 0, 90] = math.nan
    k[0, 2 * page, 1, :] = math.nan  # the first of the third, in the other head
    for a, b in ((0, n),) if at_once else ((0, 2), (2, 4), (4, page + 3), (page + 3, n)):
        akv.akv_paged_append(p, c.pages, k[:, a:b], v[:, a:b])
        c.lens += b - a
    c.lens_h = [n]
    for h in range(2):
        got = torch.from_numpy(bounds_of(c, 0, h)).cuda()
        for j in range(3):
            x = k[0, j * page : min(n, (j + 1) * page), h].double()
            want = torch.stack((x.amin(0), x.amax(0)))  # (pass a NaN on)
            assert torch.equal(got[j].nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0)), (h, j)
    # a page's first slot written again: nothing of the NaN stays
    c.lens.zero_()
    k2, v2 = c.rows(page)
    akv.akv_paged_append(p, c.pages, k2, v2)
    c.lens.fill_(page)
    c.lens_h = [page]
    for h in range(2):
        x = k2[0, :, h].double()
        assert torch.equal(torch.from_numpy(bounds_of(c, 0, h)).cuda()[0], torch.stack((x.amin(0), x.amax(0))))


@pytest.mark.parametrize("half", [False, True])
def test_a_page_with_a_nan_key_is_kept(half):
    """Its score is +infinity, as with an infinite key: the queries that would have seen the NaN do."""
    p = params(1, 2, 16, 64, half, False, bounds=True)
    c = Cache(p, [40 * 16], seed=5)
    k, v = c.rows(640)
    k[0, 16 * 21 + 4] *= 1e-3  # not one that its score would keep
    k[0, 16 * 21 : 16 * 22] *= 1e-3
    k[0, 16 * 21 + 4, 0, 9] = math.nan
    akv.akv_paged_append(p, c.pages, k, v)
    c.lens.fill_(640)
    q = queries(c, 1)
    sel = selection(c, 1, 5)
    akv.akv_paged_select(p, c.pages, q, sel)
    want = wanted(c, q, 1, 5, 1, 1)
    assert 21 in want[0][0][0]
    check_selection(sel, want)
    out, lse = attend(c, q, sel=sel)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())
