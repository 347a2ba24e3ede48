"""Attention of queries of any size: large rows beside small ones, rows that are no numbers."""
import math

import pytest

import paged_exact as exact
from test_paged_cache import Cache, attend, params, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def filled(G, rotate, lens=(300, 64, 1), half=False):
    c = Cache(params(1, G, 32, 64, half, rotate), list(lens), seed=G)
    c.fill()
    return c


def check_rows(c, q, out, lse, sm, rows):
    """The query heads `rows` (a mask [B][T][Hq]) against the 64-bit form."""
    want, want_lse, tol, tol_lse = exact.Exact(c.p, c.pool[0], c.table, c.lens.tolist()).attend(q.nan_to_num(0, 0, 0), sm)
    share = ((out.double() - want).abs() / tol)[rows]
    assert bool((share <= 1).all()), float(share.max())
    assert bool(((lse.double() - want_lse).abs()[rows] <= tol_lse[rows]).all())


@pytest.mark.parametrize("G,T,rotate", [(4, 1, False), (8, 1, True), (4, 4, True), (3, 5, False)])
@pytest.mark.parametrize("factor", [2.0**20, 1e9, 1e20, 1e30])
def test_large_rows_beside_others(G, T, rotate, factor):
    """As rows that pad a batch may be, filled with anything: the other rows of the KV head are what they are without them."""
    c = filled(G, rotate, (300, 64, 9))
    q = queries(c, T)
    alone = attend(c, q)
    big = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
    big[:, 0, 1] = True
    big[1, -1, G - 1] = True
    q[big] = (q[big].float() * factor).to(q.dtype)
    out, lse = attend(c, q)
    check_rows(c, q, out, lse, 1 / math.sqrt(D), ~big)
    check_rows(c, q, *alone, 1 / math.sqrt(D), ~big)


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("e", [99, 110, 124, -60, -110])
def test_large_and_small_queries_with_a_scale_to_match(e, rotate):
    """q of 2^e and a scale of 2^-e."""
    c = filled(4, rotate)
    q = (queries(c, 1, 1.0).float() / (4 if e > 120 else 1) * 2.0**e).to(torch.bfloat16)
    sm = 2.0**-e / math.sqrt(D)
    exact.check(c.p, c, q, *attend(c, q, sm_scale=sm), sm)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("G,T,rotate", [(4, 1, False), (4, 4, True)])
def test_rows_that_are_no_numbers_spoil_themselves(bad, G, T, rotate):
    c = filled(G, rotate, (300, 64, 9))
    q = queries(c, T)
    q[:, 0, 2, 5] = bad
    rows = torch.ones(q.shape[:3], dtype=torch.bool, device="cuda")
    rows[:, 0, 2] = False
    out, lse = attend(c, q)
    check_rows(c, q, out, lse, 1 / math.sqrt(D), rows)
    assert bool(torch.isnan(out[~rows]).all())
