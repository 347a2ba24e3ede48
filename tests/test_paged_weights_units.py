"""Accumulated attention weights of many query rows a unit: units of one tile among longer ones, and units of more rows than are held at a time."""
import pytest

import paper_2608_02901_gb300 as akv
from test_paged_cache import params
from test_paged_weights import SM, attended, check, make, scores

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def weigh(p, lens, T, seed, times=1):
    c, q = make(p, lens, T, seed=seed)
    lse, was = attended(c, q), torch.rand_like(scores(c))
    before, first = scores(c, 3.0), None
    for _ in range(times):
        now = before.clone()
        akv.akv_paged_weights(p, c.pages, q, lse, now, was=was, decay=0.5, sm_scale=SM)
        first = now if first is None else first
        assert torch.equal(now, first)
    check(c, q, lse, first, was, 0.5, before)


@pytest.mark.parametrize("H,G,T,page,group,rotate", [(8, 4, 5, 16, 64, True), (5, 3, 7, 64, 128, False)])
def test_units_of_one_tile(H, G, T, page, group, rotate):
    """Several units a CTA, most of one tile, which one of the two product warps has nothing to do for."""
    p = params(H, G, page, group, False, rotate)
    weigh(p, ([100, 1, 128, 17, 0, 300, 64, 129] * 14)[:110] + [1500], T, seed=H, times=3)


@pytest.mark.parametrize("G,T,group,half,rotate", [(8, 64, 64, False, True), (5, 53, 128, True, False), (64, 5, 64, False, False)])
def test_more_rows_than_are_held(G, T, group, half, rotate):
    """Up to 512 query rows a unit: its tiles are gone over again for each 256."""
    weigh(params(2, G, 64, group, half, rotate), [700, 130, 40], T, seed=T, times=2)
