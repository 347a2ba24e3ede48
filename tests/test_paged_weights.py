"""Accumulated attention weights of the paged cache against 64-bit sums; the bound is each number's own (paged_share_ref)."""
import math

import pytest

import paged_exact as exact
import paged_share_ref as plain
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, params, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SM = 1 / math.sqrt(128)


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def make(p, lens, T, seed=0, layers=1):
    c = Cache(p, lens, seed=seed, layers=layers)
    for l in range(layers):
        c.fill(layer=l)
    q = queries(c, T, 1.0)
    return c, q


def attended(c, q, layer=0):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    akv.akv_paged_attn(c.p, c.pages, q, out, lse=lse, sm_scale=SM, layer=layer)
    return lse


def scores(c, value=0.0):
    return torch.full((len(c.lens_h), c.p.n_kv_heads, c.table.shape[1] * c.p.page_tokens), value, device="cuda")


def check(c, q, lse, now, was, decay, before, layer=0, sm=SM):
    """now against decay was + weights; numbers behind the tokens held as before."""
    E = exact.Exact(c.p, c.pool[layer], c.table, c.lens.tolist())
    total, tol = plain.weights(E, q, lse, sm)
    for b, n in enumerate(E.lens):
        n = max(n, 0)
        for h in range(c.p.n_kv_heads):
            old = decay * was[b, h, :n].double() if was is not None and decay else torch.zeros(n, dtype=torch.float64, device="cuda")
            want = old + total[b][h]
            bound = tol[b][h] + 2.0**-23 * (old.abs() + want.abs()) + 1e-37
            d = (now[b, h, :n].double() - want).abs()
            assert bool((d <= bound).all()), (b, h, float((d / bound).max()))
            assert torch.equal(now[b, h, n:], before[b, h, n:])


@pytest.mark.parametrize("decay", [0.0, 0.9])
@pytest.mark.parametrize("H,G,T,page,group,half,rotate", [
    (2, 4, 1, 64, 64, False, False), (2, 1, 1, 16, 128, True, True), (1, 8, 2, 32, 64, False, True), (3, 3, 3, 128, 64, True, False),
    (1, 4, 64, 64, 64, False, True), (2, 8, 9, 64, 128, False, False), (1, 64, 2, 16, 64, False, False), (1, 2, 33, 16, 128, True, True)])
def test_weights(H, G, T, page, group, half, rotate, decay):
    p = params(H, G, page, group, half, rotate)
    c, q = make(p, [300, 1, 77, 0, 129, 16, 640], T, seed=T)
    lse = attended(c, q)
    now, was = scores(c, 5.0), torch.rand_like(scores(c))
    before = now.clone()
    akv.akv_paged_weights(p, c.pages, q, lse, now, was=was, decay=decay, sm_scale=SM)
    check(c, q, lse, now, was, decay, before)


@pytest.mark.parametrize("G,T,rotate", [(4, 1, True), (8, 1, False), (4, 2, True), (4, 16, False)])
def test_long_rows(G, T, rotate):
    """Many tiles a CTA, units cut anywhere."""
    p = params(4, G, 64, 64, False, rotate)
    c, q = make(p, [20001, 777, 9000], T, seed=G)
    lse = attended(c, q)
    now = scores(c)
    before = now.clone()
    akv.akv_paged_weights(p, c.pages, q, lse, now, sm_scale=SM)
    check(c, q, lse, now, None, 1.0, before)
    # a query's weights add up to one
    total = now.double().sum(-1)
    assert bool(((total - G * T).abs() <= 1e-4 * G * T).all())


def test_in_place_and_layers():
    p = params(2, 4, 32, 64, False, True)
    c, q = make(p, [500, 33], 1, seed=5, layers=2)
    now = torch.rand_like(scores(c))
    for layer in (0, 1):
        lse = attended(c, q, layer)
        before = now.clone()
        akv.akv_paged_weights(p, c.pages, q, lse, now, was=now, decay=0.5, sm_scale=SM, layer=layer)
        check(c, q, lse, now, before, 0.5, before, layer)


def test_strides():
    p = params(2, 4, 64, 64, False, False)
    c, q = make(p, [400, 90], 2, seed=6)
    wide = torch.zeros((2, 2, 2, 10, 128), dtype=q.dtype, device="cuda")[:, :, 0]
    view = wide[:, :, 1:9]
    view.copy_(q)
    lse = attended(c, q)
    flat, room = scores(c, 0.0), torch.full((2, 2, flat_cap(c) + 7), 3.0, device="cuda")
    now = room.transpose(0, 1)[:, :, 3 : 3 + flat_cap(c)]
    before = now.clone()
    was = torch.rand((1, 1, flat_cap(c)), device="cuda").expand(2, 2, flat_cap(c))
    akv.akv_paged_weights(p, c.pages, view, lse, now, was=was, decay=2.0, sm_scale=SM)
    check(c, q, lse, now, was, 2.0, before)
    assert bool((room[:, :, :3] == 3).all()) and bool((room[:, :, 3 + flat_cap(c) :] == 3).all())


def flat_cap(c):
    return c.table.shape[1] * c.p.page_tokens


def test_what_adds_nothing():
    """Queries without a finite lse, or with a NaN; tokens with a NaN key; pages outside the pool."""
    p = params(1, 4, 16, 64, False, False)
    c = Cache(p, [100, 100, 60])
    k, v = c.rows(100)
    k[0, 50, 0, 3] = math.nan
    v[0, 20, 0, 3] = math.inf
    akv.akv_paged_append(p, c.pages, k, v, n_new=torch.tensor(c.lens_h, dtype=torch.int32, device="cuda"))
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))
    q = queries(c, 2, 1.0)
    lse = torch.full(q.shape[:3], 3.0, device="cuda")
    lse[0, 0, 0], lse[0, 1, 1], lse[1, 0, 2] = math.nan, math.inf, -math.inf
    q[1, 1, 3, 7] = math.nan
    c.table[2, 1] = 10**6
    now, was = scores(c, 1.0), torch.rand_like(scores(c))
    akv.akv_paged_weights(p, c.pages, q, lse, now, was=was, decay=1.0, sm_scale=SM)
    assert bool(torch.isfinite(now).all())
    assert float(now[0, 0, 50]) == float(was[0, 0, 50])
    assert torch.equal(now[2, 0, 16:32], was[2, 0, 16:32])
    # against the sums over what counts
    lse2 = lse.clone()
    lse2[1, 1, 3] = math.nan
    c.table[2, 1] = c.table[2, 0]
    E = exact.Exact(p, c.pool[0], c.table, c.lens.tolist())
    total, tol = plain.weights(E, torch.nan_to_num(q), lse2, SM)
    for b, n in enumerate(c.lens_h):
        ok = torch.isfinite(total[b][0])
        if b == 2:
            ok[16:32] = False
        want = was[b, 0, :n].double() + total[b][0]
        bound = tol[b][0] + 2.0**-22 * want.abs()
        assert bool(((now[b, 0, :n].double() - want).abs() <= bound)[ok].all())


def test_graph():
    p = params(2, 4, 64, 64, False, True)
    c, q = make(p, [900, 33], 1, seed=8)
    lse, now = attended(c, q), scores(c)
    run = lambda: akv.akv_paged_weights(p, c.pages, q, lse, now, was=now, sm_scale=SM)  # noqa: E731
    run()
    torch.cuda.synchronize()
    once = now.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    now.zero_()
    g.replay()
    assert torch.equal(now, once)


def test_lengths_outside_the_table():
    p = params(2, 4, 16, 64, False, False)
    c, q = make(p, [100, 31], 1, seed=9)
    lse = torch.zeros(q.shape[:3], device="cuda")
    c.lens.copy_(torch.tensor([-5, 10**9], dtype=torch.int32))
    now = scores(c, 2.0)
    before = now.clone()
    akv.akv_paged_weights(p, c.pages, q, lse, now, sm_scale=0.0)
    assert torch.equal(now[0], before[0])
    assert bool((now[1, :, :31] == 4.0).all())  # e^0 of four query heads
    assert bool((now[1, :, 31:32] == 0.0).all())  # a place that no token was written to: its scale is a NaN
