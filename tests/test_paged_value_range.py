"""Attention where a few tokens' values are far larger than the rest, but hardly weigh or are not seen: they cost the others nothing."""
import math

import pytest

import paged_exact as exact
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, attend, params, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def put(c, k, v):
    akv.akv_paged_append(c.p, c.pages, k, v)
    c.lens.fill_(k.shape[1])


@pytest.mark.parametrize("half,group,G,rotate", [(True, 64, 2, False), (False, 128, 2, False), (True, 64, 8, True), (False, 64, 8, False)])
@pytest.mark.parametrize("n", [40, 1000])
def test_large_values_that_a_row_does_not_see(half, group, G, rotate, n):
    """A draft's last token has values of 30000, the others of 2^-10 or 2^-14: its earlier rows do not see it."""
    p = params(1, G, 32, group, half, rotate)
    c = Cache(p, [n], seed=n + G)
    k, v = c.rows(n)
    v *= 2.0**-10 if half else 2.0**-14
    v[:, -1] = (30000 * torch.sign(torch.randn(v[:, -1].shape, generator=c.gen, device="cuda"))).to(v.dtype)
    put(c, k, v)
    q = queries(c, 3)
    out, lse = attend(c, q)
    # the rows that do not see it (the last one's outputs are 30000 strong)
    want, want_lse, tol, tol_lse = exact.Exact(p, c.pool[0], c.table, [n]).attend(q, 1 / math.sqrt(D))
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())
    assert float(want[:, :2].abs().max()) < 0.01 < float(want[:, 2].abs().max())


@pytest.mark.parametrize("place", [0, 17, 250, 599])
@pytest.mark.parametrize("half,group,G,rotate", [(True, 64, 2, False), (False, 64, 4, True), (True, 128, 16, False)])
def test_large_values_that_hardly_weigh(place, half, group, G, rotate):
    """One token's values are 2^25 to 2^29 times the others', its logits some 100 below."""
    p = params(1, G, 16, group, half, rotate)
    c = Cache(p, [600], seed=place)
    k, v = c.rows(600)
    base = torch.randn(D, generator=c.gen, device="cuda")
    v *= 2.0**-10 if half else 2.0**-14
    v[:, place] = (30000 * torch.sign(torch.randn(v[:, place].shape, generator=c.gen, device="cuda"))).to(v.dtype)
    k[:, place] = (-6 * base).to(k.dtype)
    put(c, k, v)
    q = (1.5 * base + 0.3 * torch.randn((1, 1, G, D), generator=c.gen, device="cuda")).to(k.dtype)
    exact.check(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("half,G", [(True, 4), (False, 8), (True, 16)])
@pytest.mark.parametrize("up", [True, False])
def test_values_that_grow_and_fall_along_a_request(half, G, up):
    """Scales from 2^-17 to 2^12 along the tokens, logits against them: what weighs is now small, now large."""
    p = params(1, G, 64, 64, half, False)
    c = Cache(p, [1500], seed=G)
    k, v = c.rows(1500)
    at = torch.linspace(-14, 13, 1500, device="cuda")
    at = at if up else at.flip(0)
    v *= torch.exp2(at.round())[None, :, None, None].to(v.dtype)
    base = torch.randn(D, generator=c.gen, device="cuda")
    k = (0.2 * k.float() - 0.25 * at[:, None, None] * base).to(k.dtype)  # the larger the values, the lower the logit
    put(c, k, v)
    q = (1.5 * base + 0.3 * torch.randn((1, 1, G, D), generator=c.gen, device="cuda")).to(k.dtype)
    exact.check(p, c, q, *attend(c, q), 1 / math.sqrt(D))


def test_constant_values_on_top():
    """The tokens with the largest logits have constant values (a scale of 0), those below them have not."""
    p = params(1, 4, 16, 64, True, False)
    c = Cache(p, [300], seed=3)
    k, v = c.rows(300)
    base = torch.randn(D, generator=c.gen, device="cuda")
    v[:, 100:120] = 0.75
    k[:, 100:120] = (0.5 * base).to(k.dtype)
    put(c, k, v)
    q = (1.5 * base + 0.3 * torch.randn((1, 1, 4, D), generator=c.gen, device="cuda")).to(k.dtype)
    for sm in (1 / math.sqrt(D), 1.0, 4.0):
        exact.check(p, c, q, *attend(c, q, sm_scale=sm), sm)
