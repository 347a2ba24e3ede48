"""Accumulated attention weights where lse is all there is of a logit: scales of zero, or nearly, and query rows of zeros.

A weight is then e^-lse, to paged_share_ref's bound: without a logit 2^-22 of lse's size, 2^-21 for e^x and 2^-24 for each term of a sum,
under 5e-6 of its size here."""
import pytest

import paper_2608_02901_gb300 as akv
from test_paged_cache import params
from test_paged_weights import check, make, scores

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sm", [0.0, 1e-38, 3e-30, 1e-7, -1e-7, 0.1])
@pytest.mark.parametrize("G,T,group,half,rotate", [(4, 1, 64, False, False), (8, 1, 128, True, True), (4, 3, 64, False, True), (16, 1, 128, True, False),
                                                   (4, 8, 64, False, False), (2, 17, 128, True, True)])
def test_logits_of_nearly_zero(G, T, group, half, rotate, sm):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    p = params(2, G, 64, group, half, rotate)
    c, q = make(p, [1000, 77, 3001], T, seed=G + T)
    q[0] = 0
    q[1, :, ::3] = 0
    lse = torch.empty(q.shape[:3], device="cuda")
    akv.akv_paged_attn(p, c.pages, q, torch.empty_like(q), lse=lse, sm_scale=sm)
    now = scores(c)
    before = now.clone()
    akv.akv_paged_weights(p, c.pages, q, lse, now, sm_scale=sm)
    check(c, q, lse, now, None, 1.0, before, sm=sm)
    # the row of zeros by itself: each query token that sees a token gives it e^-lse of its heads
    seen = T - (torch.arange(1000, device="cuda") - (1000 - T)).clamp(min=0)
    for h in range(2):
        w = torch.exp(-lse[0, :, h * G : (h + 1) * G].double()).sum(1)  # of a query token
        want = torch.stack([w[T - int(n) :].sum() for n in seen])
        bound = 2.0**-21 + 2.0**-22 * float(lse[0].abs().max()) + T * G * 2.0**-24
        assert bool(((now[0, h, :1000].double() - want).abs() <= bound * want).all())
