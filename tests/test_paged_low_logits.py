"""Attention where every logit of a row is far below zero."""
import pytest

import paged_exact as exact
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, attend, params, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("rotate,sm", [(False, 1.0), (True, 1.0), (False, -1.0)])
def test_logits_far_below_zero(rotate, sm):
    """Rows all of whose logits are -10^30 and less see their tokens all the same: the largest logit's value is the output."""
    c = Cache(params(1, 4, 32, 64, False, rotate), [1, 1, 40, 200], seed=4)
    k, v = c.rows(200)
    k = (k.float() * 0.1 + torch.sign(torch.tensor(sm)) * 3).to(k.dtype)
    akv.akv_paged_append(c.p, c.pages, k, v, n_new=torch.tensor(c.lens_h, dtype=torch.int32, device="cuda"))
    c.lens.copy_(torch.tensor(c.lens_h))
    q = (-queries(c, 1).abs().float() * 2.0**98).to(torch.bfloat16)
    out, lse = attend(c, q, sm_scale=sm)
    want, want_lse, _, _ = exact.Exact(c.p, c.pool[0], c.table, c.lens_h).attend(q, sm)
    assert bool((want_lse < -1e30).all())
    # logits are 10^26 and more apart but for ties: one token's value, rounded to bf16 (rotated: fp32 sums of 128 values)
    assert bool(((out.double() - want).abs() <= 2.0**-8 * want.abs() + 2.0**-16 * 20).all())
    assert bool(((lse.double() - want_lse).abs() <= 2.0**-14 * want_lse.abs()).all())
