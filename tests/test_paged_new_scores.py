"""Scores of new tokens: in the example's loop, and in a loop of eviction in place, they are their own weights alone."""
import numpy as np
import pytest

import paper_2608_02901_gb300 as akv
import paged_exact as exact
import paged_share_ref as plain
from test_paged_example import example
from test_paged_together import SM, Loop, int32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("kw", [dict(heads=4, group=4, steps=40, budget=300), dict(heads=2, group=3, steps=7, page=16, budget=1000, answers=1, seed=3)])
def test_the_examples_new_tokens_begin_at_zero(kw, monkeypatch):
    """Where the loop weighs tokens with what was there before, nothing was there of those appended since."""
    new, looked = [], []
    append, weights = akv.akv_paged_append, akv.akv_paged_weights

    def appended(p, pages, k, v, *args, n_new=None, **kwargs):
        at = torch.arange(pages.table.shape[1] * p.page_tokens, device="cuda")
        new.append((at >= pages.lens[:, None]) & (at < (pages.lens + n_new)[:, None]))
        return append(p, pages, k, v, *args, n_new=n_new, **kwargs)

    def weighed(p, pages, q, lse, now, *args, was=None, decay=1.0, **kwargs):
        if decay:
            for places in new:
                looked.append(int(places.sum()))
                assert bool((was.transpose(1, 2)[places] == 0).all())
        new.clear()
        return weights(p, pages, q, lse, now, *args, was=was, decay=decay, **kwargs)

    monkeypatch.setattr(akv, "akv_paged_append", appended)
    monkeypatch.setattr(akv, "akv_paged_weights", weighed)
    assert example().within_budget(verbose=False, **kw)["lacked"] == 0
    assert len(looked) == kw["steps"] and min(looked) == 3 * kw.get("answers", 3)


def test_new_tokens_after_an_eviction_in_place():
    """Cut in place, the places behind the count set to 0, fork, append, weigh: a new token's score is its weight."""
    s = Loop(2, 4, 16, 64, False, True, seed=21)
    s.put(s.prompts + [0] * 8)
    q, lse = s.attend(16)
    s.weigh(q, lse, 0.0)
    s.evict([0, 1], [0, 1], [200, 150], 4, 32)
    akv.akv_pages_trim(s.p, s.pages, int32([0, 1]))
    behind = torch.arange(s.scores.shape[2], device="cuda") >= s.c.lens[:, None]
    assert bool((s.scores.transpose(1, 2)[behind] != 0).any())  # they are left as they were
    s.scores.masked_fill_(behind[:, None], 0)
    akv.akv_pages_fork(s.p, s.pages, int32([0, 1]), int32([2, 3]))
    s.scores[2:4] = s.scores[:2]
    s.put([5, 5, 3, 1] + [0] * 6)
    q, lse = s.attend(1)
    s.weigh(q, lse, 0.9)
    total, tol = plain.weights(exact.Exact(s.p, s.c.pool[0], s.c.table, s.c.lens_h), q, lse, SM)
    for b, (first, n) in enumerate(((200, 5), (150, 5), (200, 3), (150, 1))):
        for h in range(2):
            own = total[b][h][first : first + n]
            d = (s.scores[b, h, first : first + n].double() - own).abs()
            assert bool((d <= tol[b][h][first : first + n] + 2.0**-23 * own + 1e-37).all())
    assert np.array_equal(s.c.lens.cpu().numpy()[:4], [205, 155, 203, 151])
