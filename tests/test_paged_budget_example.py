"""The loop of examples/paged_decode.py that keeps a bounded number of tokens, run as a user would."""
import pytest

from test_paged_example import example

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(heads=4, group=4, steps=40, budget=300), dict(heads=2, group=3, steps=7, page=16, budget=1000, answers=1, seed=3)])
def test_loop_within_a_budget(kw):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    got = example().within_budget(verbose=False, **kw)
    assert got["lacked"] == 0
    # kept tokens hold part of the softmax, never more than all of it (1e-3: fp32 lse)
    assert 0 < got["mass"] <= 1 + 1e-3
    # every answer holds its budget, or all it has, and the tokens since it was cut
    steps, budget, answers = kw["steps"], kw["budget"], kw.get("answers", 3)
    first = [min(n, budget) for n in (3000, 1777, 940) for _ in range(answers)]
    grown = steps // 2 + 1
    assert got["lens"].tolist() == [min(n + grown, budget) + steps - grown for n in first]
    table, refs = got["table"].cpu(), got["refs"].cpu()
    assert torch.equal(torch.bincount(table[table >= 0].long(), minlength=len(refs)).int(), refs)
    assert bool(torch.isfinite(got["scores"]).all()) and bool((got["scores"] >= 0).all())
