"""The serving loop of examples/paged_decode.py, run as a user would."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("paged_decode", os.path.join(ROOT, "examples", "paged_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kw", [dict(heads=4, group=4, steps=70, top=16), dict(heads=2, group=3, steps=5, page=16, top=40, answers=1, seed=3)])
def test_serving_loop(kw):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    got = example().main(verbose=False, **kw)
    assert got["unmoved"]
    # kept pages hold part of the softmax, never more than all of it (1e-3: bf16 outputs are not in it, lse is fp32)
    assert 0 < got["share"] <= 1 + 1e-3
    # the state adds up: every table entry is held, the live pages are the pool's first
    table, refs = got["table"].cpu(), got["refs"].cpu()
    held = torch.bincount(table[table >= 0].long(), minlength=len(refs))
    assert torch.equal(held.int(), refs)
    assert got["live"] == int((refs > 0).sum()) and bool((refs[: got["live"]] > 0).all())
    if got["agree"] is not None:
        assert got["agree"] > 0.9
