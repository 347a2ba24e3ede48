"""The steps of examples/paged_decode.py do not wait for the GPU."""
import warnings

import pytest

from test_paged_example import example

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_no_step_waits():
    """Calls that wait for the GPU, as torch counts them: as many with eight steps as with two."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    module = example()
    kw = dict(heads=2, group=2, prompts=(300, 120), answers=2, page=16, top=8, verbose=False)
    module.main(steps=2, **kw)  # (what loads and compiles at first use)
    waits = []
    for steps in (2, 8):
        with warnings.catch_warnings(record=True) as seen:
            warnings.simplefilter("always")
            torch.cuda.set_sync_debug_mode("warn")
            try:
                module.main(steps=steps, **kw)
            finally:
                torch.cuda.set_sync_debug_mode("default")
        waits.append(sum("synchronizing CUDA operation" in str(w.message) for w in seen))
    assert waits[0] == waits[1] > 0  # (after the steps results are read)
