"""Appends to pages that have more than one holder."""
import pytest

import paper_2608_02901_gb300 as akv
from test_pages import ints
from test_pages_cut_back import Rows

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bounds", [False, True])
@pytest.mark.parametrize("rows", [2, 160])  # (keys and values by CTAs of their own, and by one)
def test_append_does_not_write_a_page_that_others_hold(rows, bounds):
    """A pool without room: reserve changes nothing, and the append that follows in the stream leaves shared pages as they are."""
    c = Rows(rows, 5, bounds=bounds)
    assert c.reserve([70] + [0] * (rows - 1)) == 0  # the pool is full
    c.append([70] + [0] * (rows - 1))
    akv.akv_pages_fork(c.p, c.pages, ints([0]), ints([1]))
    before, read = c.pool.clone(), c.read(70)
    new = [0, 5] + [0] * (rows - 2)
    assert c.reserve(new) == 1
    c.append(new)
    assert torch.equal(c.pool, before)
    assert torch.equal(c.read(70)[:, 0], read[:, 0])
    # the parent leaves: the page is the child's alone, and is written
    c.lens[1] = 70
    akv.akv_pages_free(c.p, c.pages, ints([0]))
    assert c.reserve(new) == 0
    c.append(new)
    assert not torch.equal(c.pool, before) and torch.equal(c.read(70)[:, 1], read[:, 1])


def test_a_serving_loop_without_room():
    """The example's steps where the pool holds the prompts and no page more: nothing is written, no length advances."""
    from test_paged_example import example

    prompts = (200, 90)
    got = example().main(heads=2, group=2, steps=4, prompts=prompts, answers=2, page=16, top=8, verbose=False, pool_pages=13 + 6)
    assert got["lacked"] > 0 and got["unmoved"]
    # both prompts and the last answer of each, as they were forked
    assert got["lens"].tolist() == [200, 90, 0, 200, 0, 90]
    table, refs = got["table"].cpu(), got["refs"].cpu()
    assert torch.equal(torch.bincount(table[table >= 0].long(), minlength=len(refs)).int(), refs)
    assert bool((refs[:19] == 2).all())


def test_pages_without_counts_are_written():
    """A cache whose program keeps no counts (refs None) is written as before."""
    c = Rows(2, 12)
    c.table.copy_(torch.arange(12, dtype=torch.int32).view(2, 6).repeat(1, 2)[:, :10])
    pages = akv.Pages(c.p, c.pool, c.table[:, :6], c.lens)
    k, v = c.tokens(33)
    akv.akv_paged_append(c.p, pages, k, v)
    c.lens.fill_(33)
    got = c.read(33)
    assert float((got[0].float() - k.float()).norm(dim=-1).max()) < 4 * 1.0
