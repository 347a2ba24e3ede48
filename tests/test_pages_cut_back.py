"""Rows whose length was cut back, to go on from an earlier token: pages that they will write and others hold become their own."""
import numpy as np
import pytest

import paper_2608_02901_gb300 as akv
from test_pages import Gpu, Sim, filled, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


class Cut(Sim):
    """The simulation with the rule for every page that the new tokens fall into."""

    def reserve(self, n_new):
        P, most = self.P, self.table.shape[1] * self.P
        spans = []
        for r, n in enumerate(n_new):
            n = min(max(int(n), 0), most - int(self.lens[r]))
            spans.append(range(int(self.lens[r]) // P, -(-(int(self.lens[r]) + n) // P)) if n else range(0))
        writers = {}
        for r, span in enumerate(spans):
            for j in span:
                if self.table[r, j] >= 0:
                    writers.setdefault(int(self.table[r, j]), []).append(r)
        want = []  # (row, position, page given up or None, its content is needed)
        for r, span in enumerate(spans):
            for j in span:
                page = int(self.table[r, j])
                if page < 0:
                    if j * P >= self.lens[r]:
                        want.append((r, j, None, False))
                elif self.refs[page] > 1 and not (len(writers[page]) == self.refs[page] and writers[page][0] == r):
                    want.append((r, j, page, bool(j * P < self.lens[r])))
        free = [i for i, x in enumerate(self.refs) if x == 0]
        if len(want) > len(free):
            return len(want) - len(free)
        was = self.content.copy()
        for (r, j, page, content), to in zip(want, free):
            if page is not None:
                self.refs[page] -= 1
                if content:
                    self.content[:, to] = was[:, page]
            self.table[r, j] = to
            self.refs[to] = 1
        return 0


@pytest.mark.parametrize("page,layers,heads,most,rows,pool", [(16, 1, 1, 9, 24, 120), (64, 3, 2, 5, 40, 120), (128, 2, 1, 70, 6, 140)])
def test_a_life_of_pages_with_cuts(page, layers, heads, most, rows, pool):
    rng = np.random.default_rng(page + 1)
    sim = filled(rows, most, pool, page, layers, [int(x) for x in rng.integers(0, most * page * 2 // 3, max(1, rows // 6))], seed=7)
    sim.__class__ = Cut
    g = Gpu(sim, heads, pad=1 if layers > 1 else 0)
    full = 0
    for step in range(80):
        kind = rng.integers(0, 6)
        if kind <= 1:
            empty = [r for r in range(rows) if sim.lens[r] == 0 and np.all(sim.table[r] < 0)]
            pairs = [(int(rng.integers(0, rows)), r) for r in empty[: int(rng.integers(1, 6))]]
            pairs = [(a, b) for a, b in pairs if a not in [y for _, y in pairs]]
            if pairs:
                akv.akv_pages_fork(g.p, g.pages, ints(a for a, _ in pairs), ints(b for _, b in pairs))
                sim.fork(pairs)
        elif kind <= 3:
            # some rows go back, a few to a page's edge, some to the start; then room for new tokens
            for r in rng.integers(0, rows, rows // 3):
                to = int(rng.integers(0, sim.lens[r] + 1))
                sim.lens[r] = to if rng.random() < 0.6 else to // page * page
            g.lens.copy_(torch.from_numpy(sim.lens))
            n = rng.integers(-1, 2, rows) if step % 2 else rng.integers(0, 4 * page, rows)
            if step % 5 == 0:
                n[rng.integers(0, rows)] = most * page
            akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
            missing = sim.reserve(n)
            assert int(g.one) == missing
            full += missing > 0
            if not missing:
                add = np.minimum(np.maximum(n, 0), most * page - sim.lens).astype(np.int32)
                sim.lens += add
                g.lens += torch.from_numpy(add).cuda()
        elif kind == 4:
            rows_ = [int(x) for x in rng.integers(0, rows, 3)]
            akv.akv_pages_free(g.p, g.pages, ints(rows_))
            sim.free(rows_)
        else:
            akv.akv_pages_compact(g.p, g.pages, g.one)
            assert int(g.one) == sim.compact()
        g.check(sim)
    assert full  # a pool without room came up too


class Rows:
    """A cache of real rows: requests that share pages, what each has been given."""

    def __init__(self, rows, n_pages, most=10, page=16, bounds=True):
        self.p = akv.PagedParams(n_kv_heads=2, n_q_heads=4, page_tokens=page, bounds=bounds)
        dev = dict(dtype=torch.int32, device="cuda")
        self.pool = torch.zeros((1, n_pages, akv.akv_paged_page_bytes(self.p)), dtype=torch.uint8, device="cuda")
        self.table, self.lens = torch.full((rows, most), -1, **dev), torch.zeros(rows, **dev)
        self.refs, self.missing = torch.zeros(n_pages, **dev), torch.zeros(1, **dev)
        self.pages = akv.Pages(self.p, self.pool, self.table, self.lens, self.refs)
        self.gen = torch.Generator(device="cuda").manual_seed(8)

    def tokens(self, T):
        shape = (len(self.lens), T, 2, 128)
        return (torch.randn(shape, generator=self.gen, device="cuda").to(torch.bfloat16) for _ in range(2))

    def reserve(self, n):
        akv.akv_pages_reserve(self.p, self.pages, ints(n), self.missing)
        return int(self.missing)

    def append(self, n):
        k, v = self.tokens(max(n))
        akv.akv_paged_append(self.p, self.pages, k, v, n_new=ints(n))
        self.lens += ints(n)
        return k, v

    def read(self, T):
        k, v = (torch.empty((len(self.lens), T, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        akv.akv_paged_read(self.p, self.pages, k, v)
        return torch.stack((k, v))


@pytest.mark.parametrize("cut,new", [(64, 1), (64, 6), (60, 1), (60, 10), (48, 30), (37, 1), (16, 60), (0, 1), (0, 80), (69, 3)])
def test_a_child_that_goes_back_leaves_its_parent_alone(cut, new):
    c = Rows(3, 40)
    assert c.reserve([70, 0, 0]) == 0
    c.append([70, 0, 0])
    akv.akv_pages_fork(c.p, c.pages, ints([0, 0]), ints([1, 2]))
    before = c.read(70)
    c.lens[1] = cut
    assert c.reserve([0, new, 0]) == 0
    k, _ = c.append([0, new, 0])
    after = c.read(160)
    assert torch.equal(after[:, 0, :70], before[:, 0]) and torch.equal(after[:, 2, :70], before[:, 2])
    assert torch.equal(after[:, 1, :cut], before[:, 1, :cut])
    assert int(c.lens[1]) == cut + new
    # the child's own tokens: a row's step is below 1, its error's norm at most 4 steps (rotated)
    err = (after[0, 1, cut : cut + new].float() - k[1, :new].float()).norm(dim=-1)
    assert float(err.max()) < 4 * 1.0
    held = torch.bincount(c.table[c.table >= 0].long(), minlength=40)
    assert torch.equal(held.int(), c.refs)


def test_all_holders_go_back_to_different_lengths():
    c = Rows(3, 40)
    c.reserve([70, 0, 0])
    c.append([70, 0, 0])
    akv.akv_pages_fork(c.p, c.pages, ints([0, 0]), ints([1, 2]))
    before = c.read(70)
    cuts = [32, 40, 64]
    c.lens.copy_(ints(cuts))
    new = [20, 20, 20]
    assert c.reserve(new) == 0
    kept = c.table.cpu()
    c.append(new)
    after = c.read(84)
    for r in range(3):
        assert torch.equal(after[:, r, : cuts[r]], before[:, r, : cuts[r]])
    written = [set(kept[r, cuts[r] // 16 : -(-(cuts[r] + 20) // 16)].tolist()) for r in range(3)]
    assert not (written[0] & written[1] or written[0] & written[2] or written[1] & written[2])
    held = torch.bincount(c.table[c.table >= 0].long(), minlength=40)
    assert torch.equal(held.int(), c.refs)


def test_a_page_that_is_missing_under_tokens_stays_missing():
    sim = filled(2, 6, 20, 16, 1, [40, 20], seed=9)
    sim.__class__ = Cut
    sim.refs[sim.table[0, 2]] = 0
    sim.table[0, 2] = -1
    g = Gpu(sim)
    akv.akv_pages_reserve(g.p, g.pages, ints([20, 20]), g.one)
    assert int(g.one) == sim.reserve([20, 20]) == 0
    assert sim.table[0, 2] == -1 and sim.table[0, 3] >= 0
    g.check(sim)
