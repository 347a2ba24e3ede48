"""Page operations of the paged cache on the GPU against a plain simulation of their rules."""
import numpy as np
import pytest

import paper_2608_02901_gb300 as akv

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


class Sim:
    """The state on the host: every rule of the header spelled out, a page's content as one number per layer."""

    def __init__(self, rows, max_pages, n_pages, page, layers):
        self.P, self.layers = page, layers
        self.table = np.full((rows, max_pages), -1, np.int32)
        self.lens = np.zeros(rows, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.content = np.arange(layers * n_pages, dtype=np.int64).reshape(layers, n_pages) + 1

    def fork(self, pairs):
        for a, b in pairs:
            if a == b or not (0 <= a < len(self.lens) and 0 <= b < len(self.lens)):
                continue
            n = -(-int(self.lens[a]) // self.P)
            self.table[b] = -1
            self.table[b, :n] = self.table[a, :n]
            self.lens[b] = self.lens[a]
            for page in self.table[a, :n]:
                self.refs[page] += 1

    def free(self, rows):
        for r in rows:
            if not 0 <= r < len(self.lens):
                continue
            for page in self.table[r]:
                if page >= 0:
                    self.refs[page] -= 1
            self.table[r] = -1
            self.lens[r] = 0

    def reserve(self, n_new):
        P, most = self.P, self.table.shape[1] * self.P
        want = []  # (row, position, page that is copied or None)
        tails = {}
        for r, n in enumerate(n_new):
            n = min(max(int(n), 0), most - int(self.lens[r]))
            if n and self.lens[r] % P:
                tails.setdefault(int(self.table[r, self.lens[r] // P]), []).append(r)
        for r, n in enumerate(n_new):
            n = min(max(int(n), 0), most - int(self.lens[r]))
            if not n:
                continue
            at = int(self.lens[r]) // P
            if self.lens[r] % P:
                page = int(self.table[r, at])
                writers = tails[page]
                if self.refs[page] > 1 and not (len(writers) == self.refs[page] and writers[0] == r):
                    want.append((r, at, page))
            want += [(r, j, None) for j in range(-(-int(self.lens[r]) // P), -(-(int(self.lens[r]) + n) // P)) if self.table[r, j] < 0]
        free = [i for i, x in enumerate(self.refs) if x == 0]
        if len(want) > len(free):
            return len(want) - len(free)
        for (r, j, page), to in zip(want, free):
            if page is not None:
                self.content[:, to] = self.content[:, page]
                self.refs[page] -= 1
            self.table[r, j] = to
            self.refs[to] = 1
        return 0

    def compact(self):
        live = [i for i, x in enumerate(self.refs) if x > 0]
        n = len(live)
        holes = [i for i in range(n) if self.refs[i] <= 0]
        for a, b in zip([i for i in live if i >= n], holes):
            self.content[:, b] = self.content[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b
        return n


class Gpu:
    def __init__(self, sim, heads=1, pad=0, bounds=False):
        self.p = akv.PagedParams(n_kv_heads=heads, n_q_heads=heads, page_tokens=sim.P, rotate=False, bounds=bounds)
        dev = dict(device="cuda")
        size = akv.akv_paged_page_bytes(self.p)
        self.table = torch.from_numpy(sim.table).cuda()
        self.lens, self.refs = torch.from_numpy(sim.lens).cuda(), torch.from_numpy(sim.refs).cuda()
        n = sim.content.shape[1]
        wide = torch.zeros((sim.layers, n + pad, size // 8), dtype=torch.int64, **dev)
        self.pool = wide[:, :n]
        self.pool.copy_(torch.from_numpy(sim.content)[:, :, None].cuda() + torch.arange(size // 8, **dev) * 1000003)
        self.pages = akv.Pages(self.p, self.pool, self.table, self.lens, self.refs)
        self.one = torch.full((1,), -9, dtype=torch.int32, **dev)
        self.size = size

    def check(self, sim, live_only=False):
        assert np.array_equal(self.lens.cpu().numpy(), sim.lens)
        assert np.array_equal(self.refs.cpu().numpy(), sim.refs)
        assert np.array_equal(self.table.cpu().numpy(), sim.table)
        got = (self.pool - torch.arange(self.size // 8, device="cuda") * 1000003).cpu().numpy()
        assert np.array_equal(got, np.broadcast_to(sim.content[:, :, None], got.shape))


def ints(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device="cuda")


def filled(rows, max_pages, n_pages, page, layers, lens, seed):
    sim = Sim(rows, max_pages, n_pages, page, layers)
    ids = np.random.default_rng(seed).permutation(n_pages)
    at = 0
    for r, n in enumerate(lens):
        k = -(-n // page)
        sim.table[r, :k] = ids[at : at + k]
        sim.refs[ids[at : at + k]] = 1
        sim.lens[r] = n
        at += k
    return sim


@pytest.mark.parametrize("page,layers,heads,bounds", [(16, 1, 1, False), (64, 3, 2, True), (128, 2, 3, False)])
def test_a_life_of_pages(page, layers, heads, bounds):
    """Random forks, reservations, frees and compactions, each checked whole."""
    rng = np.random.default_rng(page)
    rows, most = 24, 9
    sim = filled(rows, most, 260, page, layers, [int(x) for x in rng.integers(0, 5 * page, 8)], seed=1)
    g = Gpu(sim, heads, pad=2 if layers > 1 else 0, bounds=bounds)
    for step in range(60):
        kind = rng.integers(0, 4)
        if kind == 0:
            empty = [r for r in range(rows) if sim.lens[r] == 0 and np.all(sim.table[r] < 0)]
            pairs = [(int(rng.integers(0, rows)), r) for r in empty[: int(rng.integers(1, 6))]]
            pairs = [(a, b) for a, b in pairs if a not in [y for _, y in pairs]]
            if pairs:
                akv.akv_pages_fork(g.p, g.pages, ints(a for a, _ in pairs), ints(b for _, b in pairs))
                sim.fork(pairs)
        elif kind == 1:
            n = rng.integers(-1, 2, rows) if step % 2 else rng.integers(0, 3 * page, rows)
            akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
            missing = sim.reserve(n)
            assert int(g.one) == missing
            if not missing and step % 3:  # the tokens come
                add = np.minimum(np.maximum(n, 0), most * page - sim.lens).astype(np.int32)
                sim.lens += add
                g.lens += torch.from_numpy(add).cuda()
        elif kind == 2:
            rows_ = [int(x) for x in rng.integers(0, rows, 3)]
            akv.akv_pages_free(g.p, g.pages, ints(rows_))
            sim.free(rows_)
        else:
            akv.akv_pages_compact(g.p, g.pages, g.one)
            assert int(g.one) == sim.compact()
        g.check(sim)


def test_the_last_holder_that_writes_keeps_the_page():
    sim = filled(4, 4, 20, 16, 2, [20], seed=2)
    sim.fork([(0, 1), (0, 2)])
    g = Gpu(sim)
    for n in ([0, 0, 1, 0], [1, 1, 0, 0]):
        akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
        assert int(g.one) == sim.reserve(n) == 0
        g.check(sim)
    # row 0 kept its page: rows 1 and 2 have copies
    assert len({int(sim.table[r, 1]) for r in range(3)}) == 3 and sim.refs[sim.table[0, 1]] == 1


def test_a_pool_without_room_is_left_alone():
    sim = filled(3, 8, 6, 16, 1, [40, 16], seed=3)
    sim.fork([(0, 2)])
    g = Gpu(sim)
    n = [1, 20, 1]
    akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
    assert int(g.one) == sim.reserve(n) == 1
    g.check(sim)
    n = [1, 16, 0]
    akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
    assert int(g.one) == sim.reserve(n) == 0
    g.check(sim)


def test_lists_outside_the_table_and_the_pool():
    sim = filled(4, 4, 20, 16, 1, [30, 17], seed=4)
    g = Gpu(sim)
    pairs = [(0, 2), (-1, 3), (7, 3), (1, 9), (1, -2), (1, 1)]
    akv.akv_pages_fork(g.p, g.pages, ints(a for a, _ in pairs), ints(b for _, b in pairs))
    sim.fork(pairs)
    g.check(sim)
    akv.akv_pages_free(g.p, g.pages, ints([-1, 4, 2, 2, 100]))
    sim.free([2])
    g.check(sim)
    akv.akv_pages_copy(g.p, g.pages, ints([0, -1, 3, 20, 5]), ints([1, 2, 20, 4, 5]))
    sim.content[:, 1] = sim.content[:, 0]
    g.check(sim)
    akv.akv_pages_copy(g.p, g.pages, ints([]), ints([]))
    akv.akv_pages_free(g.p, g.pages, ints([]))
    g.check(sim)


@pytest.mark.parametrize("n_pages,rows,most", [(5000, 3, 1500), (1, 1, 1), (4097, 1500, 4), (100003, 12, 9000)])
def test_sizes_of_pools_and_tables(n_pages, rows, most):
    """Lists that pass one round of the plan kernel, long rows, many rows."""
    rng = np.random.default_rng(n_pages)
    share = max(1, n_pages * 2 // 3 // rows)
    sim = filled(rows, most, n_pages, 16, 1, [16 * int(rng.integers(0, min(share, most) + 1)) for _ in range(rows)], seed=5)
    g = Gpu(sim)
    gone = [int(x) for x in rng.integers(0, rows, max(1, rows // 3))]
    akv.akv_pages_free(g.p, g.pages, ints(gone))
    sim.free(gone)
    n = rng.integers(0, 16 * max(2, n_pages // rows // 3), rows)
    akv.akv_pages_reserve(g.p, g.pages, ints(n), g.one)
    assert int(g.one) == sim.reserve(n)
    g.check(sim)
    akv.akv_pages_compact(g.p, g.pages, g.one)
    assert int(g.one) == sim.compact()
    g.check(sim)


def test_forked_requests_go_apart():
    """Two answers to one prompt: the same prefix, each its own tokens after it."""
    p = akv.PagedParams(n_kv_heads=2, n_q_heads=4, page_tokens=32, bounds=True)
    pool = torch.zeros((1, 40, akv.akv_paged_page_bytes(p)), dtype=torch.uint8, device="cuda")
    table = torch.full((2, 10), -1, dtype=torch.int32, device="cuda")
    lens, refs = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
    pages = akv.Pages(p, pool, table, lens, refs)
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(6)
    rows = []

    def add(n):
        n = ints(n)
        akv.akv_pages_reserve(p, pages, n, missing)
        k, v = torch.randn((2, 2, int(n.max()), 2, 128), generator=gen, device="cuda").to(torch.bfloat16)
        akv.akv_paged_append(p, pages, k, v, n_new=n)
        lens.add_(n)
        rows.append((k, v, n.tolist()))

    def read():
        k, v = torch.empty((2, 2, 150, 2, 128), dtype=torch.bfloat16, device="cuda")
        akv.akv_paged_read(p, pages, k, v)
        return k, v

    add([77, 0])
    akv.akv_pages_fork(p, pages, ints([0]), ints([1]))
    prompt = read()
    assert torch.equal(prompt[0][0], prompt[0][1]) and torch.equal(prompt[1][0], prompt[1][1])
    for _ in range(30):
        add([1, 1])
    after = read()
    for a, b in zip(prompt, after):
        assert torch.equal(a[:, :77], b[:, :77])
    assert not torch.equal(after[0][0, 77:107], after[0][1, 77:107])
    # each answer's tokens are within half a step of what was given (a row's range is below 11 after the rotation's
    # scaling by sqrt(2), a step below 1; the inverse rotation's rows have norm sqrt(128) / 16)
    for b in range(2):
        k = torch.cat([x[0][b, : x[2][b]] for x in rows[1:]])
        assert float((after[0][b, 77:107].float() - k.float()).abs().max()) < 0.5 * 128 / 16
    shared = (table[0] == table[1]) & (table[0] >= 0)
    assert shared.tolist() == [True, True] + [False] * 8
    akv.akv_pages_free(p, pages, ints([0]))
    akv.akv_pages_compact(p, pages, missing)
    assert torch.equal(read()[0][1], after[0][1]) and int(missing) == 4
