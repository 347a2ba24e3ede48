"""Eviction from the paged cache by scores, and giving up the pages behind a length: whole bytes, equal to a simulation of the rules."""
import math

import numpy as np
import pytest

import paged_share_ref as plain
import paper_2608_02901_gb300 as akv

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def int32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


class State:
    """A pool of random bytes; rows with tokens, then rows with room."""

    def __init__(self, lens, room, H=2, page=16, group=64, layers=1, seed=0, refs=True, extra=3):
        rng = self.rng = np.random.default_rng(seed)
        self.p = akv.PagedParams(n_kv_heads=H, n_q_heads=H, page_tokens=page, group=group)
        need = [-(-max(a, b) // page) for a, b in zip(lens, room)]
        most = max(need) + 1
        n_pages = sum(need) + extra
        ids = rng.permutation(n_pages)[: sum(need)]
        self.table = np.full((len(lens), most), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at : at + n]
            at += n
        self.lens = np.array(lens, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.refs[ids] = 1
        self.pool = rng.integers(0, 256, (layers, n_pages, akv.akv_paged_page_bytes(self.p)), dtype=np.uint8)
        cap = most * page
        self.scores = np.exp(2 * rng.standard_normal((len(lens), H, cap))).astype(np.float32)
        self.scores[rng.random(self.scores.shape) < 0.1] = 0
        some = rng.random(self.scores.shape) < 0.3
        self.scores[some] = np.round(self.scores[some])
        self.with_refs = refs

    def upload(self):
        self.d = dict(pool=torch.from_numpy(self.pool).cuda(), table=int32(self.table), lens=int32(self.lens), refs=int32(self.refs),
                      scores=torch.from_numpy(self.scores).cuda())
        return akv.Pages(self.p, self.d["pool"], self.d["table"], self.d["lens"], self.d["refs"] if self.with_refs else None)

    def check(self, src, dst, keep, sink, recent, top=None, layer=0, scores=None):
        pages = self.upload()
        top = max([*keep, 1]) if top is None else top
        H = self.p.n_kv_heads
        kept = akv.KeptTokens(torch.full((len(src), H, top), 7, dtype=torch.int32, device="cuda"), int32(np.full(len(src), 7)))
        dev = self.d["scores"] if scores is None else scores(self.d["scores"])
        akv.akv_paged_evict(self.p, pages, int32(src), int32(dst), dev, kept, keep=None if keep is None else int32(keep), sink=sink,
                            recent=recent, layer=layer)
        pool, sc = self.pool.copy(), self.scores.copy()
        view = pool[layer].reshape(pool.shape[1], H, -1)
        tokens, count = plain.evict(self.p, view, self.table, self.lens, self.refs if self.with_refs else None, src, dst, sc, keep, sink,
                                    recent, top)
        assert np.array_equal(kept.count.cpu().numpy(), count)
        assert np.array_equal(kept.tokens.cpu().numpy(), tokens)
        assert np.array_equal(dev.cpu().numpy(), sc, equal_nan=True)
        assert np.array_equal(self.d["pool"].cpu().numpy(), pool)
        assert np.array_equal(self.d["table"].cpu().numpy(), self.table) and np.array_equal(self.d["refs"].cpu().numpy(), self.refs)
        assert np.array_equal(self.d["lens"].cpu().numpy(), self.lens)
        return count


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page,group,H", [(16, 64, 2), (64, 128, 3), (128, 64, 1), (32, 128, 2)])
def test_kept_tokens_move(page, group, H, in_place):
    lens = [300, 1, 77, 1021, 16, 0, 129]
    keep = [100, 1, 76, 500, 15, 4, 128]
    s = State(lens + [0] * 7, [0] * 7 + keep, H, page, group, seed=page)
    src = list(range(7))
    s.check(src, src if in_place else list(range(7, 14)), keep, 3, 10)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,keep", [(9000, 7777), (9000, 8991), (5000, 33), (4100, 4099), (2048, 2047)])
def test_many_rounds(n, keep, in_place):
    """A cluster moves 2048 tokens a round."""
    s = State([n, 0], [0, keep], H=2, page=64, seed=keep)
    s.check([0], [0 if in_place else 1], [keep], 4, 32)


@pytest.mark.parametrize("sink,recent", [(0, 0), (5, 0), (0, 5), (60, 60), (200, 0), (0, 200), (1000, 1000)])
def test_forced_tokens(sink, recent):
    s = State([200, 0], [0, 100], seed=sink + recent)
    s.check([0], [1], [100], sink, recent)
    s.check([0], [0], [100], sink, recent)


@pytest.mark.parametrize("keep", [0, 1, 17, 199, 200, 1000, -5])
def test_counts(keep):
    s = State([200, 0, 0], [0, 200, 0], seed=4)
    for dst in (0, 1):
        s.check([0], [dst], [keep], 2, 2, top=1000)
    s.check([0], [1], None, 2, 2, top=50)


def test_scores_of_every_kind():
    s = State([700, 0], [0, 300], H=4, seed=9)
    s.scores[0, 0] = 1.0  # ties: the lower ones stay
    s.scores[0, 1, ::3] = np.nan
    s.scores[0, 1, 1::3] = -np.inf
    s.scores[0, 2, ::2] = np.inf
    s.scores[0, 2, 1::4] = -0.0
    s.scores[0, 2, 3::4] = 0.0
    s.scores[0, 3] *= np.float32(1e-42)  # subnormal numbers
    s.scores[0, 3, ::2] *= -1
    for keep in (10, 299, 300):
        s.check([0], [1], [keep], 2, 9)


def test_many_of_one_score_at_the_cut():
    s = State([5000, 0], [0, 2500], H=1, page=64, seed=3)
    s.scores[0] = 0
    s.scores[0, 0, 4000:4100] = 2
    s.check([0], [1], [2500], 0, 0)
    s.check([0], [0], [2500], 0, 0)


@pytest.mark.parametrize("near", [1.0, 0.3, 0.05])
@pytest.mark.parametrize("n,H", [(20000, 1), (40000, 3), (7000, 100)])
def test_scores_close_together(near, n, H):
    """All, some or few of the scores alike in their first bits, some of them the same; clusters of all sizes."""
    s = State([n, 0], [0, n // 3], H=H, page=128, seed=n)
    far = s.rng.random(s.scores.shape) > near
    s.scores = (1 + s.rng.random(s.scores.shape) / 16).astype(np.float32)
    s.scores[s.rng.random(s.scores.shape) < 0.2] = 1.03125
    s.scores[far] = np.exp(4 * s.rng.standard_normal(int(far.sum()))).astype(np.float32)
    s.check([0], [1], [n // 3], 4, 32)


def test_pairs_left_alone():
    s = State([100, 100, 100, 100, 0, 0], [0, 0, 0, 0, 50, 50], seed=5)
    s.refs[s.table[1, 1]] = 2      # a page that would be written has another holder
    s.table[2, 3] = -1             # a page with tokens is not there
    s.table[5, 2] = 10**6          # a page to write is not there
    got = s.check([0, 1, 2, 3, 9, 0], [4, 1, 2, 5, 3, -1], [50] * 6, 1, 1, top=60)
    assert got.tolist() == [50, -1, -1, -1, -1, -1]
    # nothing is written in place where all stay: a shared page does not matter
    assert s.check([1], [1], [100], 1, 1).tolist() == [100]
    s.with_refs = False
    assert s.check([1], [1], [50], 1, 1).tolist() == [50]


def test_from_shared_pages():
    """Rows that share pages: one of them keeps some tokens in pages of its own, the others are as they were."""
    s = State([200, 200, 0], [0, 0, 90], seed=6)
    s.table[1, :12] = s.table[0, :12]
    s.refs[s.table[0, :12]] = 2
    s.check([1], [2], [90], 4, 16)


def test_lengths_outside_the_table():
    s = State([300, 0], [0, 300], page=16, seed=7)
    s.lens[:] = [10**6, -4]
    s.table[0, -1] = s.table[0, 0]
    s.check([0, 1], [1, 0], [40, 40], 1, 1)


def test_layers_and_strides():
    s = State([500, 0], [0, 200], H=3, layers=3, seed=8)

    def strided(x):
        wide = torch.full((3, 2, x.shape[2] + 5), math.nan, device="cuda")  # heads first, rows apart
        y = wide.transpose(0, 1)[:, :, : x.shape[2]]
        y.copy_(x)
        return y

    s.check([0], [1], [200], 4, 8, layer=1, scores=strided)


def test_no_pairs():
    s = State([5], [0])
    pages = s.upload()
    kept = akv.KeptTokens(torch.empty((0, 2, 4), dtype=torch.int32, device="cuda"), int32([]))
    akv.akv_paged_evict(s.p, pages, int32([]), int32([]), s.d["scores"], kept)
    akv.akv_pages_trim(s.p, pages, int32([]))


def test_graph_and_again():
    """A captured eviction, replayed on other contents."""
    s = State([900, 0], [0, 400], seed=10)
    pages = s.upload()
    kept = akv.KeptTokens(torch.empty((1, 2, 400), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"))
    src, dst, keep = int32([0]), int32([1]), int32([400])
    run = lambda: akv.akv_paged_evict(s.p, pages, src, dst, s.d["scores"], kept, keep=keep, sink=2, recent=20)  # noqa: E731
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    s.scores = s.rng.random(s.scores.shape).astype(np.float32)
    s.d["scores"].copy_(torch.from_numpy(s.scores))
    s.d["pool"].copy_(torch.from_numpy(s.pool))
    keep.fill_(123)
    g.replay()
    pool, sc = s.pool.copy(), s.scores.copy()
    tokens, count = plain.evict(s.p, pool[0].reshape(pool.shape[1], 2, -1), s.table, s.lens, s.refs, [0], [1], sc, [123], 2, 20, 400)
    assert np.array_equal(kept.tokens.cpu().numpy(), tokens) and kept.count.tolist() == [123]
    assert np.array_equal(s.d["pool"].cpu().numpy(), pool) and np.array_equal(s.d["scores"].cpu().numpy(), sc)


@pytest.mark.parametrize("page", [16, 128])
def test_trim(page):
    s = State([300, 1, 0, 128, 500, 40], [300] * 6, page=page, seed=11)
    s.lens[:] = [10, 1, 0, 128, 10**7, -3]
    s.refs[s.table[0, -2]] = 3
    s.table[3, -2] = 10**6  # (a number outside the pool is taken out of the table)
    pages = s.upload()
    rows = [0, 2, 3, 4, 5, 0, -1, 99]
    akv.akv_pages_trim(s.p, pages, int32(rows))
    table, refs = s.table.copy(), s.refs.copy()
    for r in sorted({r for r in rows if 0 <= r < 6}):
        n = min(max(int(s.lens[r]), 0), table.shape[1] * page)
        for j in range(-(-n // page), table.shape[1]):
            if 0 <= table[r, j] < len(refs):
                refs[table[r, j]] -= 1
            table[r, j] = -1
    assert np.array_equal(s.d["table"].cpu().numpy(), table) and np.array_equal(s.d["refs"].cpu().numpy(), refs)
    assert np.array_equal(s.d["lens"].cpu().numpy(), s.lens)
