"""The operators of the paged cache in a row, as a serving loop uses them, and side by side on streams and in graphs."""
import math

import numpy as np
import pytest

import paged_exact as exact
import paged_share_ref as plain
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, params, queries
from test_paged_shared import grouped
from test_paged_weights import check as check_weights
from test_paged_weights import scores

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SM = 1 / math.sqrt(128)


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def int32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


class Loop:
    """Two prompts, four answers, four spare rows; every page is the pool's, handed out by the page operations."""

    def __init__(self, H, G, page, group, half, rotate, prompts=(700, 333), room=40, seed=0, always=True):
        self.p = params(H, G, page, group, half, rotate)
        self.c = c = Cache(self.p, [0] * 10, room=max(prompts) + room, seed=seed)
        c.table.fill_(-1)
        self.refs = torch.zeros(c.pool.shape[1], dtype=torch.int32, device="cuda")
        self.pages = c.pages = akv.Pages(self.p, c.pool, c.table, c.lens, self.refs)
        self.missing = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.share = akv.PageShare(torch.zeros((4, 10), dtype=torch.int32, device="cuda"), always)
        self.scores = scores(c)
        self.prompts = list(prompts)

    def put(self, n_new):
        k, v = self.c.rows(max(n_new))
        n = int32(n_new)
        akv.akv_pages_reserve(self.p, self.pages, n, self.missing)
        akv.akv_paged_append(self.p, self.pages, k, v, n_new=n)
        self.c.lens.add_(n)
        assert int(self.missing) == 0

    def attend(self, T):
        q = queries(self.c, T, 1.0)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        akv.akv_pages_share(self.p, self.pages, self.share)
        akv.akv_paged_attn_shared(self.p, self.pages, q, out, self.share, lse=lse, sm_scale=SM)
        self.c.lens_h = self.c.lens.tolist()
        plain.check_shared(self.p, self.c, q, out, lse, SM)
        want = plain.share(self.c.table.cpu().numpy(), self.c.lens_h, self.p.page_tokens, self.c.pool.shape[1])
        assert np.array_equal(self.share.arrays.cpu().numpy(), want)
        return q, lse

    def weigh(self, q, lse, decay):
        before = self.scores.clone()
        akv.akv_paged_weights(self.p, self.pages, q, lse, self.scores, was=self.scores, decay=decay, sm_scale=SM)
        check_weights(self.c, q, lse, self.scores, before, decay, before)

    def evict(self, src, dst, keep, sink, recent):
        """The pairs' tokens, scores and counts against the rules; lens follows, as a caller would have it."""
        c, H = self.c, self.p.n_kv_heads
        pool, sc = c.pool.cpu().numpy().copy(), self.scores.cpu().numpy().copy()
        top = max(keep)
        tokens, count = plain.evict(self.p, pool[0].reshape(pool.shape[1], H, -1), c.table.cpu().numpy(), c.lens.cpu().numpy(), self.refs.cpu().numpy(),
                                    src, dst, sc, keep, sink, recent, top)
        kept = akv.KeptTokens(torch.empty((len(src), H, top), dtype=torch.int32, device="cuda"), torch.empty(len(src), dtype=torch.int32, device="cuda"))
        akv.akv_paged_evict(self.p, self.pages, int32(src), int32(dst), self.scores, kept, keep=int32(keep), sink=sink, recent=recent)
        assert kept.count.tolist() == count.tolist() and min(count) >= 0
        assert np.array_equal(kept.tokens.cpu().numpy(), tokens)
        assert np.array_equal(c.pool.cpu().numpy(), pool) and np.array_equal(self.scores.cpu().numpy(), sc)
        c.lens[int32(dst).long()] = kept.count

    def add_up(self):
        table, refs = self.c.table.cpu(), self.refs.cpu()
        assert torch.equal(torch.bincount(table[table >= 0].long(), minlength=len(refs)).int(), refs)


@pytest.mark.parametrize("H,G,page,group,half,rotate", [(2, 4, 64, 64, False, True), (1, 3, 16, 128, True, False), (3, 8, 32, 64, False, False)])
def test_a_loop_within_a_budget(H, G, page, group, half, rotate):
    """Prompts, weights of their last tokens, eviction in place, answers that share what is left, a few steps of each kind, and
    eviction of the answers into rows of their own."""
    s = Loop(H, G, page, group, half, rotate, seed=page)
    s.put(s.prompts + [0] * 8)
    q, lse = s.attend(32)
    s.weigh(q, lse, 0.0)
    s.evict([0, 1], [0, 1], [300, 150], 4, 32)
    akv.akv_pages_trim(s.p, s.pages, int32([0, 1]))
    s.add_up()
    assert int((s.refs > 0).sum()) == sum(-(-n // page) for n in (300, 150))
    akv.akv_pages_fork(s.p, s.pages, int32([0, 0, 0, 1]), int32([2, 3, 4, 5]))
    s.scores[2:6] = s.scores[[0, 0, 0, 1]]
    for step, T in enumerate((1, 1, 4)):
        s.put([0, 0] + [T] * 4 + [0] * 4)
        q, lse = s.attend(T)
        assert s.share.arrays[1].tolist()[:6] == [300 // page] * 1 + [150 // page] + [300 // page] * 3 + [150 // page]
        s.weigh(q, lse, 0.9)
    keep = [200, 201, 306, 100]
    akv.akv_pages_reserve(s.p, s.pages, int32([0] * 6 + keep), s.missing)
    s.evict([2, 3, 4, 5], [6, 7, 8, 9], keep, 4, 16)
    akv.akv_pages_free(s.p, s.pages, int32([2, 3, 4, 5]))
    s.put([0] * 6 + [1] * 4)
    q, lse = s.attend(1)
    s.weigh(q, lse, 0.9)
    s.add_up()


def test_a_step_in_a_graph():
    """Reservation, append, plan, shared attention, weights and eviction in one graph; its replays do what the calls do."""
    s, t = (Loop(2, 4, 16, 64, False, True, seed=5) for _ in range(2))
    for x in (s, t):
        x.put(x.prompts + [0] * 8)
        akv.akv_pages_fork(x.p, x.pages, int32([0, 0, 1]), int32([2, 3, 4]))
        x.k, x.v = (y.clone() for y in x.c.rows(1))
        x.q = queries(x.c, 1, 1.0)
        x.new, x.src, x.dst, x.keep = int32([0, 0, 1, 1, 1, 0, 0, 0, 0, 0]), int32([2, 4]), int32([6, 7]), int32([100, 60])
        x.room = int32([0] * 6 + [100, 60, 0, 0])
        x.out, x.lse = torch.zeros_like(x.q), torch.zeros(x.q.shape[:3], device="cuda")
        x.kept = akv.KeptTokens(torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"))
        x.ws = torch.empty(max(akv.akv_pages_workspace_size(x.pages), akv.akv_paged_attn_shared_workspace_size(x.p, x.pages),
                               akv.akv_paged_weights_workspace_size(x.p, x.pages)), dtype=torch.uint8, device="cuda")

    def step(x):
        akv.akv_pages_reserve(x.p, x.pages, x.new, x.missing, ws=x.ws)
        akv.akv_paged_append(x.p, x.pages, x.k, x.v, n_new=x.new)
        x.c.lens.add_(x.new)
        akv.akv_pages_share(x.p, x.pages, x.share, ws=x.ws)
        akv.akv_paged_attn_shared(x.p, x.pages, x.q, x.out, x.share, lse=x.lse, sm_scale=SM, ws=x.ws)
        akv.akv_paged_weights(x.p, x.pages, x.q, x.lse, x.scores, was=x.scores, decay=0.9, sm_scale=SM, ws=x.ws)
        akv.akv_pages_reserve(x.p, x.pages, x.room, x.missing, ws=x.ws)
        akv.akv_paged_evict(x.p, x.pages, x.src, x.dst, x.scores, x.kept, keep=x.keep, sink=2, recent=8)

    for x in (s, t):
        step(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(t)
    for _ in range(3):
        step(s)
        g.replay()
    for name in ("pool", "table", "lens"):
        assert torch.equal(getattr(s.c, name), getattr(t.c, name)), name
    for name in ("out", "lse", "scores", "refs", "missing"):
        assert torch.equal(getattr(s, name), getattr(t, name)), name
    assert torch.equal(s.kept.tokens, t.kept.tokens) and s.kept.count.tolist() == t.kept.count.tolist() == [100, 60]


def test_graphs_that_share_a_workspace():
    """Two graphs of different sizes with one workspace, replayed in turn."""
    cases = []
    for seed, groups in ((1, [(5000, [10, 700]), (900, [1, 2, 3])]), (2, [(300, [20] * 40)])):
        p = params(2, 8, 64, 64, False, True)
        c = grouped(p, groups, seed=seed)
        cases.append((c, queries(c, 1, 1.0)))
    ws = torch.empty(max(max(akv.akv_pages_workspace_size(c.pages), akv.akv_paged_attn_shared_workspace_size(c.p, c.pages),
                             akv.akv_paged_weights_workspace_size(c.p, c.pages)) for c, _ in cases), dtype=torch.uint8, device="cuda")
    graphs = []
    for c, q in cases:
        out, lse, now = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda"), scores(c)
        share = akv.PageShare(torch.zeros((4, len(c.lens_h)), dtype=torch.int32, device="cuda"), always=not graphs)

        def step():
            akv.akv_pages_share(c.p, c.pages, share, ws=ws)
            akv.akv_paged_attn_shared(c.p, c.pages, q, out, share, lse=lse, sm_scale=SM, ws=ws)
            akv.akv_paged_weights(c.p, c.pages, q, lse, now, sm_scale=SM, ws=ws)

        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (out, lse, now)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append((g, (out, lse, now), want))
    for _, got, _ in graphs:
        for x in got:
            x.zero_()
    for _ in range(3):
        for g, _, _ in graphs:
            g.replay()
    for _, got, want in graphs:
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_on_streams_that_run_together():
    """Plans, shared attention and weights without a workspace of the caller's, on three streams with nothing between them."""
    p = params(4, 8, 64, 64, False, True)
    c = grouped(p, [(9000, [40] * 8), (700, [5, 9, 400])], seed=3)
    side = [torch.cuda.Stream() for _ in range(2)]
    streams = [None, side[0], side[1].cuda_stream]
    n = 24
    qs = [queries(c, 1 + i % 5) for i in range(n)]

    def run(which):
        outs, lses = [torch.zeros_like(q) for q in qs], [torch.zeros(q.shape[:3], device="cuda") for q in qs]
        now, shares = [scores(c) for _ in qs], [akv.PageShare(torch.zeros((4, len(c.lens_h)), dtype=torch.int32, device="cuda")) for _ in qs]
        torch.cuda.synchronize()
        for i, q in enumerate(qs):
            at = which(i)
            akv.akv_pages_share(p, c.pages, shares[i], stream=at)
            akv.akv_paged_attn_shared(p, c.pages, q, outs[i], shares[i], lse=lses[i], sm_scale=SM, stream=at)
            akv.akv_paged_weights(p, c.pages, q, lses[i], now[i], sm_scale=SM, stream=at)
        torch.cuda.synchronize()
        return outs + lses + now

    want = run(lambda i: None)
    for shift in range(3):
        assert all(torch.equal(x, y) for x, y in zip(run(lambda i: streams[(i + shift) % 3]), want))


def test_weights_add_up_to_one_a_query_row():
    """What shared attention's lse makes of the weights: a query head's sum to one, so a KV head's to the number of its query rows."""
    p = params(2, 4, 64, 64, False, False)
    c = grouped(p, [(3000, [30, 1, 77])], seed=8)
    q = queries(c, 2, 1.0)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    share = akv.PageShare(torch.zeros((4, 3), dtype=torch.int32, device="cuda"))
    akv.akv_pages_share(p, c.pages, share)
    akv.akv_paged_attn_shared(p, c.pages, q, out, share, lse=lse, sm_scale=SM)
    now = scores(c)
    akv.akv_paged_weights(p, c.pages, q, lse, now, sm_scale=SM)
    E = exact.Exact(p, c.pool[0], c.table, c.lens.tolist())
    _, want_lse, _, tol_lse = plain.attend_shared(E, q, SM)
    total, tol = plain.weights(E, q, lse, SM)
    for b, n in enumerate(c.lens_h):
        for h in range(2):
            rows = slice(4 * h, 4 * h + 4)
            # each weight to its bound, lse to its own: e^(error) - 1 of the row's sum of one
            bound = float(tol[b][h].sum()) + 2.0**-22 * float(total[b][h].sum()) + 1.01 * float(tol_lse[b, :, rows].sum())
            assert abs(float(now[b, h, :n].double().sum()) - 8) <= bound
