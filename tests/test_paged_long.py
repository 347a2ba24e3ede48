"""The paged cache's attention against 64-bit sums where a CTA goes over many tiles, rotated and not: the ring of stages
wraps several times, units are cut anywhere and joined.  The bound is each output's own (paged_exact)."""
import math

import pytest

import paper_2608_02901_gb300 as akv
import paged_exact as exact
import paged_ref as ref
from test_paged_cache import Cache, attend, params, queries, selection

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def looking_for(c, k, T, share):
    """Queries of which each is near one key of its own request and head, anywhere in it: a tile that is left out, taken twice or
    taken for another one shows in whole rows."""
    p = c.p
    B, Hq, G = len(c.lens_h), p.n_q_heads, p.G
    q = queries(c, T, 1 - share).float()
    for b, n in enumerate(c.lens_h):
        at = torch.randint(0, max(1, n - T + 1), (T, Hq), generator=c.gen, device="cuda")
        q[b] += share * k[b, at, torch.arange(Hq, device="cuda") // G].float()
    return q.to(k.dtype)


# tiles of all units over 304 CTAs of 8 rows a unit (4 stages), 152 of 16 (6 stages): 10 to 44 tiles a CTA
@pytest.mark.parametrize("share", [0.0, 0.5])
@pytest.mark.parametrize("H,G,T,page,group,half,rotate", [
    (8, 4, 1, 64, 64, False, True), (8, 4, 1, 16, 64, False, False), (8, 8, 1, 64, 128, False, True), (8, 1, 1, 128, 64, True, True),
    (8, 4, 4, 64, 128, True, False), (8, 8, 2, 32, 64, False, True), (4, 12, 1, 64, 64, True, True)])
def test_many_tiles_a_cta(H, G, T, page, group, half, rotate, share):
    p = params(H, G, page, group, half, rotate)
    c = Cache(p, [8 // H * 30001, 8 // H * 21000, 77], seed=H * G + T)
    k, _ = c.fill()
    q = looking_for(c, k, T, share)
    out, lse = attend(c, q)
    exact.check(p, c, q, out, lse, 1 / math.sqrt(D))


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("lens,G", [([9000, 5, 6001, 2500], 4), ([700, 129, 128, 1], 3), ([20000], 8)])
def test_joined_units(lens, G, rotate):
    p = params(2, G, 64, 64, False, rotate)
    c = Cache(p, lens, seed=G)
    k, _ = c.fill()
    for share in (0.0, 0.5):
        q = looking_for(c, k, 1, share)
        exact.check(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("T,top", [(1, 200), (3, 60)])
def test_many_tiles_of_kept_pages(T, top):
    p = params(8, 4, 64, 64, False, True, bounds=True)
    c = Cache(p, [30000, 17001, 900, 13], seed=top)
    k, _ = c.fill()
    q = looking_for(c, k, T, 0.4)
    sel = selection(c, T, top)
    akv.akv_paged_select(p, c.pages, q, sel, sink=1, recent=2)
    pages, count = sel.pages.cpu(), sel.count.cpu()
    kept = [[[pages[b, t, h, : count[b, t, h]].tolist() for h in range(8)] for t in range(T)] for b in range(4)]
    exact.check(p, c, q, *attend(c, q, sel=sel), 1 / math.sqrt(D), kept=kept)


def test_the_bound_sees_what_it_should():
    """Planted in the 64-bit form: a wrong tile's worth of values, outputs of zeros, a third off, are all beyond the bound."""
    p = params(2, 4, 64, 64, False, True)
    c = Cache(p, [9000], seed=4)
    k, _ = c.fill()
    q = looking_for(c, k, 1, 0.0)
    want, lse, tol, _ = exact.Exact(p, c.pool[0], c.table, [9000]).attend(q, 1 / math.sqrt(D))
    assert float((want.abs() > tol).double().mean()) > 0.85  # zeros
    assert float((want.abs() / 3 > tol).double().mean()) > 0.6  # a third off
    fewer, _, _, _ = exact.Exact(p, c.pool[0], c.table, [9000 - 9000 // 16]).attend(q, 1 / math.sqrt(D))
    assert bool(((fewer - want).abs() > tol).any(-1).all())  # the last sixteenth left out


@pytest.mark.parametrize("page,group,rotate", [(32, 64, True), (16, 128, True), (64, 64, False)])
def test_rows_of_forked_requests_are_the_codecs(page, group, rotate):
    """A prompt and two answers to it read back: a row is at most half a step a group away from what was given.  In the units of
    what is quantised the error of a dimension is at most a / 2 (the code's rounding; a minimum rounded up cuts off what lies below
    it, 2^-11 of its size), and the rotation back keeps an error's norm but for sqrt(128) / 16."""
    p = akv.PagedParams(n_kv_heads=2, n_q_heads=4, page_tokens=page, group=group, rotate=rotate, rot_seed=77)
    n_pages, most = 60, 12
    dev = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, n_pages, akv.akv_paged_page_bytes(p)), dtype=torch.uint8, device="cuda")
    table, lens = torch.full((3, most), -1, **dev), torch.zeros(3, **dev)
    refs, missing = torch.zeros(n_pages, **dev), torch.zeros(1, **dev)
    pages = akv.Pages(p, pool, table, lens, refs)
    gen = torch.Generator(device="cuda").manual_seed(page)
    given = [[], [], []]

    def add(n):
        n = torch.tensor(n, **dev)
        akv.akv_pages_reserve(p, pages, n, missing)
        x = torch.randn((2, 3, int(n.max()), 2, D), generator=gen, device="cuda").to(torch.bfloat16)
        akv.akv_paged_append(p, pages, x[0], x[1], n_new=n)
        lens.add_(n)
        for r in range(3):
            if int(n[r]):
                given[r].append(x[:, r, : int(n[r])])

    add([77, 0, 0])
    akv.akv_pages_fork(p, pages, torch.tensor([0, 0], **dev), torch.tensor([1, 2], **dev))
    given[1], given[2] = list(given[0]), list(given[0])
    for n in ([1, 1, 0], [0, 3, 20], [1, 0, 1], [5, 5, 5]):
        add(n)
    assert int(missing) == 0
    for r in range(3):
        x = torch.cat(given[r], 1).double()  # [2][n][H][128]
        n = x.shape[1]
        assert n == int(lens[r])
        K, V = (torch.empty((3, n, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        akv.akv_paged_read(p, pages, K, V)
        got = torch.stack((K[r], V[r])).double()
        _, a, m = exact.rows_of_pages(p, pool[0][table[r, : -(-n // page)].long()].view(-1, 2, ref.block_bytes(p)))
        a, m = (y[:, :n].repeat_interleave(group, -1) for y in (a, m))
        each = a / 2 * (1 + 2.0**-10) + 2.0**-11 * m.abs()
        norm = each.square().sum(-1).sqrt() * (math.sqrt(D) / 16 if rotate else 1)
        err = ((got - x).abs() - 2.0**-8 * got.abs()).clamp_min(0).square().sum(-1).sqrt()  # (bf16 rows)
        assert bool((err <= norm).all()), float((err / norm).max())
        assert float(norm.max()) < 0.25 * float(x.square().sum(-1).sqrt().mean())  # far from the rows themselves
