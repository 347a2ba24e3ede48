"""Attention over pages that rows share: which rows share what, against a plain search, and the attention against 64-bit sums."""
import math

import numpy as np
import pytest

import paged_share_ref as plain
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, attend, params, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D, SM = 128, 1 / math.sqrt(128)


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def share_of(c, always=True):
    share = akv.PageShare(torch.full((4, len(c.lens_h)), -7, dtype=torch.int32, device="cuda"), always)
    akv.akv_pages_share(c.p, c.pages, share)
    return share


def check_share(c, share):
    want = plain.share(c.table.cpu().numpy(), c.lens.tolist(), c.p.page_tokens, c.pool.shape[1])
    assert np.array_equal(share.arrays.cpu().numpy(), want)
    return want


def grouped(p, groups, seed=0, fill=True):
    """Rows of groups (shared tokens, [own tokens of each row]); rows of different groups are mixed."""
    rows = [(g, s, n) for g, (s, own) in enumerate(groups) for n in own]
    order = np.random.default_rng(seed).permutation(len(rows))
    rows = [rows[i] for i in order]
    c = Cache(p, [s + n for _, s, n in rows], seed=seed)
    if fill:
        c.k, c.v = c.fill()
    c.unshared = c.table.clone()
    first = {}
    for b, (g, s, _) in enumerate(rows):
        if g in first:
            c.table[b, : s // p.page_tokens] = c.table[first[g], : s // p.page_tokens]
        first.setdefault(g, b)
    return c


def put(c, k, v):
    """Every row's tokens into pages of its own; then the rows share again."""
    shared = c.table.clone()
    c.table.copy_(c.unshared)
    n = torch.tensor(c.lens_h, dtype=torch.int32, device="cuda")
    c.lens.zero_()
    akv.akv_paged_append(c.p, c.pages, k, v, n_new=n)
    c.lens.copy_(n)
    c.table.copy_(shared)


def run(c, q, share=None, sm=SM, layer=0):
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:3], math.nan, device="cuda")
    akv.akv_paged_attn_shared(c.p, c.pages, q, out, share or share_of(c), lse=lse, sm_scale=sm, layer=layer)
    return out, lse


@pytest.mark.parametrize("page", [16, 64])
def test_which_rows_share(page):
    p = params(1, 1, page)
    c = grouped(p, [(300, [1, 5, 100, 0]), (0, [40]), (1000, [3, 900]), (64, [1]), (2000, [7] * 9), (10, [3, 2])], seed=page, fill=False)
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))
    want = check_share(c, share_of(c))
    assert (want[1] > 0).sum() >= 15
    # lengths that end earlier, nowhere, or outside the table; pages outside the pool
    c.lens[0], c.lens[3], c.lens[5], c.lens[7] = 5, 0, -3, 10**8
    c.table[2, 1], c.table[8, 0], c.table[9, 0] = -1, 10**6, -1
    check_share(c, share_of(c))
    c.table[:] = c.table[0]
    check_share(c, share_of(c))


def test_many_rows_and_pages():
    p = params(1, 1, 16)
    c = grouped(p, [(16 * 2500, [16 * k for k in range(5)]), (32, [0] * 400), (16, [1] * 300)], seed=3, fill=False)
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))
    check_share(c, share_of(c))


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 300])
def test_numbers_of_rows(rows):
    """Rows without tokens, of one page, of the same first pages, and pages outside the pool among them."""
    p = params(1, 1, 16)
    rng = np.random.default_rng(rows)
    c = Cache(p, [int(n) for n in rng.integers(0, 80, rows)], seed=rows)
    some = rng.integers(0, rows, rows)
    for b in range(rows):
        if rng.random() < 0.7:
            n = int(rng.integers(1, 6))
            c.table[b, :n] = c.table[int(some[b]), :n]
    c.table[rows // 2, 0] = -1
    c.table[rows // 3, 1] = 10**6
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))
    check_share(c, share_of(c))


GROUPS = [(300, [1, 5, 100, 0]), (0, [40]), (1000, [3, 140]), (64, [1]), (129, [7] * 3)]


@pytest.mark.parametrize("H,G,T,page,group,half,rotate", [
    (2, 4, 1, 64, 64, False, False), (2, 4, 1, 16, 64, False, True), (1, 8, 1, 32, 128, True, True), (3, 3, 2, 128, 64, True, False),
    (1, 1, 1, 16, 128, False, False), (2, 8, 5, 64, 64, False, True), (1, 4, 64, 16, 64, False, False), (1, 64, 1, 64, 64, False, True)])
def test_shared_attention(H, G, T, page, group, half, rotate):
    p = params(H, G, page, group, half, rotate)
    c = grouped(p, GROUPS, seed=H + G + T)
    q = queries(c, T, 1.0)
    out, lse = run(c, q)
    plain.check_shared(p, c, q, out, lse, SM)


def looking_for(c, T, share):
    q = queries(c, T, 1 - share).float()
    for b, n in enumerate(c.lens_h):
        lead = (c.table[:, 0] == c.table[b, 0]).nonzero()[0, 0]  # the row whose rows the shared pages hold
        at = torch.randint(0, max(1, n - T + 1), (T, c.p.n_q_heads), generator=c.gen, device="cuda")
        head = torch.arange(c.p.n_q_heads, device="cuda") // c.p.G
        q[b] += share * torch.where((at < 4096)[..., None], c.k[lead, at, head], c.k[b, at, head]).float()
    return q.to(c.k.dtype)


@pytest.mark.parametrize("rotate,group,half", [(False, 64, False), (True, 64, False), (True, 128, True)])
@pytest.mark.parametrize("groups,H,G", [
    ([(16000, [100, 1, 900])], 8, 4),                    # units cut over many CTAs
    ([(4096, [50] * 40)], 2, 8),                         # several blocks of 128 query rows
    ([(4099, [5, 7]), (900, [3] * 5), (8001, [11] * 4), (130, [1] * 20)], 4, 3)])
def test_long_prefixes(groups, H, G, rotate, group, half):
    p = params(H, G, 64, group, half, rotate)
    c = grouped(p, groups, seed=G)
    for share in (0.0, 0.5):
        q = looking_for(c, 1, share)
        out, lse = run(c, q)
        plain.check_shared(p, c, q, out, lse, SM)


def test_same_as_row_by_row():
    """No row shares: the attention of each row by itself, up to the order of sums."""
    p = params(2, 4, 32, 64, False, True)
    c = Cache(p, [500, 3, 0, 129], seed=2)
    c.fill()
    q = queries(c, 1, 1.0)
    out, lse = run(c, q)
    want, want_lse = attend(c, q)
    assert bool(torch.isneginf(lse[2]).all()) and bool((out[2] == 0).all())
    d = (out.double() - want.double()).abs()
    assert bool((d <= 2 * 2.0**-8 * want.double().abs() + 1e-5).all())
    plain.check_shared(p, c, q, out, lse, SM)


def test_drafts_longer_than_rows():
    """Query tokens that see nothing, or only some of the shared tokens."""
    p = params(1, 2, 16, 64, False, False)
    c = grouped(p, [(32, [0, 1, 2]), (16, [0, 0])], seed=4)
    q = queries(c, 40, 1.0)
    out, lse = run(c, q)
    plain.check_shared(p, c, q, out, lse, SM)


@pytest.mark.parametrize("sm", [0.0, -0.1, 3.0])
def test_scales(sm):
    p = params(1, 4, 64, 64, False, True)
    c = grouped(p, [(700, [3, 60])], seed=5)
    q = queries(c, 1, 1.0)
    out, lse = run(c, q, sm=sm)
    plain.check_shared(p, c, q, out, lse, sm)


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("k_scale,v_scale,q_scale", [(1e-3, 1e-3, 1e3), (1.0, 3e4, 1.0), (3e4, 1.0, 1e-4), (1.0, 1e-6, 1.0), (1e-5, 1.0, 3e4)])
def test_numbers_of_any_size(k_scale, v_scale, q_scale, rotate):
    p = params(1, 4, 64, 64, False, rotate)
    c = grouped(p, [(400, [30, 60, 9])], seed=6, fill=False)
    k, v = c.rows(max(c.lens_h))
    put(c, (k.float() * k_scale).to(k.dtype), (v.float() * v_scale).to(v.dtype))
    q = (queries(c, 1, 1.0).float() * q_scale).to(k.dtype)
    q[1] *= 2.0**-30  # a row far smaller than the others of its group
    out, lse = run(c, q)
    plain.check_shared(p, c, q, out, lse, SM)


def test_nan_tokens_and_queries():
    """A NaN among the shared tokens reaches the queries that see it, a NaN query itself alone; what nobody sees, nobody."""
    p = params(1, 2, 16, 64, False, False)
    c = grouped(p, [(320, [0, 0, 0])], seed=7, fill=False)
    k, v = c.rows(320)
    k[:, 319, 0, 3] = math.nan
    v[:, 318, 0, 100] = math.inf
    put(c, k, v)
    q = queries(c, 4, 1.0)
    q[1, 0, 1, 5] = math.nan
    out, lse = run(c, q)
    bad = torch.isnan(out).all(-1)
    want = torch.zeros_like(bad)
    want[:, 2:] = True    # they see token 318 or 319
    want[1, 0, 1] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(out).any(-1), want)
    q[1, 0, 1, 5] = 0
    c.lens.fill_(318)  # (the NaNs are behind the tokens held, in a shared page)
    out, lse = run(c, q)
    plain.check_shared(p, c, q, out, lse, SM)


def test_pages_outside_the_pool():
    p = params(1, 2, 16, 64, False, False)
    c = grouped(p, [(320, [5, 9]), (100, [4])], seed=8)
    share = share_of(c)
    rows = [b for b, n in enumerate(c.lens_h) if n > 200]
    c.table[rows, 3] = 10**6  # after the plan
    q = queries(c, 1, 1.0)
    out, lse = run(c, q, share)
    bad = torch.isnan(out).all(-1).all(-1).all(-1)
    assert bad.tolist() == [b in rows for b in range(3)]


def test_numbers_out_of_range_in_share():
    """Arrays that no plan gave: nothing outside the cache is read, and rows that they do not concern are right."""
    p = params(1, 2, 16, 64, False, False)
    c = grouped(p, [(320, [5, 9]), (100, [4])], seed=9)
    q = queries(c, 1, 1.0)
    alone = c.lens_h.index(104)
    good = share_of(c)
    want, want_lse = run(c, q, good)
    for row, value in ((0, 10**9), (0, -1), (1, -4), (1, 10**9), (2, 10**9), (2, -8), (3, -1), (3, 10**9)):
        arrays = good.arrays.clone()
        for b in range(3):
            if b != alone:
                arrays[row, b] = value
        if row == 3:
            arrays[3] = torch.where(good.arrays[3] == alone, good.arrays[3], value)
        out, lse = run(c, q, akv.PageShare(arrays, always=True))
        if row < 2:
            assert torch.equal(out[alone], want[alone])


def test_graph_follows_the_cache():
    """Append, plan and attention in one graph: rows fork, grow and take pages of their own between replays."""
    p = params(2, 4, 16, 64, False, True)
    c = Cache(p, [200, 0, 0], room=100, seed=10)
    c.fill()
    refs = torch.zeros(c.pool.shape[1], dtype=torch.int32, device="cuda")
    refs[c.table[0, :13].long()] = 1
    c.table[0, 13:], c.table[1:] = -1, -1
    pages = c.pages = akv.Pages(p, c.pool, c.table, c.lens, refs)
    k, v = c.rows(1)
    q = queries(c, 1, 1.0)
    one, missing = (c.lens > 0).int(), torch.zeros(1, dtype=torch.int32, device="cuda")
    arrays = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    share = akv.PageShare(arrays, always=True)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    ws = torch.empty(max(akv.akv_pages_workspace_size(pages), akv.akv_paged_attn_shared_workspace_size(p, pages)), dtype=torch.uint8, device="cuda")

    def step():
        akv.akv_pages_reserve(p, pages, one, missing, ws=ws)
        akv.akv_paged_append(p, pages, k, v, n_new=one)
        c.lens.add_(one)
        akv.akv_pages_share(p, pages, share, ws=ws)
        akv.akv_paged_attn_shared(p, pages, q, out, share, lse=lse, sm_scale=SM, ws=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        if i == 1:
            akv.akv_pages_fork(p, pages, torch.tensor([0, 0], dtype=torch.int32, device="cuda"), torch.tensor([1, 2], dtype=torch.int32, device="cuda"))
            one.fill_(1)
        g.replay()
        c.lens_h = c.lens.tolist()
        check_share(c, share)
        plain.check_shared(p, c, q, out, lse, SM)
    assert arrays[1].tolist() == [12] * 3


def test_again_and_on_another_stream():
    """The same bits each time, in order behind the stream's other work."""
    p = params(4, 8, 64, 64, False, True)
    c = grouped(p, [(9000, [40] * 20)], seed=11)
    q = queries(c, 1, 1.0)
    share = share_of(c)
    out, lse = run(c, q, share)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    with torch.cuda.stream(s):
        for _ in range(5):
            o, l = torch.empty_like(q), torch.empty_like(lse)
            akv.akv_paged_attn_shared(p, c.pages, q, o, share, lse=l, sm_scale=SM)
            outs.append((o, l))
    s.synchronize()
    for o, l in outs:
        assert torch.equal(o, out) and torch.equal(l, lse)


def test_layers_and_strides():
    p = params(2, 4, 64, 64, True, False)
    c = Cache(p, [300, 290], seed=12, layers=2)
    c.fill(layer=1)
    c.table[1, :4] = c.table[0, :4]
    q = queries(c, 2, 1.0)
    wide = torch.zeros((2, 8, 2, 3 * D), dtype=q.dtype, device="cuda").transpose(1, 2)[..., 1 : D + 1]
    wide.copy_(q)
    out = torch.full((2, 8, 2, 3 * D), math.nan, dtype=q.dtype, device="cuda").transpose(1, 2)[..., 3 : D + 3]
    lse = torch.empty(q.shape[:3], device="cuda")
    akv.akv_paged_attn_shared(p, c.pages, wide, out, share_of(c), lse=lse, sm_scale=SM, layer=1)
    plain.check_shared(p, c, q, out, lse, SM, layer=1)


@pytest.mark.parametrize("groups,H,G,T", [
    ([(16000, [40] * 40), (900, [3, 7]), (5000, [1, 2, 3])], 4, 8, 1),  # one group is worth it, the others are row by row
    ([(16000, [40] * 24), (9000, [5, 9]), (300, [1] * 3)], 4, 4, 4),    # pairs too, of 16 query rows
    ([(2000, [40] * 10), (900, [3, 7])], 2, 4, 1),                      # all groups are row by row
])
def test_where_it_pays(groups, H, G, T):
    p = params(H, G, 64, 64, False, True)
    c = grouped(p, groups, seed=13)
    q = queries(c, T, 1.0)
    out, lse = run(c, q, share_of(c, always=False))
    plain.check_shared(p, c, q, out, lse, SM)
