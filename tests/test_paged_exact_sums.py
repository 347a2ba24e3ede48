"""Weights and shared attention on numbers whose sums on the tensor cores are exact, against bounds of the few roundings that are left.

Codes are random; scales, minima and queries are such that products and their sums are whole multiples of one unit below 2^24 of it, however
they are added up.  What is left are fp32 steps behind the sums, u = 2^-24 of a partial result each, e^x (2^-22) and the sum over query rows:
some 1e-6.  A low half of a query or a key, or the low part of lse, is 1e-4 and more of a weight here; that the bound tells them apart is
asserted with references that lack them."""
import math

import pytest

import paged_exact as exact
import paged_ref as ref
import paged_share_ref as plain
import paper_2608_02901_gb300 as akv
from test_paged_cache import Cache, dtype, params
from test_paged_shared import grouped, share_of
from test_paged_weights import scores

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D, U, LOG2E, LN2 = 128, 2.0**-24, math.log2(math.e), math.log(2)


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def write(c, a, m):
    """Random codes and one scale and minimum for all tokens, as the pages' bytes."""
    p = c.p
    sub = 2048 + 128 * (D // p.group)
    c.pool.copy_(torch.randint(0, 256, c.pool.shape, generator=c.gen, device="cuda", dtype=torch.uint8))
    blocks = c.pool.view(c.pool.shape[1], p.n_kv_heads, ref.block_bytes(p))
    words = blocks[..., : p.page_tokens // 16 * sub].unflatten(-1, (-1, sub))[..., 2048:]
    words.copy_(torch.tensor([a, m], dtype=torch.float16, device="cuda").view(torch.uint8).repeat(32 * (D // p.group)))
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))


def two_dimensions(c, T):
    """Queries of 2 in one dimension and 2^-11 in another: rotated, +-(1 +- 2^-12) / 8, of which a half holds the first bit."""
    q = torch.zeros((len(c.lens_h), T, c.p.n_q_heads, D), device="cuda")
    i = torch.rand(q.shape, generator=c.gen, device="cuda").argsort(-1)
    return q.scatter(-1, i[..., :1], 2.0).scatter(-1, i[..., 1:2], 2.0**-11).to(dtype(c.p))


def one_large(c, T):
    """Queries of 128 in one dimension and multiples of 2^-6 up to 2 in the others."""
    q = torch.randint(-128, 129, (len(c.lens_h), T, c.p.n_q_heads, D), generator=c.gen, device="cuda") * 2.0**-6
    i = torch.randint(0, D, (*q.shape[:3], 1), generator=c.gen, device="cuda")
    return q.scatter(-1, i, 128.0).to(dtype(c.p))


def few_high(x, p):
    """High half of a query of few rows: whole multiples of 2^-11 of the power of two above its largest value."""
    step = 2.0 ** (math.floor(math.log2(float(x.abs().max()))) + 1 - 11)
    return (x / step).round() * step


def weights(E, q, lse, sm, high=None, coarse=False):
    """Weights' sums [B][H] of [n] and their bound.

    In log2 units, L the logit, l the lse, A the sum over groups of a logit's part: d + rest, two steps a group, the step that joins l, and the
    scale's own rounding: u (4 A + L + l + |L - l|) with a few rows; of many rows 5 A + 8 l (l is in the partial sums; three parts of it are
    added up with two cuts at 2 u of it)."""
    p = E.p
    B, T, Hq, _ = q.shape
    G = Hq // p.n_kv_heads
    total, tol = [], []
    for b, n in enumerate(E.lens):
        for h in range(p.n_kv_heads):
            r = plain.Rows(E, b, h, n)
            k = r.kc * r.ka + r.km  # as stored
            w, e = (torch.zeros(n, dtype=torch.float64, device=q.device) for _ in range(2))
            for t in range(T):
                sees = max(0, n - T + 1 + t)
                for g in range(G):
                    x = q[b, t, h * G + g].double()
                    x = (x * E.s) @ E.h / 16 if p.rotate else x
                    l = lse[b, t, h * G + g].double() * LOG2E
                    if coarse:
                        l = (l * 256).round() / 256
                    L = k @ (high(x, p) if high else x) * (sm * LOG2E)
                    A = (k * x).unflatten(-1, (-1, p.group)).sum(-1).abs().sum(-1) * (sm * LOG2E)
                    y = torch.exp2(L - l)[:sees]
                    w[:sees] += y
                    rel = LN2 * U * (5 * A + L.abs() + 8 * l.abs() + (L - l).abs()) + 2.0**-22
                    e[:sees] += 1.01 * y * rel[:sees]
            total.append(w)
            tol.append(e + T * G * U * w + 1e-37)
    H = p.n_kv_heads
    return [total[b * H : (b + 1) * H] for b in range(B)], [tol[b * H : (b + 1) * H] for b in range(B)]


@pytest.mark.parametrize("G,T,group,rotate", [
    (4, 1, 64, True), (8, 1, 128, True), (4, 1, 64, False), (8, 1, 128, False), (4, 4, 64, True), (16, 1, 128, False), (8, 4, 64, True), (4, 64, 128, True),
    (5, 7, 64, False)])
def test_weights(G, T, group, rotate):
    p = params(2, G, 32, group, False, rotate)
    c = Cache(p, [700, 129], seed=G + T)
    write(c, 0.25, -1.875)
    few = T * G <= 16
    q, sm = (two_dimensions(c, T), 1.0) if rotate else (one_large(c, T), 2.0**-7)
    lse = torch.empty(q.shape[:3], device="cuda")
    akv.akv_paged_attn(p, c.pages, q, torch.empty_like(q), lse=lse, sm_scale=sm)
    now = scores(c)
    akv.akv_paged_weights(p, c.pages, q, lse, now, sm_scale=sm)
    E = exact.Exact(p, c.pool[0], c.table, c.lens.tolist())
    total, tol = weights(E, q, lse, sm)
    mistakes = []
    if few:
        mistakes = [weights(E, q, lse, sm, high=few_high)[0], weights(E, q, lse, sm, coarse=True)[0]]
    elif rotate:
        mistakes = [weights(E, q, lse, sm, high=lambda x, _: x.half().double())[0]]
    for b, n in enumerate(E.lens):
        for h in range(2):
            d = (now[b, h, :n].double() - total[b][h]).abs()
            assert bool((d <= tol[b][h]).all()), float((d / tol[b][h]).max())
            for wrong in mistakes:
                assert float(((wrong[b][h] - total[b][h]).abs() / tol[b][h]).max()) > 10


def shared_lse(E, q, sm, wrong=False):
    """lse and its bound.  In log2 units of a logit L of weight w, M the largest: u (2 L + 2 M + 15 + |L - M|); sums of at most 64 terms a
    thread, two e^x, log2 (2 u of it) and the steps from it to lse."""
    p = E.p
    B, T, Hq, _ = q.shape
    G = Hq // p.n_kv_heads
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(lse)
    for b, n in enumerate(E.lens):
        for h in range(p.n_kv_heads):
            r = plain.Rows(E, b, h, n)
            k = r.kc * r.ka + r.km
            if wrong and not p.rotate:  # keys without their low halves
                k = (((2 * r.kc - 15) * r.ka).half().double() + (2 * r.km + 15 * r.ka)) / 2
            for t in range(T):
                sees = n - T + 1 + t
                if sees <= 0:
                    continue
                for g in range(G):
                    x = q[b, t, h * G + g].double()
                    x = (x * E.s) @ E.h / 16 if p.rotate else x
                    if wrong and p.rotate:
                        x = x.half().double()
                    L = (k @ x * (sm * LOG2E))[:sees]
                    M = L.max()
                    w = torch.softmax(L * LN2, 0)
                    y = lse[b, t, h * G + g] = torch.logsumexp(L * LN2, 0)
                    tol[b, t, h * G + g] = 1.01 * (LN2 * U * (w * (2 * L.abs() + 2 * M.abs() + 15 + (L - M).abs())).sum()
                                                   + 64 * U + 2.0**-21 + 4 * U * (y.abs() + M.abs() + 10))
    return lse, tol


@pytest.mark.parametrize("G,T,group,rotate", [(4, 16, 64, False), (8, 16, 128, True), (3, 5, 128, False), (2, 16, 64, True)])
def test_shared_lse(G, T, group, rotate):
    """Queries that see a token or a few, so that nothing averages out."""
    p = params(2, G, 16, group, False, rotate)
    c = grouped(p, [(16, [0, 0, 0]), (48, [0] * 4), (112, [0] * 2)], seed=G + T, fill=False)
    if rotate:
        write(c, 0.25, -1.875)
        q, sm = two_dimensions(c, T), 1.0
    else:
        a = 0.25 * (1 + 2.0**-10)
        write(c, a, float(torch.tensor(-7.5 * a).half()))
        q = torch.randint(-1, 2, (len(c.lens_h), T, p.n_q_heads, D), generator=c.gen, device="cuda").to(dtype(p))
        sm = 1 / 8
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    akv.akv_paged_attn_shared(p, c.pages, q, out, share_of(c), lse=lse, sm_scale=sm)
    E = exact.Exact(p, c.pool[0], c.table, c.lens.tolist())
    want, tol = shared_lse(E, q, sm)
    some = torch.isfinite(want)
    assert torch.equal(torch.isneginf(lse), ~some) and int(some.sum()) > 50
    d = (lse.double() - want)[some].abs()
    assert bool((d <= tol[some]).all()), float((d / tol[some]).max())
    wrong, _ = shared_lse(E, q, sm, wrong=True)
    assert float(((wrong - want)[some].abs() / tol[some]).max()) > 5
