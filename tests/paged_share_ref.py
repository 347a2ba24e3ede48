"""Plain forms for rows that share pages, accumulated weights and eviction: 64 bits or whole numbers, one thing at a time.

Attention and weights in 64 bits on the GPU, from the pages' bytes, each with the bound of what a kernel of the documented
roundings may be off by (first order; u = 2^-24)."""
import math

import numpy as np
import torch

import paged_exact as exact
import paged_ref as ref

D = 128


# ---- which rows share ----------------------------------------------------------------------


def share(table, lens, P, n_pages):
    """leader, pages, size, order of numpy tables."""
    B, most = table.shape
    held = [-(-min(max(int(n), 0), most * P) // P) for n in lens]
    first = [int(table[b, 0]) if held[b] and 0 <= table[b, 0] < n_pages else -1 for b in range(B)]
    leader = [min(j for j in range(B) if first[j] == first[b]) if first[b] >= 0 else b for b in range(B)]
    pages, size = [], []
    for b in range(B):
        group = [j for j in range(B) if leader[j] == leader[b]]
        n = 0
        if len(group) > 1:
            least = min(held[j] for j in group)
            while n < least and len({int(table[j, n]) for j in group}) == 1 and 0 <= table[group[0], n] < n_pages:
                n += 1
        pages.append(n)
        size.append(len(group))
    order = sorted(range(B), key=lambda b: (leader[b], b))
    return np.array([leader, pages, size, order], np.int32)


# ---- attention and weights -------------------------------------------------------------------


class Rows:
    """One request's and head's cached rows: codes, scales and minima as 64-bit numbers, keys and values rotated back."""

    def __init__(self, E, b, h, n):
        p = self.p = E.p
        codes, a, m = exact.rows_of_pages(p, E.blocks[E.table[b, : -(-n // p.page_tokens)].long()])
        spread = [exact.spread_groups(x, p) for x in (a[0, :n, h], a[1, :n, h], m[0, :n, h], m[1, :n, h])]
        self.ka, self.va, self.km, self.vm = spread
        self.kc, self.vc = codes[0, :n, h], codes[1, :n, h]
        self.k_mag = self.kc * self.ka + self.km.abs()
        self.v = self.vc * self.va + self.vm
        self.k_back, self.v_back = E.back(self.kc * self.ka + self.km), E.back(self.v)


def logits(E, r, x, sm_scale, products):
    """One query row's logits, and their bound.

    Products of operands are exact.  `products` tensor-core products of 16 terms are added up, and one cuts at most 17 terms at 2^-23 of
    the largest: products * 17 * 2^-23 of the sum of magnitudes M_i = |sm| sum |q'| (a c + |m|); the fp32 steps after them (and the
    three-part sums of q') 2^-21 of it.  A rotated query has 7 fp32 stages and a low half that ends 2^-22 below: 2^-20 of
    sum |q| / 16 in each dimension."""
    p = E.p
    l = (r.k_back @ x) * sm_scale
    xr = (x * E.s) @ E.h / 16 if p.rotate else x
    el = (products * 17 * 2.0**-23 + 2.0**-21) * abs(sm_scale) * (r.k_mag @ xr.abs())
    if p.rotate:
        el = el + 2.0**-20 * abs(sm_scale) * x.abs().sum() / 16 * r.k_mag.sum(-1)
    return l, el


def attend_shared(E, q, sm_scale):
    """out, lse and their bounds for every query row of the cache E (paged_exact.Exact).

      weights  a share of a weight is rounded to fp16: 2^-11 of what it brings (either w a with the codes, or w with the whole value, which
               bounds both), and 2^-29 of the row's largest for each token
      values   fp16(m + c a): 2^-11 of each, 2^-25 below the normal range; where a sub-block has a scale above 2048 or a minimum
               beyond 16384, 2^-20
      sums     of at most 2^13 tiles' steps a thread, four at a time, over parts of at most 2^9 steps here: 2^9 u of sum w |v|
               and of the normaliser; 2^-14 of sum w |v| on tensor cores
      output   half an ulp of its type"""
    p = E.p
    B, T, Hq, _ = q.shape
    G = Hq // p.n_kv_heads
    q = q.double()
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    tol_lse = torch.zeros_like(lse)
    for b, n in enumerate(E.lens):
        if n <= 0:
            continue
        for h in range(p.n_kv_heads):
            r = Rows(E, b, h, n)
            coarse = bool((r.va > 2048).any() or (r.vm.abs() > 16384).any())
            for t in range(T):
                sees = n - T + 1 + t
                if sees <= 0:
                    continue
                for g in range(G):
                    hq = h * G + g
                    x = q[b, t, hq]
                    l, el = logits(E, r, x, sm_scale, 25)
                    l, el = l[:sees], el[:sees]
                    lse[b, t, hq] = torch.logsumexp(l, 0)
                    w = torch.exp(l - lse[b, t, hq])
                    vb, v = r.v_back[:sees], r.v[:sees]
                    y = w @ vb
                    out[b, t, hq] = y
                    tol_lse[b, t, hq] = (w * el).sum() + 2.0**9 * 2.0**-24 + 2.0**-22 * lse[b, t, hq].abs() + 1e-6
                    total = (lambda z: z.sum() / 16) if p.rotate else (lambda z: z)
                    mag = w @ v.abs()
                    e = (w * el) @ (vb - y).abs() + 2.0**-11 * (w @ (vb.abs() + exact_codes(E, r, sees)))
                    e = e + total(2.0**-11 * mag + (2.0**-20 if coarse else 2.0**-25)) + total((2.0**-15 + 2.0**-14) * mag)
                    e = e + total(sees * 2.0**-29 * (w[:, None] * v.abs()).amax(0)) + 2.0**-15 * y.abs()
                    half_ulp = y.abs() * 2.0**-11 + 2.0**-25 if p.half else y.abs() * 2.0**-8
                    tol[b, t, hq] = e * 1.02 + half_ulp + 1e-30
    return out, lse, tol, tol_lse


def exact_codes(E, r, sees):
    """What a rounded w a of each group touches: the codes' part of a value, rotated back group by group."""
    p = E.p
    parts = []
    for g in range(D // p.group):
        one = torch.zeros(D, dtype=torch.float64, device=r.v.device)
        one[g * p.group : (g + 1) * p.group] = 1
        parts.append(E.back(r.vc[:sees] * r.va[:sees] * one).abs())
    return torch.stack(parts).sum(0)


def check_shared(p, c, q, out, lse, sm_scale, layer=0):
    want, want_lse, tol, tol_lse = attend_shared(exact.Exact(p, c.pool[layer], c.table, c.lens.tolist()), q, sm_scale)
    got = out.double()
    assert bool(torch.isfinite(got).all())
    share_ = float(((got - want).abs() / tol.clamp_min(1e-30)).max())
    assert share_ <= 1, share_
    empty = torch.isneginf(want_lse)
    assert bool((torch.isneginf(lse) == empty).all()) and bool((got[empty] == 0).all())
    d = (lse.double() - want_lse)[~empty].abs()
    assert bool((d <= tol_lse[~empty]).all()), float((d / tol_lse[~empty]).max())
    return share_


def weights(E, q, lse, sm_scale):
    """sum of exp(l - lse) for each request, head and token [B][H] of [n], and its bound: e^x's 2^-22, the logit's bound, lse in
    log2 units (2^-23 of it), sums of T G terms; a logit's fp32 reference 2^-23 of its size."""
    p = E.p
    B, T, Hq, _ = q.shape
    G = Hq // p.n_kv_heads
    q = q.double()
    total, tol = [], []
    for b, n in enumerate(E.lens):
        for h in range(p.n_kv_heads):
            w, e = (torch.zeros(n, dtype=torch.float64, device=q.device) for _ in range(2))
            if n > 0:
                r = Rows(E, b, h, n)
                for t in range(T):
                    sees = max(0, n - T + 1 + t)
                    for g in range(G):
                        ref_ = lse[b, t, h * G + g].double()
                        if not bool(torch.isfinite(ref_)):
                            continue
                        l, el = logits(E, r, q[b, t, h * G + g], sm_scale, 25)
                        x = torch.exp(l - ref_)[:sees]
                        w[:sees] += x
                        e[:sees] += x * (1.05 * el[:sees] + 2.0**-22 * (ref_.abs() + l[:sees].abs()) + 2.0**-21 + T * G * 2.0**-24)
            total.append(w)
            tol.append(e)
    H = p.n_kv_heads
    return [total[b * H : (b + 1) * H] for b in range(B)], [tol[b * H : (b + 1) * H] for b in range(B)]


# ---- eviction --------------------------------------------------------------------------------


def kept_tokens(scores, m, sink, recent):
    """The m tokens kept of scores [n], ascending: forced ones first, then the highest, ties to the lower; NaN lowest."""
    n = len(scores)
    forced = [i for i in range(n) if i < sink or i >= n - recent]
    s = np.where(np.isnan(scores), -np.inf, scores.astype(np.float64))
    isnan = np.isnan(scores)
    rest = sorted((i for i in range(n) if sink <= i < n - recent), key=lambda i: (-s[i], isnan[i], i))
    return sorted((forced + rest)[:m])


def token_places(p, i):
    """Places of the bytes of token i of a page in a head's block."""
    ng = D // p.group
    k, at = i % 16, i // 16 * (2048 + 128 * ng)
    keys = [64 * k + j for j in range(64)]
    values = []
    for s in range(2):
        for g in range(8):
            for u in range(2):
                for half in range(2):
                    values.append(1024 + 512 * (k // 8) + 16 * (4 * g + k % 8 // 2) + 4 * (2 * s + u) + 2 * (k % 2) + half)
    return np.array([at + x for x in keys + values + [2048 + 8 * ng * k + j for j in range(8 * ng)]])


def evict(p, pool, table, lens, refs, src, dst, scores, keep, sink, recent, top):
    """pool [n_pages][H][block] (uint8) and scores [rows][H][cap] are changed; returns tokens and count."""
    P, H = p.page_tokens, p.n_kv_heads
    n_pages, (rows, most) = pool.shape[0], table.shape
    tokens, count = np.full((len(src), H, top), -1, np.int32), np.full(len(src), -1, np.int32)
    places = [token_places(p, i) for i in range(P)]
    was = pool.copy()
    old = scores.copy()
    for i, (a, b) in enumerate(zip(src, dst)):
        if not (0 <= a < rows and 0 <= b < rows):
            continue
        n = min(max(int(lens[a]), 0), most * P)
        m = min(n, min(max(int(keep[i]) if keep is not None else top, 0), top))
        stays = a == b and m == n
        of = lambda r, j: int(table[r, j]) if 0 <= table[r, j] < n_pages else -1  # noqa: E731
        if any(of(a, j) < 0 for j in range(-(-n // P))):
            continue
        if any(of(b, j) < 0 or (not stays and refs is not None and refs[of(b, j)] > 1) for j in range(-(-m // P))):
            continue
        count[i] = m
        for h in range(H):
            kept = kept_tokens(old[a, h, :n], m, sink, recent)
            tokens[i, h, :m] = kept
            for to, t in enumerate(kept):
                pool[of(b, to // P), h, places[to % P]] = was[of(a, t // P), h, places[t % P]]
                scores[b, h, to] = old[a, h, t]
    return tokens, count


block_bytes = ref.block_bytes
