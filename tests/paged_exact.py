"""Attention over the paged 4-bit cache in 64 bits on the GPU, and what a kernel of the documented roundings may be off by.

Rows come from the pages' bytes as the header lays them out, whole arrays at a time.  The bound is carried through each output
with the weights of its own tokens, so that it stays far below the outputs for long requests, rotated or not."""
import math

import torch

import paged_ref as ref

D = 128


def rows_of_pages(p, blocks):
    """Blocks [N][H][bytes] of pages -> codes [2][N * P][H][128] (key, value) and scales, minima [2][N * P][H][NG], fp64."""
    N, H, _ = blocks.shape
    ng, P = D // p.group, p.page_tokens
    sub = 2048 + 128 * ng
    x = blocks[:, :, : P // 16 * sub].reshape(N, H, P // 16, sub)
    dev = blocks.device
    d, i = torch.arange(D, device=dev), torch.arange(16, device=dev)[:, None]
    at = (64 * i + 4 * (4 * (d // 8 % 4) + d // 32) + d % 8 // 2,
          1024 + 512 * (i // 8) + 16 * (4 * (d // 8 % 8) + i % 8 // 2) + 4 * (2 * (d // 64) + d // 4 % 2) + 2 * (i % 2) + d % 4 // 2)
    codes = torch.stack([(x[..., b] >> 4 * (d % 2).to(torch.uint8) & 15).double() for b in at])  # [2][N][H][P/16][16][128]
    codes = codes.permute(0, 1, 3, 4, 2, 5).reshape(2, N * P, H, D)
    w = x[..., 2048:].contiguous().view(torch.float16).double().view(N, H, P, 2, ng, 2)
    w = w.permute(3, 0, 2, 1, 4, 5).reshape(2, N * P, H, ng, 2)
    return codes, w[..., 0], w[..., 1]


def spread_groups(x, p):
    return x.repeat_interleave(p.group, -1)


class Exact:
    def __init__(self, p, pool_layer, table, lens):
        self.p = p
        self.lens = [int(n) for n in lens]
        self.blocks = pool_layer.reshape(pool_layer.shape[0], p.n_kv_heads, ref.block_bytes(p))
        self.table = table
        dev = pool_layer.device
        self.h = torch.from_numpy(ref.hadamard()).to(dev)
        self.s = torch.from_numpy(ref.signs(p.rot_seed)).to(dev)

    def back(self, v):
        return v @ self.h / 16 * self.s if self.p.rotate else v

    def attend(self, q, sm_scale, kept=None):
        """q [B][T][Hq][128]: out and lse, and the bounds of their errors.

        In units of u = 2^-24, first order, for tokens i of a row with weights w_i (softmax), rows v_i, codes c, scales a, minima m:
          logits   products of codes and queries are exact; at most 8 matrix products of 16 terms a half add them up, and one cuts
                   at most 17 terms at 2^-23 of the largest: 8 x 17 x 2^-23 < 2^-15.9 of the sum of magnitudes
                   M_i = |sm| sum |q'| (a c + |m|); the fp32 steps after them a few u of it.  A rotated query has 7 fp32 stages
                   and a low half that ends 2^-22 below: 2^-20 of sum |q| / 16 in each dimension.
          weights  w_i a rounded to fp16: 2^-11 of what it brings, w_i |back(a c)| by groups (an fp16 cache: back(a (c - 7.5)));
                   below the normal range, 2^-31 of the largest weight for each token
          sums     of a warp, at most 64 steps here: 64 u of sum w |m| and of the normaliser, 2^-14 of sum w a c on tensor cores
          output   half an ulp of its type"""
        p = self.p
        B, T, Hq, _ = q.shape
        G, P = Hq // p.n_kv_heads, p.page_tokens
        q = q.double()
        out, tol = torch.zeros_like(q), torch.zeros_like(q)
        lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
        tol_lse = torch.zeros_like(lse)
        for b, n in enumerate(self.lens):
            if n <= 0:
                continue
            codes, a, m = rows_of_pages(p, self.blocks[self.table[b, : -(-n // P)].long()])
            for h in range(p.n_kv_heads):
                kc, vc = codes[:, :n, h]
                ka, va = (spread_groups(x, p) for x in a[:, :n, h])
                km, vm = (spread_groups(x, p) for x in m[:, :n, h])
                k, v = km + kc * ka, vm + vc * va
                k_mag = kc * ka + km.abs()
                k_back, v_back = self.back(k), self.back(v)
                # what a weight's rounding touches, by groups
                mid = vc - 7.5 if p.half else vc
                parts = torch.stack([self.back(torch.where(spread_groups(torch.eye(D // p.group, device=q.device), p)[g] > 0, mid * va, 0.0)).abs()
                                     for g in range(D // p.group)]).sum(0)
                for t in range(T):
                    sees = n - T + 1 + t
                    if sees <= 0:
                        continue
                    at = torch.arange(sees, device=q.device)
                    if kept is not None:
                        pages = torch.as_tensor(kept[b][t][h], dtype=torch.int64, device=q.device)
                        at = (pages[:, None] * P + torch.arange(P, device=q.device)).flatten()
                        at = at[at < sees]
                        if not len(at):
                            continue
                    for g in range(G):
                        hq = h * G + g
                        x = q[b, t, hq]
                        l = (k_back[at] @ x) * sm_scale
                        lse[b, t, hq] = torch.logsumexp(l, 0)
                        w = torch.exp(l - lse[b, t, hq])
                        y = w @ v_back[at]
                        out[b, t, hq] = y
                        xr = (x * self.s) @ self.h / 16 if p.rotate else x
                        el = 2.0**-15.5 * abs(sm_scale) * (k_mag[at] @ xr.abs())
                        if p.rotate:
                            el = el + 2.0**-20 * abs(sm_scale) * x.abs().sum() / 16 * k_mag[at].sum(-1)
                        tol_lse[b, t, hq] = (w * el).sum() + 64 * 2.0**-24 + 2.0**-22 * lse[b, t, hq].abs() + 1e-6
                        e = (w * el) @ (v_back[at] - y).abs()
                        e = e + 2.0**-11 * (w @ parts[at])
                        # rotated back, a dimension gets a 16th of every one's error
                        total = (lambda z: z.sum() / 16) if p.rotate else (lambda z: z)
                        wa = w[:, None] * va[at]
                        e = e + total(15 * len(at) * 2.0**-31 * wa.amax(0))
                        e = e + total(64 * 2.0**-24 * (w @ vm[at].abs()) + 2.0**-14 * (w @ (vc[at] * va[at])))
                        e = e + 128 * 2.0**-24 * y.abs()
                        # fp16 numbers below 2^-14 are 2^-24 apart
                        half_ulp = y.abs() * 2.0**-11 + 2.0**-25 if p.half else y.abs() * 2.0**-8
                        tol[b, t, hq] = e * 1.02 + half_ulp + 1e-30
        return out, lse, tol, tol_lse


def check(p, c, q, out, lse, sm_scale, kept=None, layer=0):
    """out and lse of a call against the 64-bit ones; returns the largest share of the bound that was needed."""
    want, want_lse, tol, tol_lse = Exact(p, c.pool[layer], c.table, c.lens.tolist()).attend(q, sm_scale, kept)
    got = out.double()
    assert bool(torch.isfinite(got).all())
    share = float(((got - want).abs() / tol.clamp_min(1e-30)).max())
    assert share <= 1, share
    empty = torch.isneginf(want_lse)
    assert bool((torch.isneginf(lse) == empty).all()) and bool((got[empty] == 0).all())
    d = (lse.double() - want_lse)[~empty].abs()
    assert bool((d <= tol_lse[~empty]).all()), float((d / tol_lse[~empty]).max())
    return share
