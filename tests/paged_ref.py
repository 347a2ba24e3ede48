"""Plain 64-bit forms of the paged 4-bit cache's operators, for the tests: numpy, one thing at a time."""
import math

import numpy as np

D = 128


def signs(rot_seed):
    m = 2**64 - 1

    def mix(x):
        z = (x + 0x9E3779B97F4A7C15) & m
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
        return z ^ (z >> 31)

    return np.array([-1.0 if mix(rot_seed + j // 64) >> (j % 64) & 1 else 1.0 for j in range(D)])


def hadamard():
    h = np.ones((1, 1))
    while len(h) < D:
        h = np.block([[h, h], [h, -h]])
    return h


def rotated(x, p):
    """What is quantised of rows x."""
    return (x * signs(p.rot_seed)) @ hadamard() / 8 if p.rotate else x


def rotated_back(v, p):
    return (v @ hadamard()) / 16 * signs(p.rot_seed) if p.rotate else v


def block_bytes(p):
    return p.page_tokens // 16 * (2048 + 128 * (D // p.group)) + (512 if p.bounds else 0)


def rows_of_block(block, p):
    """A head's block of one page: codes [2][P][128], scales and minima [2][P][NG] (key side, value side)."""
    ng, P = D // p.group, p.page_tokens
    sub = 2048 + 128 * ng
    codes = np.zeros((2, P, D), int)
    a, m = np.zeros((2, 2, P, ng))
    for i in range(P):
        s = block[i // 16 * sub : (i // 16 + 1) * sub]
        k = i % 16
        for d in range(D):
            j, t, n = d // 32, d // 8 % 4, d % 8
            codes[0, i, d] = s[64 * k + 4 * (4 * t + j) + n // 2] >> 4 * (n % 2) & 15
            sd, g, u, n = d // 64, d // 8 % 8, d // 4 % 2, d % 4
            at = 1024 + 512 * (k // 8) + 16 * (4 * g + k % 8 // 2) + 4 * (2 * sd + u) + 2 * (k % 2) + n // 2
            codes[1, i, d] = s[at] >> 4 * (n % 2) & 15
        w = s[2048 + 8 * ng * k : 2048 + 8 * ng * (k + 1)].copy().view(np.float16).astype(float).reshape(2, ng, 2)
        a[:, i], m[:, i] = w[..., 0], w[..., 1]
    return codes, a, m


def values(codes, a, m):
    """v^ [..., 128] of codes and per-group scales and minima."""
    group = D // a.shape[-1]
    return np.repeat(m, group, -1) + codes * np.repeat(a, group, -1)


class Ref:
    """The logical rows of a cache as its bytes say: v^ per request, side, token, head."""

    def __init__(self, p, pool_layer, table, lens):
        self.p, self.lens = p, [int(n) for n in lens]
        H, bb, P = p.n_kv_heads, block_bytes(p), p.page_tokens
        pool = pool_layer.reshape(-1, H, bb)
        done = {}
        self.v = []  # [2][len][H][128]
        self.bounds = []
        for b, n in enumerate(self.lens):
            parts = []
            for j in range(-(-n // P)):
                page = int(table[b, j])
                if page not in done:
                    done[page] = np.stack([values(*rows_of_block(pool[page, h], p)) for h in range(H)], 2)
                parts.append(done[page])
            self.v.append(np.concatenate(parts, 1)[:, :n] if parts else np.zeros((2, 0, H, D)))

    def attend(self, q, sm_scale, kept=None):
        """q [B][T][Hq][128] fp64: out, lse, and what tolerances need: the largest sum |q x| and the range of v^."""
        p = self.p
        B, T, Hq, _ = q.shape
        out, lse = np.zeros_like(q), np.full((B, T, Hq), -math.inf)
        mass, spread = np.zeros((B, T, Hq)), np.zeros((B, T, Hq))
        for b in range(B):
            for t in range(T):
                sees = max(0, self.lens[b] - T + 1 + t)
                for hq in range(Hq):
                    h = hq // (Hq // p.n_kv_heads)
                    k, v = self.v[b][0, :sees, h], self.v[b][1, :sees, h]
                    if kept is not None:
                        at = [i for j in kept[b][t][h] for i in range(j * p.page_tokens, min(sees, (j + 1) * p.page_tokens))]
                        k, v = k[at], v[at]
                    if not len(k):
                        continue
                    k = rotated_back(k, p)
                    x = k @ q[b, t, hq] * sm_scale
                    top = x.max()
                    e = np.exp(x - top)
                    out[b, t, hq] = rotated_back((e @ v / e.sum())[None], p)[0]
                    lse[b, t, hq] = top + np.log(e.sum())
                    mass[b, t, hq] = (np.abs(k) @ np.abs(q[b, t, hq])).max() * abs(sm_scale)
                    spread[b, t, hq] = np.ptp(v, -1).max() + 1e-30
        return out, lse, mass, spread


def select(p, q, bounds, sees, top, sink, recent):
    """Pages that one query group's rows q [G][128] keep, bounds [n][2][128] (fp64, exact values)."""
    n = -(-max(0, sees) // p.page_tokens)
    if n <= top:
        return list(range(n))

    def whole(x, e):
        return np.clip(np.rint(x * 2.0 ** (7 - e)), -127, 127)

    def exponent(a):
        return int(np.clip(math.frexp(a)[1], -100, 100))

    qw = whole(q, exponent(np.abs(q).max()))
    score = []
    for j in range(n):
        big = np.abs(bounds[j]).max()
        if not math.isfinite(big):
            score.append(math.inf)
            continue
        bw = whole(bounds[j], exponent(big))
        score.append(np.maximum(qw * bw[0], qw * bw[1]).sum(-1).max() * 2.0 ** exponent(big))
    middle = sorted(range(sink, n - recent), key=lambda j: (-score[j], j))
    return sorted([j for j in range(n) if j < sink or j >= n - recent] + middle[: top - sink - recent])
