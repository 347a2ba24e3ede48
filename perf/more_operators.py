"""Operators of the paged 4-bit cache for many answers in little memory, as cases that can be timed and compared.

share    akv_pages_share finds rows whose tables begin with the same pages, akv_paged_attn_shared attends those pages once
         for all of them and each row's own tokens beside, in one softmax
weigh    akv_paged_weights adds the attention weights that tokens got to their scores
evict    akv_paged_evict keeps the first, the last and the heaviest tokens of a row, head by head, and moves them together

Every case is one pass of calls on one layer's cache. Sizes: 1 to 64 rows of 1 to 131072 tokens, 1 to 8 KV heads (the heads one
GPU holds), 1 to 8 query heads each, 1 to 64 query tokens, pages of 16 to 128 tokens, groups of 64 or 128 dimensions per
scale, rotated or not, bf16 or fp16 rows.

Bytes of a cache.  A page holds a block per KV head: page_tokens / 16 sub-blocks of 16 tokens.  A sub-block is
  1024 B  key codes: 64 B per token; 32-bit word 4 t + j, nibble i: dimension 32 j + 8 t + i   (t, j < 4, i < 8)
  1024 B  value codes: token 8 p + 2 t + o (p, o < 2, t < 4), dimension 64 s + 8 g + 4 u + n (s, u < 2, g < 8, n < 4):
          byte 512 p + 16 (4 g + t) + 4 (2 s + u) + 2 o + n / 2, its low half where n is even
  16 x 2 NG words  per token the key's NG groups, then the value's: fp16 scale | fp16 minimum << 16
"""
import math

import numpy as np
import torch

own = False

D = 128
ROT_SEED = 0x5EED
SM_SCALE = 1 / math.sqrt(D)


# ---- cases -------------------------------------------------------------------------------


def _text(xs):
    return ",".join(str(x) for x in xs)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _case(name, op, H, page=64, group=64, rotate=False, half=False, **more):
    return dict(name=name, op=op, H=H, page=page, group=group, rotate=rotate, half=half, **more)


def _share(name, prompts, answers, tail, H, G, T=1, **kw):
    """Answers of each prompt: rows that share its full pages and go on for up to `tail` tokens of their own."""
    return _case(name, "share", H, G=G, T=T, prompts=_text(prompts), answers=_text(answers), tail=tail, **kw)


def _weigh(name, lens, H, G, T=1, decay=1.0, **kw):
    return _case(name, "weigh", H, G=G, T=T, decay=decay, lens=_text(lens), **kw)


def _evict(name, lens, keep, sink, recent, H, **kw):
    return _case(name, "evict", H, lens=_text(lens), keep=_text(keep), sink=sink, recent=recent, **kw)


RAGGED = [131072, 8193, 50021, 23456, 100003, 12345]


def listed():
    return [
        # four answers to one chat prompt: the smallest call, launches and latency
        _share("share-chat", [1021], [4], 40, 8, 4),
        # eight prompts at 32K with eight answers each
        _share("share-beam", [32761] * 8, [8] * 8, 256, 8, 4, rotate=True),
        # drafts of four tokens for the answers of a ragged batch of prompts, one of them with a single answer; fp16, small pages
        _share("share-draft", [9000, 4173, 777, 5001], [5, 3, 9, 1], 700, 4, 4, T=4, page=16, group=128, half=True),
        # 32 samples of one long problem
        _share("share-samples", [16001], [32], 500, 8, 8),
        # the same over a document of 128K tokens, rotated: the largest attention
        _share("share-128k", [131072], [32], 256, 8, 8, rotate=True),
        # a decode step of 32 requests: each token's weight goes to its score
        _weigh("weigh-step", [1021 + 37 * b for b in range(32)], 8, 4, decay=0.99),
        # the last 64 tokens of a prompt at 32K say which of its tokens matter
        _weigh("weigh-window", [32768], 8, 4, T=64, decay=0.0, rotate=True),
        # a draft's step of a ragged batch, fp16, one scale per row, small pages
        _weigh("weigh-ragged", RAGGED, 8, 8, T=2, page=16, group=128, half=True),
        # eight requests at 128K: the most bytes
        _weigh("weigh-70b-128k", [131072] * 8, 8, 8, rotate=True),
        # 32 chats go back to 1024 tokens each
        _evict("evict-chat", [1088 + b for b in range(32)], [1024] * 32, 4, 64, 8, page=16),
        # a prompt at 32K keeps an eighth of its tokens, a shorter one all of them
        _evict("evict-prompt", [32768, 2001], [4096, 4096], 4, 64, 8),
        # four requests at 128K keep half: the most bytes
        _evict("evict-70b-128k", [131072] * 4, [65536] * 4, 16, 256, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["share", "share", "share", "weigh", "weigh", "evict"])
    H, G = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 8, 8])
    kw = dict(page=rng.choice([16, 32, 64, 64, 128]), group=rng.choice([64, 64, 128]), rotate=rng.random() < 0.5, half=rng.random() < 0.3)
    if op == "share":
        T = rng.choice([1, 1, 1, 2, 4])
        groups = _log_int(rng, 1, 8)
        answers = [rng.randint(1, 2 * _log_int(rng, 1, 32 // groups)) for _ in range(groups)]
        # 32 rows of 8 heads with 8 query heads each over 131072 tokens are the most work
        room = 32 * 8 * 8 * 131072 // (H * max(4, G * T) * sum(answers))
        room = min(room, (1 << 22) // (H * groups))
        S = _log_int(rng, 16, max(64, min(131072, room)))
        prompts = [S] * groups if rng.random() < 0.3 else [rng.randint(max(1, S // 4), S) for _ in range(groups)]
        c = _share("", prompts, answers, _log_int(rng, 1, 600), H, G, T=T, **kw)
    elif op == "weigh":
        T = rng.choice([1, 1, 1, 2, 4, 32, 64])
        B = _log_int(rng, 1, 32)
        S = _log_int(rng, 16, max(64, min(131072, (1 << 23) // (H * B * max(1, T * G // 8)))))
        lens = [S] * B if rng.random() < 0.3 else [rng.randint(max(1, S // 4), S) for _ in range(B)]
        c = _weigh("", lens, H, G, T=T, decay=rng.choice([0.0, 0.9, 1.0]), **kw)
    else:
        B = _log_int(rng, 1, 32)
        S = _log_int(rng, 16, max(64, min(131072, (5 << 19) // (H * B))))
        lens = [S] * B if rng.random() < 0.3 else [rng.randint(max(1, S // 4), S) for _ in range(B)]
        share = rng.choice([0.05, 0.25, 0.5, 0.9])
        keep = [max(1, int(n * share)) if rng.random() < 0.9 else n + rng.randint(0, 40) for n in lens]
        c = _evict("", lens, keep, rng.randint(0, 8), rng.randint(0, 80), H, **kw)
    del c["name"]
    return c


# ---- the cache's bytes -------------------------------------------------------------------


def _ng(case):
    return D // case["group"]


def _sub_bytes(case):
    return 2048 + 128 * _ng(case)


def _block_bytes(case):
    return case["page"] // 16 * _sub_bytes(case)


def _dtype(case):
    return torch.float16 if case["half"] else torch.bfloat16


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + what * 7919) & 0x7FFFFFFFFFFFFFFF)


def _mix(x):
    z = (x + 0x9E3779B97F4A7C15) & (2**64 - 1)
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & (2**64 - 1)
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & (2**64 - 1)
    return z ^ (z >> 31)


def _signs():
    """+1 or -1 per dimension: the rotation's sign pattern of ROT_SEED."""
    words = [_mix(ROT_SEED), _mix(ROT_SEED + 1)]
    return torch.tensor([-1.0 if words[j // 64] >> (j % 64) & 1 else 1.0 for j in range(D)], device="cuda")


def _stage(x, h):
    y = x.unflatten(-1, (-1, 2, h))
    a, b = y[..., 0, :], y[..., 1, :]
    return torch.stack((a + b, a - b), -2).flatten(-3)


def _wht(x):
    """Sylvester Hadamard product of the last axis (128), in radix-2 stages."""
    return _stage(_stage(_stage(_stage(_stage(_stage(_stage(x, 1), 2), 4), 8), 16), 32), 64)


def _quantise(case, x):
    """fp32 rows [..., 128] -> codes (uint8 [..., 128]), scales and minima (fp16 [..., NG])."""
    v = _wht(x * _signs()) * 0.125 if case["rotate"] else x
    v = v.unflatten(-1, (_ng(case), case["group"]))
    lo = v.amin(-1, keepdim=True).clamp(-65504, 65504).half()
    step = ((v.amax(-1, keepdim=True) - lo.float()).clamp_min(0) / 15).clamp_max(65504).half()
    c = torch.where(step > 0, ((v - lo.float()) / step.float()).round().clamp(0, 15), 0.0)
    return c.flatten(-2).to(torch.uint8), step[..., 0], lo[..., 0]


def _words(step, lo):
    w = step.view(torch.int16).int() & 0xFFFF | lo.view(torch.int16).int() << 16
    return w.contiguous().view(torch.uint8)  # [..., 4 NG]


def _pack(case, K, V):
    """Dense rows [N pages * page, H, 128] (fp32) -> bytes of the pages' blocks [N, H, block bytes]."""
    P, H = case["page"], case["H"]
    n = K.shape[0] // 16
    sub = torch.empty((n, H, _sub_bytes(case)), dtype=torch.uint8, device="cuda")
    ck, ak, mk = _quantise(case, K)
    ck = ck.unflatten(-1, (4, 4, 4, 2)).transpose(-4, -3)  # dimension 32 j + 8 t + i to word 4 t + j, nibble i
    sub[:, :, :1024] = (ck[..., 0] | ck[..., 1] << 4).flatten(-3).view(n, 16, H, 64).transpose(1, 2).reshape(n, H, 1024)
    cv, av, mv = _quantise(case, V)
    # value codes: (p, t, o | H | s, g, u, n) -> (H | p, g, t, s, u, o, n)
    cv = cv.view(n, 2, 4, 2, H, 2, 8, 2, 2, 2).permute(0, 4, 1, 6, 2, 5, 7, 3, 8, 9)
    sub[:, :, 1024:2048] = (cv[..., 0] | cv[..., 1] << 4).reshape(n, H, 1024)
    meta = torch.cat((_words(ak, mk), _words(av, mv)), -1)  # [tokens, H, 8 NG]
    sub[:, :, 2048:] = meta.view(n, 16, H, -1).transpose(1, 2).reshape(n, H, -1)
    return sub.view(n * 16 // P, P // 16, H, -1).transpose(1, 2).flatten(2)


def _unpack(case, blocks):
    """Bytes [..., block bytes] of page blocks -> fp32 rows as stored (still rotated) [..., page, 128], twice."""
    sub = blocks.unflatten(-1, (-1, _sub_bytes(case)))
    lead = sub.shape[:-1]
    k = sub[..., :1024].reshape(*lead, 16, 4, 4, 4)  # token, t, j, byte
    k = torch.stack((k & 15, k >> 4), -1).transpose(-4, -3).reshape(*lead, 16, _ng(case), case["group"])
    v = sub[..., 1024:2048].reshape(*lead, 2, 8, 4, 2, 2, 2, 2)  # p, g, t, s, u, o, n / 2
    v = torch.stack((v & 15, v >> 4), -1)
    e = len(lead)
    v = v.permute(*range(e), e, e + 2, e + 5, e + 3, e + 1, e + 4, e + 6, e + 7).reshape(*lead, 16, _ng(case), case["group"])
    meta = sub[..., 2048:].contiguous().view(torch.float16).view(*lead, 16, 2, _ng(case), 2).float()
    k = k.float() * meta[..., 0, :, :1] + meta[..., 0, :, 1:]
    v = v.float() * meta[..., 1, :, :1] + meta[..., 1, :, 1:]
    return k.flatten(-4, -3).flatten(-2), v.flatten(-4, -3).flatten(-2)


# ---- inputs ------------------------------------------------------------------------------


def _rows(gen, n, H, dtype):
    """Keys and values [n, H, 128]: 64 clusters, four outlier channels among a head's keys."""
    ck, cv = torch.randn((2, 64, H, D), generator=gen, device="cuda")
    cid = torch.randint(0, 64, (n,), generator=gen, device="cuda")
    nk, nv = 1.0 + 0.2 * torch.randn((2, n, 1, 1), generator=gen, device="cuda")
    k = nk * (ck[cid] + 0.5 * torch.randn((n, H, D), generator=gen, device="cuda"))
    v = nv * (cv[cid] + 0.5 * torch.randn((n, H, D), generator=gen, device="cuda"))
    k[..., torch.randperm(D, generator=gen, device="cuda")[:4]] *= 4
    return k.to(dtype), v.to(dtype)


def _int32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _pages_of(case, n):
    return -(-n // case["page"])


def _tails(case):
    """Own tokens of each answer, in row order."""
    rows = sum(_ints(case["answers"]))
    return [1 + (37 * k) % case["tail"] for k in range(rows)]


def _share_rows(case):
    """(prompt, tokens held) of each row."""
    rows = [g for g, n in enumerate(_ints(case["answers"])) for _ in range(n)]
    prompts = _ints(case["prompts"])
    return [(g, prompts[g] + t) for g, t in zip(rows, _tails(case))]


def _fill(case, s, gen, pages):
    """Clustered keys and values in the given pages, 4096 tokens and more at a time."""
    step = max(1, 65536 // case["page"])
    for at in range(0, len(pages), step):
        part = pages[at : at + step]
        k, v = _rows(gen, len(part) * case["page"], case["H"], _dtype(case))
        s["pool"][0, part] = _pack(case, k.float(), v.float())


def _prepare_share(case, s, gen):
    P, H = case["page"], case["H"]
    rows, prompts = _share_rows(case), _ints(case["prompts"])
    full = [n // P for n in prompts]  # pages that a prompt's answers share
    total = sum(full) + sum(_pages_of(case, n) - full[g] for g, n in rows)
    ids = torch.randperm(total + 5, generator=gen, device="cuda")[:total]
    s["pool"] = torch.zeros((1, total + 5, H, _block_bytes(case)), dtype=torch.uint8, device="cuda")
    s["table"] = torch.full((len(rows), max(_pages_of(case, n) for _, n in rows) + 1), -1, dtype=torch.int32, device="cuda")
    _fill(case, s, gen, ids)
    at, first = 0, []
    for n in full:
        first.append(at)
        at += n
    for b, (g, n) in enumerate(rows):
        s["table"][b, : full[g]] = ids[first[g] : first[g] + full[g]]
        mine = _pages_of(case, n) - full[g]
        s["table"][b, full[g] : full[g] + mine] = ids[at : at + mine]
        at += mine
    s["lens"] = _int32([n for _, n in rows])
    B, T, Hq = len(rows), case["T"], H * case["G"]
    s["q"] = (torch.randn((B, T, Hq, D), generator=gen, device="cuda") * 1.5).to(_dtype(case))
    s["share"] = torch.empty((4, B), dtype=torch.int32, device="cuda")
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((B, T, Hq), device="cuda")


def _spread(case, s, gen, need, spare=5):
    """A table of pages spread over the pool for rows of `need` pages each, and the pool."""
    total = sum(need)
    ids = torch.randperm(total + spare, generator=gen, device="cuda")[:total]
    s["table"] = torch.full((len(need), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        s["table"][b, :n] = ids[at : at + n]
        at += n
    return ids, total + spare


def _prepare_weigh(case, s, gen):
    P, H, lens = case["page"], case["H"], _ints(case["lens"])
    ids, n_pages = _spread(case, s, gen, [_pages_of(case, n) for n in lens])
    s["pool"] = torch.zeros((1, n_pages, H, _block_bytes(case)), dtype=torch.uint8, device="cuda")
    _fill(case, s, gen, ids)
    s["lens"] = _int32(lens)
    B, T, Hq = len(lens), case["T"], H * case["G"]
    s["q"] = (torch.randn((B, T, Hq, D), generator=gen, device="cuda") * 1.5).to(_dtype(case))
    # the attention that came before gave the queries' lse
    s["lse"] = torch.empty((B, T, Hq), device="cuda")
    for b in range(B):
        for h in range(H):
            x = _logits(case, s, b, h)
            s["lse"][b, :, h * case["G"] : (h + 1) * case["G"]] = torch.logsumexp(x, -1).view(T, -1)
    cap = (s["table"].shape[1]) * P
    s["old"] = torch.rand((B, H, cap), generator=gen, device="cuda") ** 4
    s["new"] = torch.zeros((B, H, cap), device="cuda")


def _prepare_evict(case, s, gen):
    P, H, lens = case["page"], case["H"], _ints(case["lens"])
    held = [min(n, k) for n, k in zip(lens, _ints(case["keep"]))]
    # rows with the tokens, then a row for what each of them keeps
    _, n_pages = _spread(case, s, gen, [_pages_of(case, n) for n in lens] + [_pages_of(case, n) for n in held])
    s["pool"] = torch.randint(-(2**62), 2**62, (1, n_pages, H * _block_bytes(case) // 8), generator=gen, device="cuda")
    B = len(lens)
    s["lens"] = _int32(lens + [0] * B)
    s["src"], s["dst"] = torch.arange(B, dtype=torch.int32, device="cuda"), torch.arange(B, 2 * B, dtype=torch.int32, device="cuda")
    s["keep"] = _int32(_ints(case["keep"]))
    # weights that have been added up: a long tail, some tokens with none, some alike
    cap = s["table"].shape[1] * P
    s["scores"] = torch.zeros((2 * B, H, cap), device="cuda")
    w = torch.exp(2.0 * torch.randn((B, H, cap), generator=gen, device="cuda"))
    w = torch.where(torch.rand((B, H, cap), generator=gen, device="cuda") < 0.1, 0.0, w)
    s["scores"][:B] = torch.where(torch.rand((B, H, cap), generator=gen, device="cuda") < 0.2, (w * 8).round() / 8, w)
    s["kept"] = torch.empty((B, H, max(_ints(case["keep"]))), dtype=torch.int32, device="cuda")
    s["count"] = torch.empty(B, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    s = dict(case=case)
    {"share": _prepare_share, "weigh": _prepare_weigh, "evict": _prepare_evict}[case["op"]](case, s, _gen(seed, 1))
    return s


# ---- the framework's calls ---------------------------------------------------------------


def _handle(s):
    """The parameters, pages and workspaces that a program makes once and keeps."""
    import paper_2608_02901_gb300 as akv

    case = s["case"]
    p = akv.PagedParams(n_kv_heads=case["H"], n_q_heads=case["H"] * case.get("G", 1), page_tokens=case["page"], group=case["group"],
                        half=bool(case["half"]), rotate=bool(case["rotate"]), rot_seed=ROT_SEED)
    h = dict(akv=akv, p=p, pages=akv.Pages(p, s["pool"], s["table"], s["lens"]))
    if case["op"] == "share":
        h["share"] = akv.PageShare(s["share"])
        ws = max(akv.akv_pages_workspace_size(h["pages"]), akv.akv_paged_attn_shared_workspace_size(p, h["pages"], case["T"]))
        h["ws"] = torch.empty(ws, dtype=torch.uint8, device="cuda")
    if case["op"] == "evict":
        h["kept"] = akv.KeptTokens(s["kept"], s["count"])
    return h


def _run_own(s):
    if "handle" not in s:
        s["handle"] = _handle(s)
    h, case = s["handle"], s["case"]
    akv, p, pages = h["akv"], h["p"], h["pages"]
    if case["op"] == "share":
        akv.akv_pages_share(p, pages, h["share"], ws=h["ws"])
        akv.akv_paged_attn_shared(p, pages, s["q"], s["out"], h["share"], lse=s["lse"], sm_scale=SM_SCALE, ws=h["ws"])
        return {"share": s["share"], "out": s["out"], "lse": s["lse"]}
    if case["op"] == "weigh":
        old = s["old"] if case["decay"] else None
        akv.akv_paged_weights(p, pages, s["q"], s["lse"], s["new"], was=old, decay=case["decay"], sm_scale=SM_SCALE)
        return {"new": s["new"]}
    akv.akv_paged_evict(p, pages, s["src"], s["dst"], s["scores"], h["kept"], keep=s["keep"], sink=case["sink"], recent=case["recent"])
    return {"kept": s["kept"], "count": s["count"], "scores": s["scores"], "pool": s["pool"]}


# ---- the plain forms ---------------------------------------------------------------------


def _stored_rows(case, s, b, n=None):
    """Keys and values as stored [H, tokens, 128] of row b's first n tokens (all it holds), whole pages."""
    n = int(s["lens"][b]) if n is None else n
    page = s["table"][b, : _pages_of(case, n)].long()
    K, V = _unpack(case, s["pool"][0][page].transpose(0, 1))  # [H, pages, page, 128]
    return K.flatten(1, 2), V.flatten(1, 2)


def _sees(case, s, b):
    """Tokens that each of row b's query tokens sees [T]."""
    return s["lens"][b] - case["T"] + 1 + torch.arange(case["T"], device="cuda")


def _logits(case, s, b, h):
    """Row b's logits with KV head h [T G, tokens of whole pages], -infinity where a token is not seen (as stored, in fp32)."""
    n = _ints(case["lens"])[b]
    page = s["table"][b, : _pages_of(case, n)].long()
    K, _ = _unpack(case, s["pool"][0][page, h])
    K = K.flatten(0, 1)
    T, G = case["T"], case["G"]
    q = s["q"][b, :, h * G : (h + 1) * G].float().reshape(T * G, D)
    if case["rotate"]:
        q = _wht(q * _signs()) * 0.0625
    there = torch.arange(K.shape[0], device="cuda") < _sees(case, s, b)[:, None]
    return (q @ K.T * SM_SCALE).masked_fill(~there.repeat_interleave(G, 0), -math.inf)


def _run_share(s):
    case = s["case"]
    B, T, H, G = len(s["lens"]), case["T"], case["H"], case["G"]
    # which rows begin with the same page, and how many pages they have alike
    held = (s["lens"] + case["page"] - 1) // case["page"]
    col = torch.arange(s["table"].shape[1], device="cuda")
    table = torch.where(col < held[:, None], s["table"], -1)
    same0 = (table[:, None, 0] == table[None, :, 0]) & (table[:, 0] >= 0)
    row = torch.arange(B, device="cuda")
    leader = torch.where(same0, row[None, :], B).amin(1)
    leader = torch.where(leader < B, leader, row)
    alike = ((table == table[leader]) & (table >= 0)).int().cumprod(1).sum(1)
    same = leader[:, None] == leader[None, :]
    size = same.sum(1)
    alike = torch.where(same, alike[None, :], 1 << 30).amin(1)
    alike = torch.where(size > 1, alike, 0)
    order = (leader * B + row).argsort()
    s["share"].copy_(torch.stack((leader, alike, size, order)))
    # attention, a row at a time
    for b, (_, n) in enumerate(_share_rows(case)):
        K, V = _stored_rows(case, s, b, n)
        q = s["q"][b].float().view(T, H, G, D).transpose(0, 1).reshape(H, T * G, D)
        if case["rotate"]:
            q = _wht(q * _signs()) * 0.0625
        there = (torch.arange(K.shape[1], device="cuda") < _sees(case, s, b)[:, None]).repeat_interleave(G, 0)
        x = (q @ K.transpose(-1, -2) * SM_SCALE).masked_fill(~there, -math.inf)
        top = x.amax(-1, keepdim=True).clamp_min(-3e38)
        e = (x - top).exp()
        l = e.sum(-1, keepdim=True)
        out = e @ V / l.clamp_min(1e-30)
        if case["rotate"]:
            out = _wht(out) * 0.0625 * _signs()
        s["out"][b].view(T, H, G, D).copy_(out.view(H, T, G, D).transpose(0, 1))
        s["lse"][b].view(T, H, G).copy_((l.log() + top).masked_fill(l == 0, -math.inf).view(H, T, G).transpose(0, 1))
    return {"share": s["share"], "out": s["out"], "lse": s["lse"]}


def _run_weigh(s):
    case = s["case"]
    T, G = case["T"], case["G"]
    for b, n in enumerate(_ints(case["lens"])):
        for h in range(case["H"]):
            lse = s["lse"][b, :, h * G : (h + 1) * G].reshape(T * G, 1)
            w = torch.where(torch.isfinite(lse), (_logits(case, s, b, h) - lse).exp(), 0.0).sum(0)[:n]
            s["new"][b, h, :n] = case["decay"] * s["old"][b, h, :n] + w if case["decay"] else w
    return {"new": s["new"]}


def _token_bytes(case, i):
    """Places of the bytes of tokens i (of a block) in it [..., 128 + 8 NG]."""
    dev = i.device
    k = i % 16
    sub = (i // 16 * _sub_bytes(case))[..., None]
    keys = 64 * k[..., None] + torch.arange(64, device=dev)
    x = torch.arange(64, device=dev)  # s, g, u, n / 2
    values = 1024 + (512 * (k // 8) + 16 * (k % 8 // 2) + 2 * (k % 2))[..., None] + 64 * (x // 4 % 8) + 8 * (x // 32) + 4 * (x // 2 % 2) + x % 2
    meta = 2048 + 8 * _ng(case) * k[..., None] + torch.arange(8 * _ng(case), device=dev)
    return sub + torch.cat((keys, values, meta), -1)


def _run_evict(s):
    case = s["case"]
    P, H, top = case["page"], case["H"], s["kept"].shape[2]
    flat = s["pool"].view(torch.uint8).view(-1)
    s["kept"].fill_(-1)
    for i, (n, keep) in enumerate(zip(_ints(case["lens"]), _ints(case["keep"]))):
        m = min(n, keep)
        s["count"][i] = m
        at = torch.arange(n, device="cuda")
        x = s["scores"][i, :, :n].masked_fill((at < case["sink"]) | (at >= n - case["recent"]), math.inf)
        kept = x.sort(dim=-1, descending=True, stable=True).indices[:, :m].sort(-1).values  # [H, m]
        s["kept"][i, :, :m] = kept
        s["scores"][len(s["kept"]) + i, :, :m] = s["scores"][i].gather(1, kept)
        head = torch.arange(H, device="cuda")[:, None] * _block_bytes(case)
        to = torch.arange(m, device="cuda").expand(H, m)
        src = s["table"][i].long()[kept // P] * (H * _block_bytes(case)) + head
        dst = s["table"][len(s["kept"]) + i].long()[to // P] * (H * _block_bytes(case)) + head
        for a in range(0, m, 16384):  # (places are 64-bit numbers, 144 a token)
            part = slice(a, a + 16384)
            flat[dst[:, part, None] + _token_bytes(case, to[:, part] % P)] = flat[src[:, part, None] + _token_bytes(case, kept[:, part] % P)]
    return {"kept": s["kept"], "count": s["count"], "scores": s["scores"], "pool": s["pool"]}


def run(s):
    if own:
        return _run_own(s)
    return {"share": _run_share, "weigh": _run_weigh, "evict": _run_evict}[s["case"]["op"]](s)


# ---- what cannot be done without ---------------------------------------------------------


def work(case):
    P, H = case["page"], case["H"]
    side = (64 + 4 * _ng(case)) * H  # bytes of a token's keys, or values, of all heads
    if case["op"] == "evict":
        lens = _ints(case["lens"])
        kept = sum(min(n, k) for n, k in zip(lens, _ints(case["keep"])))
        # scores; the kept tokens in and out, with their scores and their places
        return {"bytes": 4 * H * sum(lens) + kept * (4 * side + 8 * H), "flops": 0}
    T, G = case["T"], case["G"]
    if case["op"] == "share":
        rows, prompts = _share_rows(case), _ints(case["prompts"])
        many = [n > 1 for n in _ints(case["answers"])]
        once = [n // P * P if m else 0 for n, m in zip(prompts, many)]
        tokens = sum(once) + sum(n - once[g] for g, n in rows)
        seen = sum(max(0, n - T + 1 + t) for _, n in rows for t in range(T))
        return {"bytes": 2 * side * tokens + len(rows) * (T * H * G * (4 * D + 4) + 16) + 4 * tokens // P, "flops": 4 * D * H * G * seen}
    lens = _ints(case["lens"])
    seen = sum(max(0, n - T + 1 + t) for n in lens for t in range(T))
    io = len(lens) * T * H * G * (2 * D + 4)
    return {"bytes": io + sum(lens) * (side + (8 if case["decay"] else 4) * H), "flops": 2 * D * H * G * seen}


# ---- the definitions in 64 bits ----------------------------------------------------------


def _back():
    """Matrix R: stored rows v (rotated) are x = v R."""
    h = np.ones((1, 1))
    while h.shape[0] < D:
        h = np.block([[h, h], [h, -h]])
    return torch.from_numpy(h).cuda() * _signs().double() / 16


def _read_rows(case, blocks, sides=(0, 1)):
    """One head's page blocks [N, bytes] -> keys, values [N * page, 128] in 64 bits, rotated back."""
    x = blocks.reshape(-1, _sub_bytes(case))
    d = torch.arange(D, device="cuda")
    i = torch.arange(16, device="cuda")[:, None]
    place = (64 * i + 4 * (4 * (d % 32 // 8) + d // 32) + d % 8 // 2,
             1024 + 512 * (i // 8) + 16 * (4 * (d % 64 // 8) + i % 8 // 2) + 4 * (2 * (d // 64) + d % 8 // 4) + 2 * (i % 2) + d % 4 // 2)
    meta = x[:, 2048:].contiguous().view(torch.float16).double().view(-1, 16, 2, _ng(case), 2)
    out = []
    for side in sides:
        c = x[:, place[side]] >> (4 * (d % 2)).to(torch.uint8) & 15
        w = meta[:, :, side].repeat_interleave(case["group"], -2)
        y = (c.double() * w[..., 0] + w[..., 1]).view(-1, D)
        out.append(y @ _back() if case["rotate"] else y)
    return out


def _exact_share(case, s):
    B, T, H, G = len(s["lens"]), case["T"], case["H"], case["G"]
    out = torch.zeros((B, T, H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H * G), -math.inf, dtype=torch.float64, device="cuda")
    rows = _share_rows(case)
    for h in range(H):
        was, K, V = None, None, None
        for b, (g, n) in enumerate(rows):
            full = _ints(case["prompts"])[g] // case["page"]
            page = s["table"][b, : _pages_of(case, n)].long()
            if was != g:
                was, shared = g, _read_rows(case, s["pool"][0, page[:full], h])
            K, V = (torch.cat(x) for x in zip(shared, _read_rows(case, s["pool"][0, page[full:], h])))
            for t in range(T):
                sees = n - T + 1 + t
                if sees <= 0:
                    continue
                at = slice(h * G, h * G + G)
                x = s["q"][b, t, at].double() @ K[:sees].T / math.sqrt(D)
                lse[b, t, at] = torch.logsumexp(x, -1)
                out[b, t, at] = torch.exp(x - lse[b, t, at][:, None]) @ V[:sees]
    return {"share": None, "out": out, "lse": lse}


def _exact_weigh(case, s):
    T, G = case["T"], case["G"]
    new = torch.zeros_like(s["new"], dtype=torch.float64)
    for b, n in enumerate(_ints(case["lens"])):
        page = s["table"][b, : _pages_of(case, n)].long()
        for h in range(case["H"]):
            (K,) = _read_rows(case, s["pool"][0, page, h], (0,))
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            for t in range(T):
                sees = max(0, n - T + 1 + t)
                x = s["q"][b, t, h * G : h * G + G].double() @ K[:sees].T / math.sqrt(D)
                lse = s["lse"][b, t, h * G : h * G + G].double()[:, None]
                total[:sees] += torch.where(torch.isfinite(lse), torch.exp(x - lse), torch.zeros_like(x)).sum(0)
            new[b, h, :n] = total + case["decay"] * s["old"][b, h, :n].double()
    return {"new": new}


def _exact_evict(case, s):
    scores = s["scores"].double()
    B = len(s["src"])
    for i, (n, keep) in enumerate(zip(_ints(case["lens"]), _ints(case["keep"]))):
        for h in range(case["H"]):
            x = s["scores"][i, h, :n].cpu().numpy().astype(np.float64)
            at = np.arange(n)
            x[(at < case["sink"]) | (at >= n - case["recent"])] = np.inf
            kept = np.sort(np.lexsort((at, -x))[:keep])
            scores[B + i, h, : len(kept)] = scores[i, h, torch.from_numpy(kept).cuda()]
    return {"kept": None, "count": None, "scores": scores, "pool": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"share": _exact_share, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, s)
