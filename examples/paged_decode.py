"""A serving loop on the paged 4-bit cache: one layer, several requests, some of them with more than one answer.

    python examples/paged_decode.py [--heads 8] [--group 4] [--steps 32] [--top 16] [--budget 512]

What a model would give (queries, keys and values of each token) is random here.  The loop
  1. reserves pages for the prompts and appends them in chunks,
  2. forks every prompt into a few answers, which share its pages until they write,
  3. generates: reserve (copy on write), append, then attention over all pages, those that answers share read once, or over the
     few that akv_paged_select keeps for each query; the last step checks a draft of several tokens in one pass,
  4. frees the answers that are done and compacts the pool,
  5. hands the longest request over to the anchor-residual cache: akv_paged_read gives its rows, akv_encode compresses
     them, akv_decode_attn attends.
Step 3's integer state stays on the device: no step waits for the GPU.

A second loop (within_budget) keeps a bounded number of tokens a row: the weights that a prompt's last queries gave its tokens choose
those that stay, the answers share them, and their own weights choose again when they have grown.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2608_02901_gb300 as akv  # noqa: E402

D = 128


def clustered(gen, centres, shape, outliers):
    """Rows around a few centres, as attention keys and values are; four channels of the keys are larger."""
    cid = torch.randint(0, centres.shape[0], shape[:2], generator=gen, device="cuda")
    x = centres[cid] + 0.5 * torch.randn((*shape, D), generator=gen, device="cuda")
    if outliers:
        x[..., :4] *= 4
    return x.to(torch.bfloat16)


def main(heads=8, group=4, steps=32, top=16, prompts=(3000, 1777, 940), answers=3, page=64, seed=0, verbose=True, pool_pages=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    say = print if verbose else (lambda *a: None)
    B = len(prompts)
    rows = B * (1 + answers)  # the prompts, then their answers
    most = max(prompts) + steps + 16
    max_pages = -(-most // page)
    n_pages = pool_pages or sum(-(-n // page) for n in prompts) + rows * (2 + (steps + 16) // page)
    p = akv.PagedParams(n_kv_heads=heads, n_q_heads=heads * group, page_tokens=page, rotate=True, bounds=True)
    page_bytes = akv.akv_paged_page_bytes(p)
    int32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, n_pages, page_bytes), dtype=torch.uint8, device="cuda")
    table = torch.full((rows, max_pages), -1, **int32)
    lens, refs = torch.zeros(rows, **int32), torch.zeros(n_pages, **int32)
    missing, lacked = torch.zeros(1, **int32), torch.zeros(1, **int32)
    pages = akv.Pages(p, pool, table, lens, refs)
    sel = akv.PageSelection(torch.empty((rows, 1, heads, top), **int32), torch.empty((rows, 1, heads), **int32))
    draft = 4
    sharing = akv.PageShare(torch.empty((4, rows), **int32))
    ws = torch.empty(max(akv.akv_pages_workspace_size(pages), akv.akv_paged_attn_shared_workspace_size(p, pages, 1),
                         akv.akv_paged_attn_workspace_size(p, pages, 1, top), akv.akv_paged_attn_workspace_size(p, pages, draft),
                         akv.akv_paged_select_workspace_size(p, pages, 1)), dtype=torch.uint8, device="cuda")
    ck, cv = torch.randn((2, 32, heads, D), generator=gen, device="cuda")
    ids = torch.arange(rows, **int32)

    def tokens(T):
        return clustered(gen, ck, (rows, T, heads), True), clustered(gen, cv, (rows, T, heads), False)

    def put(n_new, T):
        """Room for the new tokens, then their keys and values; every layer of a model would append before lens moves.  Where the
        pool has no room the step does nothing (a scheduler would look at `lacked` now and then, and free something)."""
        akv.akv_pages_reserve(p, pages, n_new, missing, ws=ws)
        torch.maximum(lacked, missing, out=lacked)
        n_new = n_new * (missing == 0)
        K, V = tokens(T)
        akv.akv_paged_append(p, pages, K, V, n_new=n_new)
        lens.add_(n_new)
        return K, V

    # 1. the prompts, in chunks
    chunk = 1024
    want = torch.tensor(list(prompts) + [0] * (rows - B), **int32)
    for _ in range(0, max(prompts), chunk):
        put((want - lens).clamp(0, chunk), chunk)
    held = int((refs > 0).sum())
    dense = sum(prompts) * heads * 2 * 2 * D
    say(f"prompts: {sum(prompts)} tokens, {held} pages, {held * page_bytes / 1e6:.1f} MB ({dense / 1e6:.1f} MB as bf16 rows)")

    # 2. their answers share them
    akv.akv_pages_fork(p, pages, torch.arange(B, **int32).repeat_interleave(answers), ids[B:])
    say(f"{rows - B} answers: still {int((refs > 0).sum())} pages, the busiest with {int(refs.max())} holders")

    # 3. generation: the answers only; a query is near some keys of its own request
    one = (ids >= B).int()
    out, lse = torch.empty((rows, 1, heads * group, D), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, 1, heads * group), device="cuda")
    kept, kept_lse = torch.empty_like(out), torch.empty_like(lse)
    share, cosine = torch.zeros(2, device="cuda")
    answering = ids[B:]
    for _ in range(steps):
        put(one, 1)
        at = torch.randint(0, 32, (rows,), generator=gen, device="cuda")
        q = ck[at].repeat_interleave(group, 1)[:, None] + 0.7 * torch.randn((rows, 1, heads * group, D), generator=gen, device="cuda")
        q = q.to(torch.bfloat16)
        akv.akv_pages_share(p, pages, sharing, ws=ws)  # (once a step: it holds for every layer)
        akv.akv_paged_attn_shared(p, pages, q, out, sharing, lse=lse, sm_scale=1 / math.sqrt(D), ws=ws)
        akv.akv_paged_select(p, pages, q, sel, sink=1, recent=2, ws=ws)
        akv.akv_paged_attn(p, pages, q, kept, lse=kept_lse, sel=sel, sm_scale=1 / math.sqrt(D), ws=ws)
        share += (kept_lse - lse)[answering].exp().mean() / steps
        cosine += torch.cosine_similarity(out[answering].float(), kept[answering].float(), dim=-1).mean() / steps
    share, cosine = float(share), float(cosine)
    assert pool_pages or int(lacked) == 0
    say(f"{steps} steps: {int((refs > 0).sum())} pages; the {top} pages kept of up to {max_pages} hold {share:.3f} of the "
        f"softmax, outputs' cosine {cosine:.4f}")
    put(one * draft, draft)
    q = torch.randn((rows, draft, heads * group, D), generator=gen, device="cuda").to(torch.bfloat16)
    checked = torch.empty_like(q)
    akv.akv_paged_attn(p, pages, q, checked, sm_scale=1 / math.sqrt(D), ws=ws)

    # 4. all answers but the last of each prompt end
    done = [B + b * answers + a for b in range(B) for a in range(answers - 1)]
    akv.akv_pages_free(p, pages, torch.tensor(done, **int32))
    n_live = torch.zeros(1, **int32)
    before = torch.empty_like(checked)
    akv.akv_paged_attn(p, pages, q, before, sm_scale=1 / math.sqrt(D), ws=ws)
    akv.akv_pages_compact(p, pages, n_live, ws=ws)
    after = torch.empty_like(checked)
    akv.akv_paged_attn(p, pages, q, after, sm_scale=1 / math.sqrt(D), ws=ws)
    unmoved = torch.equal(before, after)
    say(f"freed {len(done)} answers, compacted: {int(n_live)} pages live, outputs unchanged: {unmoved}")

    # 5. the longest prompt goes to the anchor-residual cache, if its query groups are of a size that it takes
    agree = None
    if group in (1, 2, 4, 8):
        S = int(lens[0])
        K, V = (torch.empty((rows, heads, S, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        akv.akv_paged_read(p, pages, K.transpose(1, 2), V.transpose(1, 2))
        a = akv.Params(batch=1, n_kv_heads=heads, n_q_heads=heads * group, anchor_frac=0.04, res_frac_k=0.2, res_frac_v=0.2)
        arena_bytes, scratch_bytes = akv.akv_cache_size(a, [S])
        arena, scratch = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (arena_bytes, scratch_bytes))
        akv.akv_encode(a, [S], K[:1].contiguous(), V[:1].contiguous(), arena, scratch)
        q1 = q[:1, 0].contiguous()
        far = torch.empty_like(q1)
        akv.akv_decode_attn(a, [S], arena, q1, far, sm_scale=1 / math.sqrt(D))
        qs, near = torch.zeros((rows, 1, heads * group, D), dtype=torch.bfloat16, device="cuda"), torch.empty_like(out)
        qs[0, 0] = q1[0]
        akv.akv_paged_attn(p, pages, qs, near, sm_scale=1 / math.sqrt(D), ws=ws)
        agree = float(torch.cosine_similarity(near[0, 0].float(), far[0].float(), dim=-1).mean())
        say(f"prompt of {S} tokens: {-(-S // page) * page_bytes / 1e6:.2f} MB in pages, {arena_bytes / 1e6:.2f} MB as anchors and "
            f"residuals; outputs' cosine {agree:.4f}")
    return dict(share=share, cosine=cosine, unmoved=unmoved, agree=agree, live=int(n_live), lacked=int(lacked), table=table, lens=lens, refs=refs)


def within_budget(heads=8, group=4, steps=32, budget=512, window=32, sink=4, prompts=(3000, 1777, 940), answers=3, page=64, seed=0, verbose=True):
    """Rows of at most `budget` tokens, but for those of the steps since they were last cut."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    say = print if verbose else (lambda *a: None)
    B, n = len(prompts), len(prompts) * answers
    rows = B + 2 * n  # the prompts, the answers, and the rows that they go to when they are cut
    most = max(max(prompts), budget) + steps
    max_pages = -(-most // page)
    n_pages = sum(-(-x // page) for x in prompts) + 2 * n * (2 + (budget + steps) // page)
    p = akv.PagedParams(n_kv_heads=heads, n_q_heads=heads * group, page_tokens=page, rotate=True)
    int32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, n_pages, akv.akv_paged_page_bytes(p)), dtype=torch.uint8, device="cuda")
    table = torch.full((rows, max_pages), -1, **int32)
    lens, refs, missing, lacked = torch.zeros(rows, **int32), torch.zeros(n_pages, **int32), torch.zeros(1, **int32), torch.zeros(1, **int32)
    pages = akv.Pages(p, pool, table, lens, refs)
    sharing = akv.PageShare(torch.empty((4, rows), **int32))
    scores = torch.zeros((rows, heads, max_pages * page), device="cuda")
    ws = torch.empty(max(akv.akv_pages_workspace_size(pages), *(f(p, pages, T) for T in (1, window) for f in (
        akv.akv_paged_attn_shared_workspace_size, akv.akv_paged_weights_workspace_size))), dtype=torch.uint8, device="cuda")
    ck, cv = torch.randn((2, 32, heads, D), generator=gen, device="cuda")
    ids = torch.arange(rows, **int32)

    def reserve(n_new):
        akv.akv_pages_reserve(p, pages, n_new, missing, ws=ws)
        torch.maximum(lacked, missing, out=lacked)

    def put(n_new, T):
        reserve(n_new)
        n_new = n_new * (missing == 0)
        akv.akv_paged_append(p, pages, clustered(gen, ck, (rows, T, heads), True), clustered(gen, cv, (rows, T, heads), False), n_new=n_new)
        lens.add_(n_new)

    def queries(T):
        at = torch.randint(0, 32, (rows, T), generator=gen, device="cuda")
        return (ck[at].repeat_interleave(group, 2) + 0.7 * torch.randn((rows, T, heads * group, D), generator=gen, device="cuda")).to(torch.bfloat16)

    def attend(q, decay):
        """Attention of the rows that hold tokens, and what it adds to the scores (none: not added up)."""
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        akv.akv_pages_share(p, pages, sharing, ws=ws)
        akv.akv_paged_attn_shared(p, pages, q, out, sharing, lse=lse, sm_scale=1 / math.sqrt(D), ws=ws)
        if decay is not None:
            akv.akv_paged_weights(p, pages, q, lse, scores, was=scores, decay=decay, sm_scale=1 / math.sqrt(D), ws=ws)
        return out, lse

    def cut(src, dst):
        kept = akv.KeptTokens(torch.empty((len(src), heads, budget), **int32), torch.empty(len(src), **int32))
        akv.akv_paged_evict(p, pages, src, dst, scores, kept, sink=sink, recent=window)
        lens[dst.long()] = kept.count.clamp(min=0)  # (every layer of a model has the same counts)

    def forget():
        """A new token's weights are added to what stands at its place: behind what rows hold, that is of tokens that are gone."""
        scores.masked_fill_((torch.arange(scores.shape[2], device="cuda") >= lens[:, None])[:, None], 0)

    # 1. the prompts; their last tokens' queries say which of their tokens stay
    chunk = 1024
    want = torch.tensor(list(prompts) + [0] * (rows - B), **int32)
    for _ in range(0, max(prompts), chunk):
        put((want - lens).clamp(0, chunk), chunk)
    whole = int((refs > 0).sum())
    attend(queries(window), 0.0)
    q = queries(1)
    before, all_lse = attend(q, None)
    cut(ids[:B], ids[:B])
    akv.akv_pages_trim(p, pages, ids[:B])
    forget()
    after, lse = attend(q, None)
    mass = float((lse - all_lse)[:B].exp().mean())
    cosine = float(torch.cosine_similarity(before[:B].float(), after[:B].float(), dim=-1).mean())
    say(f"prompts of {sum(prompts)} tokens cut to {int(lens.sum())}: {whole} pages before, {int((refs > 0).sum())} now; what stays holds {mass:.3f} of the "
        f"softmax, outputs' cosine {cosine:.4f}")

    # 2. the answers share what is left, and grow
    akv.akv_pages_fork(p, pages, ids[:B].repeat_interleave(answers), ids[B : B + n])
    scores[B : B + n] = scores[:B].repeat_interleave(answers, 0)
    now, spare = ids[B : B + n], ids[B + n :]
    for step in range(steps):
        new = torch.zeros(rows, **int32)
        new[now.long()] = 1
        put(new, 1)
        attend(queries(1), 0.95)
        if step == steps // 2:
            # 3. they are cut into rows of their own: pages that others hold are not written
            room = torch.zeros(rows, **int32)
            room[spare.long()] = torch.minimum(lens[now.long()], torch.full_like(now, budget))
            reserve(room)
            cut(now, spare)
            akv.akv_pages_free(p, pages, now)
            forget()
            now, spare = spare, now
    say(f"{n} answers of {int(lens[now.long()].min())} to {int(lens[now.long()].max())} tokens: {int((refs > 0).sum())} pages")
    return dict(mass=mass, cosine=cosine, lens=lens[now.long()], lacked=int(lacked), table=table, refs=refs, scores=scores)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("heads", 8), ("group", 4), ("steps", 32), ("top", 16), ("answers", 3), ("page", 64), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--budget", type=int, default=512)
    args = vars(ap.parse_args())
    budget = args.pop("budget")
    main(**args)
    args.pop("top")
    within_budget(budget=budget, **args)
