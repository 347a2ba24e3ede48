"""Launches of the paged cache run beside the ones before them in their stream: each waits before it reads what those wrote."""
import os
import re

import pytest

import paper_2608_02901_gb300 as akv

CSRC = os.path.join(os.path.dirname(os.path.abspath(akv.__file__)), "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if re.match(r"akv_page.*\.cu$", f))
# What a kernel may do before it waits: its barriers in shared memory, its own place, the signs that it was launched with.
BEFORE = {"launch_dependents", "mbar_init", "smem_u32", "volatile", "asm", "__shfl_sync", "max", "min", "if", "for", "of", "this_cluster", "rank", "__align__", "sizeof", "warps_of", "stages_of", "subs_of", "fill_signs"}


def kernels(name):
    """Names and bodies of a file's kernels, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    for m in re.finditer(r"__global__", text):
        at = text.index("{", m.end())
        depth, end = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if depth == 0:
                break
        head = text[m.end() : at]
        yield re.findall(r"(akv_\w+)\s*\(", head)[-1], text[at + 1 : end - 1]


@pytest.mark.parametrize("file", FILES)
def test_kernels_wait_before_they_read(file):
    found = list(kernels(file))
    assert found
    for name, body in found:
        assert body.count("wait_for_stream();") == 1, name
        before = body[: body.index("wait_for_stream();")]
        calls = set(re.findall(r"([A-Za-z_]\w*)\s*\(", before))
        assert calls <= BEFORE, (name, calls - BEFORE)
        # at the body's own level, so that every thread comes by
        assert before.count("{") == before.count("}"), name
        assert not re.search(r"\breturn\b", before), name


@pytest.mark.gpu
def test_calls_back_to_back():
    """Queries, plans and groups that change from call to call in one workspace, with nothing between the calls."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from test_paged_cache import params, queries
    from test_paged_shared import grouped

    p = params(4, 8, 64, 64, False, True)
    shapes = [[(9000, [40] * 8), (700, [5, 9, 400])], [(300, [20] * 11)], [(64, [1] * 5), (5000, [700] * 6)]]
    cases = [grouped(p, groups, seed=i) for i, groups in enumerate(shapes)]
    calls = [(c, queries(c, T, 1.0)) for T in (1, 3, 8) for c in cases]
    ws = torch.empty(max(max(akv.akv_pages_workspace_size(c.pages), akv.akv_paged_attn_shared_workspace_size(p, c.pages, q.shape[1]))
                         for c, q in calls), dtype=torch.uint8, device="cuda")

    def run(between):
        outs = [(torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")) for _, q in calls]
        share = [akv.PageShare(torch.zeros((4, len(c.lens_h)), dtype=torch.int32, device="cuda"), True) for c, _ in calls]
        torch.cuda.synchronize()
        for (c, q), (out, lse), s in zip(calls, outs, share):
            akv.akv_pages_share(p, c.pages, s, ws=ws)
            akv.akv_paged_attn_shared(p, c.pages, q, out, s, lse=lse, sm_scale=0.1, ws=ws)
            between()
        torch.cuda.synchronize()
        return outs

    want = run(torch.cuda.synchronize)
    for _ in range(5):
        for (out, lse), (o, l) in zip(run(lambda: None), want):
            assert torch.equal(out, o) and torch.equal(lse, l)


def test_barriers_of_the_weights_belong_to_a_warpgroup():
    """A phase is told by its parity, so whoever waits must not fall two phases behind: a product warp has tiles only where its
    warpgroup has, and may wait only for barriers on which that warpgroup waits for it in turn."""
    (body,) = [body for name, body in kernels("akv_paged_weights.cu") if name == "akv_paged_weights_kernel"]
    waits = re.findall(r"mbar_wait_w\(smem_u32\(&S\.(\w+(?:\[\w+\])?)", body)
    assert waits and all(re.fullmatch(r"\w+\[w\]", x) for x in waits), waits
