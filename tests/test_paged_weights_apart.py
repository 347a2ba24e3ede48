"""akv_paged_weights reads `was` while it writes `now`: the same numbers, or apart.  No GPU: the call is refused for its workspace, after this."""
import random

import pytest

import paper_2608_02901_gb300 as akv
from test_paged_abi import AT, INVALID, pages, params, refused
from test_paged_more_abi import built, scores, weights  # noqa: F401 - the fixture

N, ROWS, HEADS = 160, 5, 2  # numbers of a head, of the pages' and parameters' rows and heads
OTHER = "was lies on other numbers of now"


def given(was, now, decay=1.0, rows=ROWS, heads=HEADS):
    p, g = params(n_kv_heads=heads, n_q_heads=4 * heads), pages(rows=rows)
    g.pool_bytes = g.layer_stride = 1 << 50  # (as many heads as it takes)
    g.n_layers = 1
    return weights(p=p, g=g, was=lambda: scores(**was), now=lambda: scores(**now), decay=decay, ws=None)


def passes(*a, **kw):
    refused(INVALID, "workspace", *given(*a, **kw))


def view(at=0, b=HEADS * N, h=N):
    return dict(ptr=AT + 4 * at, stride_b=b, stride_h=h, cap=N)


def test_the_same_or_apart():
    passes(view(), view())
    passes(view(ROWS * HEADS * N), view())
    passes(view(), view(ROWS * HEADS * N))
    # halves of one array, taken by turns
    for first, second in ((0, N), (N, 0)):
        passes(view(first, 4 * N, 2 * N), view(second, 4 * N, 2 * N))
    passes(view(0, 4 * N, N), view(2 * N, 4 * N, N))
    passes(view(0, N, 10 * N), view(5 * N, N, 10 * N))
    # numbers for all rows, read again and again
    passes(view(ROWS * HEADS * N, 0, 0), view())
    # an axis of one has no stride
    passes(view(0, 7, N), view(0, 0, N), rows=1)
    passes(view(0, N, 3), view(0, N, 10**6), heads=1)


@pytest.mark.parametrize("was,now", [
    (view(1), view()), (view(), view(1)), (view(N), view()), (view(HEADS * N), view()), (view(), view(ROWS * HEADS * N - 1)),
    (view(), view(0, 3 * N)), (view(0, 3 * N), view()), (view(0, 0, 0), view()), (view(0, N, 5 * N), view()), (view(3, 4 * N, 2 * N), view(N, 4 * N, 2 * N))])
def test_on_top_of_one_another(was, now):
    refused(INVALID, OTHER, *given(was, now))
    passes(was, now, decay=0.0)  # it is not read


def test_strides_out_of_range():
    refused(INVALID, "was: strides out of range", *given(view(0, 2**61), view()))
    refused(INVALID, "was: strides out of range", *given(view(0, N, 2**62), view()))


def test_against_all_numbers():
    """Strides and distances of every kind, against the places themselves."""
    rng = random.Random(3)
    found = [0, 0]
    for _ in range(1500):
        rows, heads = rng.choice([1, 2, 3, 5]), rng.choice([1, 2, 3])
        near = N + rng.choice([0, 0, 1, 40, N, 3 * N])
        if rng.random() < 0.5:
            now = (near * heads + rng.choice([0, 0, 5, N, near]), near)
        else:
            now = (near, near * rows + rng.choice([0, 0, 5, N, near]))
        was = now if rng.random() < 0.4 else (rng.choice([0, 7, N, near, now[0], 2 * now[0]]), rng.choice([0, N, near, now[1], 2 * now[1]]))
        d = rng.choice([0, 1, N - 1, N, near - N, near, now[0], now[1], 2 * N, 10 * N]) * rng.choice([-1, 1]) + rng.choice([0, 0, 0, 1, -1])
        starts = {(b, h): b * now[0] + h * now[1] for b in range(rows) for h in range(heads)}
        clash = any(abs(d + b * was[0] + h * was[1] - x) < N and not (d + b * was[0] + h * was[1] == x and at == (b, h))
                    for b in range(rows) for h in range(heads) for at, x in starts.items())
        found[clash] += 1
        base = 1 << 16
        a, b = view(base + d, *was), view(base, *now)
        if clash:
            refused(INVALID, OTHER, *given(a, b, rows=rows, heads=heads))
        else:
            passes(a, b, rows=rows, heads=heads)
    assert min(found) > 300, found
