"""The paged 4-bit cache on the GPU: append and read back, attention, page selection."""
import math

import numpy as np
import pytest

import paged_ref as ref
import paper_2608_02901_gb300 as akv

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(autouse=True)
def cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def params(H, G, page=64, group=64, half=False, rotate=False, bounds=False):
    return akv.PagedParams(n_kv_heads=H, n_q_heads=H * G, page_tokens=page, group=group, half=half, rotate=rotate,
                           bounds=bounds, rot_seed=77)


def dtype(p):
    return torch.float16 if p.half else torch.bfloat16


class Cache:
    """A cache whose pages lie scattered in a pool of 0xFF bytes (NaN scales) with room after each request."""

    def __init__(self, p, lens, seed=0, layers=1, room=1, extra=3):
        self.p, self.rng = p, np.random.default_rng(seed)
        self.lens_h = list(lens)
        most = max(-(-(n + room) // p.page_tokens) for n in lens)
        n_pages = len(lens) * most + extra
        ids = self.rng.permutation(n_pages)[: len(lens) * most].reshape(len(lens), most)
        self.table = torch.from_numpy(ids.astype(np.int32)).cuda()
        self.lens = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
        self.pool = torch.full((layers, n_pages, akv.akv_paged_page_bytes(p)), 255, dtype=torch.uint8, device="cuda")
        self.pages = akv.Pages(p, self.pool, self.table, self.lens)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def rows(self, T, scale=1.0):
        """Two [B][T][H][128] tensors, keys with outlier channels."""
        shape = (len(self.lens_h), T, self.p.n_kv_heads, D)
        k, v = torch.randn((2, *shape), generator=self.gen, device="cuda") * scale
        k[..., 5] *= 8
        return k.to(dtype(self.p)), v.to(dtype(self.p))

    def fill(self, scale=1.0, layer=0):
        """Appends every request's tokens at once; returns the dense rows."""
        T = max(self.lens_h)
        k, v = self.rows(max(T, 1), scale)
        n = torch.tensor(self.lens_h, dtype=torch.int32, device="cuda")
        akv.akv_paged_append(self.p, self.pages, k, v, n_new=n, layer=layer)
        self.lens.copy_(n)
        return k, v

    def ref(self, layer=0):
        return ref.Ref(self.p, self.pool[layer].cpu().numpy(), self.table.cpu().numpy(), self.lens.cpu().numpy())


def f64(t):
    return t.double().cpu().numpy()


# ---- append and read ---------------------------------------------------------------------

CODECS = [(16, 64, False, False), (64, 64, False, True), (32, 128, True, False), (128, 128, True, True)]


def check_codec(p, x, codes, a, m):
    """Codes, scales and minima of rows x (fp64 [..., 128]) against the definition.

    fp32 errors: v itself has at most 7 roundings of sums below sum |x| (times 1/8) when rotated; then the minimum and
    the scale are rounded to fp16 (half an ulp: 2^-11, or 2^-25 below the normal range), and t = (v - m) / a takes three
    roundings of a value of at most 15.5 and the error of v over a."""
    v = ref.rotated(x, p)
    ev = (7 * 2.0**-24 * np.abs(x).sum(-1, keepdims=True) / 8)[..., None] if p.rotate else 0.0
    v = v.reshape(*v.shape[:-1], D // p.group, p.group)
    lo, hi = v.min(-1, keepdims=True), v.max(-1, keepdims=True)
    a, m = a[..., None], m[..., None]
    c = codes.reshape(v.shape)
    sat = 65504.0
    want_m = np.clip(lo, -sat, sat)
    assert np.all(np.abs(m - want_m) <= 2.0**-11 * np.abs(want_m) + 2.0**-25 + ev)
    want_a = np.clip((hi - m) / 15, 0, sat)
    assert np.all(np.abs(a - want_a) <= (2.0**-11 + 2.0**-22) * want_a + 2.0**-25 + ev)
    safe = np.where(a > 0, a, 1)
    t = np.clip((v - m) / safe, 0, 15)
    assert np.all(np.where(a > 0, np.abs(c - t) <= 0.5 + 16 * 3 * 2.0**-24 + 2 * ev / safe, c == 0))


@pytest.mark.parametrize("page,group,half,rotate", CODECS)
def test_append_writes_the_codec(page, group, half, rotate):
    p = params(2, 1, page, group, half, rotate, bounds=True)
    c = Cache(p, [1, 16, 77, 300, 0, 129])
    k, v = c.fill()
    pool = c.pool[0].cpu().numpy().reshape(-1, 2, ref.block_bytes(p))
    for b, n in enumerate(c.lens_h):
        for j in range(-(-n // page)):
            pg = int(c.table[b, j])
            m_ = min(page, n - j * page)
            for h in range(2):
                codes, a, m = ref.rows_of_block(pool[pg, h], p)
                for side, rows in ((0, k), (1, v)):
                    x = f64(rows[b, j * page : j * page + m_, h])
                    check_codec(p, x, codes[side, :m_], a[side, :m_], m[side, :m_])
                    # what no token wrote is as it was
                    assert np.all(codes[side, m_:] == 15) and np.all(np.isnan(a[side, m_:]))
                bounds = pool[pg, h, -512:].copy().view(np.uint16)
                bounds = torch.from_numpy(bounds.view(np.int16)).view(dtype(p)).double().numpy().reshape(2, D)
                x = f64(k[b, j * page : j * page + m_, h])
                assert np.array_equal(bounds, np.stack((x.min(0), x.max(0))))
    written = {int(c.table[b, j]) for b, n in enumerate(c.lens_h) for j in range(-(-n // page))}
    rest = [i for i in range(c.pool.shape[1]) if i not in written]
    assert bool((c.pool[0, rest] == 255).all())


@pytest.mark.parametrize("page,group,half,rotate", CODECS)
def test_append_in_parts_is_append_at_once(page, group, half, rotate):
    p = params(3, 1, page, group, half, rotate, bounds=True)
    lens = [200, 37, 1, 150]
    one, parts = Cache(p, lens, seed=3), Cache(p, lens, seed=3)
    k, v = one.fill()
    done = torch.zeros(4, dtype=torch.int32, device="cuda")
    want = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for step in (1, 1, 30, 5, 64, 1, 200):
        n = torch.minimum(want - done, torch.full_like(done, step))
        take = (done[:, None] + torch.arange(step, device="cuda")).clamp(max=k.shape[1] - 1).long()
        kk, vv = (torch.take_along_dim(x, take[:, :, None, None], 1) for x in (k, v))
        akv.akv_paged_append(p, parts.pages, kk, vv, n_new=n)
        done += n
        parts.lens.copy_(done)
    assert torch.equal(done, want) and torch.equal(one.pool, parts.pool)


@pytest.mark.parametrize("page,group,half,rotate", CODECS)
def test_read_gives_what_the_bytes_stand_for(page, group, half, rotate):
    p = params(2, 1, page, group, half, rotate)
    c = Cache(p, [70, 5, 0, 200], seed=4)
    c.fill()
    r = c.ref()
    T = 90
    start = torch.tensor([0, 3, 0, 150], dtype=torch.int32, device="cuda")
    # heads before tokens, as the encoder takes its rows, in a wider buffer
    k, v = (torch.full((4, 2, T + 3, D), 7.0, dtype=dtype(p), device="cuda") for _ in range(2))
    akv.akv_paged_read(p, c.pages, k[:, :, 1 : T + 1].transpose(1, 2), v[:, :, 1 : T + 1].transpose(1, 2), start=start)
    ulp = 2.0**-11 if half else 2.0**-8
    for b, n in enumerate(c.lens_h):
        s = int(start[b])
        for side, got in ((0, k), (1, v)):
            got = f64(got)
            assert np.all(got[b, :, 0] == 7) and np.all(got[b, :, T + 1 :] == 7)
            have = max(0, min(T, n - s))
            want = ref.rotated_back(r.v[b][side, s : s + have], p).transpose(1, 0, 2)
            # one rounding to the rows' type; rotated, fp32 sums of 128 values as well
            tol = ulp * np.abs(want) + (8 * 2.0**-24 * 128 * np.abs(r.v[b][side]).max(initial=0) / 16 if rotate else 0) + 1e-30
            assert np.all(np.abs(got[b, :, 1 : have + 1] - want) <= tol)
            assert np.all(got[b, :, have + 1 : T + 1] == 0)


@pytest.mark.parametrize("rotate", [False, True])
def test_extreme_rows(rotate):
    """Constant rows, zeros, the largest and smallest numbers, infinities and NaN."""
    p = params(1, 1, 16, 64, False, rotate, bounds=True)
    x = torch.zeros((1, 8, 1, D))
    x[0, 1] = 3.25
    x[0, 2, 0, 7] = 3e38
    x[0, 3] = 1e-38 * torch.arange(D)
    x[0, 4, 0, 3] = math.inf
    x[0, 5, 0, 100] = math.nan
    x[0, 6] = torch.linspace(-70000, 70000, D)
    x[0, 7] = -0.0
    x = x.to(torch.bfloat16).cuda()
    c = Cache(p, [0], room=16)
    akv.akv_paged_append(p, c.pages, x, x)
    c.lens.fill_(8)
    k, v = torch.empty_like(x), torch.empty_like(x)
    akv.akv_paged_read(p, c.pages, k, v)
    for got in (f64(k)[0, :, 0], f64(v)[0, :, 0]):
        assert np.all(got[0] == 0) and np.all(got[7] == 0)
        assert np.all(np.isfinite(got[[0, 1, 2, 3, 6, 7]]))
        if rotate:  # the rotation spreads what is not finite over the row
            assert np.all(np.isnan(got[4:6]))
        else:
            assert np.all(got[1] == 3.25) and got[2, 7] <= 16 * 65504 and got[2, 7] >= 15 * 65504
            assert np.all(np.isnan(got[4, :64])) and np.all(got[4, 64:] == 0)
            assert np.all(np.isnan(got[5, 64:])) and np.all(got[5, :64] == 0)
            assert np.all(np.abs(got[6] - f64(x)[0, 6, 0]) <= 140000 / 15)


def test_append_keeps_to_the_table_and_the_pool():
    """Tokens past the table, on pages outside the pool, or none at all are not written."""
    p = params(1, 1, 16)
    c = Cache(p, [0, 0, 0, 0], room=32, extra=0)
    assert c.table.shape[1] == 2
    keep = c.table.clone()
    c.table[1, 1] = c.pool.shape[1]  # one past the pool
    c.table[2, 0] = -1
    k, v = c.rows(40)
    n = torch.tensor([40, 40, 40, -3], dtype=torch.int32, device="cuda")
    akv.akv_paged_append(p, c.pages, k, v, n_new=n)
    c.table.copy_(keep)
    c.lens.fill_(32)
    written = (c.pool[0].view(8, 2304)[:, 2048:2052] != 255).any(1).cpu().numpy()
    want = np.zeros(8, bool)
    want[keep.cpu().numpy()[[0, 0, 1, 2], [0, 1, 0, 1]]] = True
    assert np.array_equal(written, want)


# ---- attention ---------------------------------------------------------------------------


def check_attention(p, c, q, out, lse, sm_scale, kept=None, layer=0):
    """Bounds: the output's rounding (2^-8 or 2^-11); weights kept in fp16 (2^-11 of the values' range, summed over a
    rotated row at most eightfold); fp32 logits (128 products: 1e-5 of the sum of their magnitudes) move the weights by
    as much, again of the values' range."""
    want, want_lse, mass, spread = c.ref(layer).attend(f64(q), sm_scale, kept)
    back = 8 if p.rotate else 1
    el = 1e-5 * (1 + mass)
    tol = (2.0**-11 if p.half else 2.0**-8) * np.abs(want) + (back * (2.0**-11 + 2 * el) * spread)[..., None] + 1e-7
    got = f64(out)
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)
    if lse is not None:
        g = f64(lse)
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(g), empty)
        assert np.all(np.abs(g - want_lse)[~empty] <= el[~empty] + 1e-6)
        assert np.all(got[empty] == 0)


def queries(c, T, scale=1.5):
    p = c.p
    return (torch.randn((len(c.lens_h), T, p.n_q_heads, D), generator=c.gen, device="cuda") * scale).to(dtype(p))


def attend(c, q, sm_scale=1 / math.sqrt(D), sel=None, layer=0, **kw):
    out = torch.full_like(q, 9.0)
    lse = torch.full(q.shape[:3], 9.0, device="cuda")
    akv.akv_paged_attn(c.p, c.pages, q, out, lse=lse, sel=sel, sm_scale=sm_scale, layer=layer, **kw)
    return out, lse


LENS = [1, 0, 15, 16, 17, 127, 128, 129, 700]


@pytest.mark.parametrize("page,group,half,rotate", CODECS)
@pytest.mark.parametrize("G", [1, 3, 8])
def test_attention_of_single_tokens(page, group, half, rotate, G):
    p = params(2, G, page, group, half, rotate, bounds=G == 3)
    c = Cache(p, LENS, seed=G)
    c.fill()
    q = queries(c, 1)
    check_attention(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("G,T,rotate,group", [(4, 2, False, 64), (8, 2, True, 128), (3, 5, True, 64), (1, 9, False, 128), (8, 4, False, 64),
                                              (16, 1, True, 64), (12, 3, False, 128), (64, 1, False, 64), (1, 64, True, 128)])
def test_attention_of_drafts(G, T, rotate, group):
    """Several query tokens, causal among themselves; requests shorter than the draft have queries that see nothing."""
    p = params(1, G, 32, group, False, rotate)
    c = Cache(p, [0, 1, 3, 16, 64, 150, 401], seed=T)
    c.fill()
    q = queries(c, T)
    check_attention(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("G,page", [(4, 16), (8, 64), (1, 128)])
def test_attention_over_long_requests(G, page):
    """Requests that many CTAs share, and whose shares end inside a page."""
    p = params(2, G, page, 64, False, True)
    c = Cache(p, [9000, 5, 6001, 2500], seed=G)
    c.fill()
    q = queries(c, 1)
    check_attention(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("lens,page,G", [([300] * 40, 64, 2), ([1 + 7 * i % 61 for i in range(320)], 32, 1), ([390, 129] * 11, 128, 4),
                                         ([40] * 300 + [1500], 64, 1)])
def test_attention_of_batches(lens, page, G):
    """Units with CTAs of their own and cut ones, as many as CTAs and more, more requests than a CTA has threads."""
    p = params(1, G, page, 128, False, False)
    c = Cache(p, lens, seed=len(lens))
    c.fill()
    q = queries(c, 1)
    check_attention(p, c, q, *attend(c, q), 1 / math.sqrt(D))


@pytest.mark.parametrize("scale,sm", [(1e-3, 1.0), (30.0, 1.0), (2000.0, 1e-6), (1.0, -0.3), (1.0, 0.0)])
def test_attention_of_other_magnitudes(scale, sm):
    """Small and large values, peaked and flat softmaxes, a negative and a zero scale."""
    p = params(1, 4, 64, 64, True, False)
    c = Cache(p, [300, 1000, 64], seed=9)
    c.fill(scale=scale)
    q = queries(c, 1)
    check_attention(p, c, q, *attend(c, q, sm_scale=sm), sm)


def test_attention_of_rows_of_unlike_magnitude():
    """Value scales that differ by 2^20 among tokens, query rows that differ by 2^12."""
    p = params(1, 4, 16, 64, False, False)
    c = Cache(p, [200], seed=10)
    k, v = c.rows(200)
    v *= torch.exp2(torch.randint(-12, 9, (1, 200, 1, 1), generator=c.gen, device="cuda")).to(v.dtype)
    akv.akv_paged_append(p, c.pages, k, v)
    c.lens.fill_(200)
    q = queries(c, 1) * torch.tensor([1.0, 2.0**-12, 2.0**-6, 1e-30], device="cuda").to(torch.bfloat16)[:, None]
    check_attention(p, c, q, *attend(c, q), 1 / math.sqrt(D))


def test_attention_strides_layers_and_no_lse():
    p = params(2, 4, 32, 64, False, True)
    c = Cache(p, [100, 333], seed=11, layers=3)
    for layer in range(3):
        c.lens.zero_()
        c.fill(layer=layer)
    wide = torch.randn((2, 8, 2, D + 3), device="cuda").to(torch.bfloat16)  # [B][Hq][T][..]
    q = wide[..., 1 : D + 1].transpose(1, 2)
    buf = torch.full((2, 8, 2, D + 5), 9.0, dtype=torch.bfloat16, device="cuda")
    out = buf[..., 3 : D + 3].transpose(1, 2)
    akv.akv_paged_attn(p, c.pages, q, out, sm_scale=0.1, layer=2)
    check_attention(p, c, q, out, None, 0.1, layer=2)
    assert bool((buf[..., :3] == 9).all()) and bool((buf[..., D + 3 :] == 9).all())
    # one query for every request and head
    q = queries(c, 1)[:1, :, :1].expand(2, 1, 8, D)
    o = torch.empty((2, 1, 8, D), dtype=torch.bfloat16, device="cuda")
    akv.akv_paged_attn(p, c.pages, q, o, sm_scale=0.1)
    check_attention(p, c, q, o, None, 0.1)


def test_nan_reaches_only_who_sees_it():
    """A NaN value at one token: queries that see it are NaN, others are not; a page outside the pool likewise."""
    p = params(1, 2, 16, 64, False, False)
    c = Cache(p, [40, 40, 40], seed=12)
    k, v = c.rows(40)
    v[0, 38, 0, 3] = math.nan
    k[1, 39, 0, 3] = math.inf
    akv.akv_paged_append(p, c.pages, k, v)
    c.lens.fill_(40)
    c.table[2, 1] = c.pool.shape[1]
    q = queries(c, 4)
    out, lse = attend(c, q)
    out, lse = f64(out), f64(lse)
    # query tokens see 37, 38, 39, 40 tokens
    assert np.all(np.isfinite(out[0, :2])) and np.all(np.isnan(out[0, 2:, :, :64])) and np.all(np.isfinite(out[0, :, :, 64:]))
    assert np.all(np.isfinite(lse[0]))
    assert np.all(np.isfinite(out[1, :3])) and np.all(np.isnan(out[1, 3])) and np.all(np.isnan(lse[1, 3]))
    assert np.all(np.isnan(out[2])) and np.all(np.isnan(lse[2]))
    want, want_lse, _, _ = ref.Ref(p, c.pool[0].cpu().numpy(), c.table.cpu().numpy(), [40, 40, 0]).attend(f64(q), 1 / math.sqrt(D))
    assert np.allclose(out[0, :2], want[0, :2], atol=2e-2, rtol=1e-2) and np.allclose(out[1, :3], want[1, :3], atol=2e-2, rtol=1e-2)


def test_pages_beyond_four_gigabytes():
    p = params(8, 1, 128, 64)
    n_pages = (5 << 30) // akv.akv_paged_page_bytes(p)
    pool = torch.empty((1, n_pages, akv.akv_paged_page_bytes(p)), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    pages = akv.Pages(p, pool, table, lens)
    k, v = torch.randn((2, 1, 300, 8, D), device="cuda").to(torch.bfloat16)
    akv.akv_paged_append(p, pages, k, v)
    lens.fill_(300)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    akv.akv_paged_read(p, pages, k2, v2)
    # a step is at most a group's range (below 12 for these numbers) over 15, and a value at most half of one away
    assert float((k2.float() - k.float()).abs().max()) < 0.42 and float((v2.float() - v.float()).abs().max()) < 0.42
    q = torch.randn((1, 1, 8, D), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    akv.akv_paged_attn(p, pages, q, out, sm_scale=0.1)
    x = torch.einsum("bthd,bshd->bhs", q.double(), k2.double()) * 0.1
    want = torch.einsum("bhs,bshd->bhd", x.softmax(-1), v2.double())
    # the rows read back are rounded to bf16 (2^-9): logits of up to 5 move by 1e-2, weights by as much
    assert float((out[:, 0].double() - want).abs().max()) < 3e-2


def test_lengths_outside_the_table_are_clamped():
    p = params(1, 2, 16, bounds=True)
    c = Cache(p, [64, 64, 40], seed=18, room=0, extra=0)
    c.fill()
    assert c.table.shape[1] == 4
    q = queries(c, 2)
    c.lens.copy_(torch.tensor([64, 64, 0], dtype=torch.int32))
    want, sel = attend(c, q), selection(c, 2, 2)
    akv.akv_paged_select(p, c.pages, q, sel)
    c.lens.copy_(torch.tensor([65, 2**31 - 1, -5], dtype=torch.int32))
    got, sel2 = attend(c, q), selection(c, 2, 2)
    akv.akv_paged_select(p, c.pages, q, sel2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(sel.pages, sel2.pages) and torch.equal(sel.count, sel2.count)
    assert bool((got[0][2] == 0).all()) and bool(torch.isneginf(got[1][2]).all())
    before = c.pool.clone()
    k, v = c.rows(3)
    akv.akv_paged_append(p, c.pages, k[:, :3], v[:, :3], n_new=torch.tensor([3, 3, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(c.pool, before)  # no room


def test_parameters_must_be_the_pools():
    p = params(2, 4, 32)
    c = Cache(p, [10], seed=19)
    c.fill()
    q = torch.zeros((1, 1, 2, D), dtype=torch.bfloat16, device="cuda")
    akv.akv_paged_attn(params(2, 1, 32), c.pages, q, torch.empty_like(q))  # other query heads
    for other in (params(2, 1, 32, rotate=True), params(2, 1, 32, group=128), params(2, 1, 32, half=True), params(1, 2, 32)):
        with pytest.raises(ValueError):
            akv.akv_paged_attn(other, c.pages, q, torch.empty_like(q))


# ---- selection ---------------------------------------------------------------------------


def selection(c, T, top):
    B, H = len(c.lens_h), c.p.n_kv_heads
    return akv.PageSelection(torch.full((B, T, H, top), -7, dtype=torch.int32, device="cuda"),
                             torch.full((B, T, H), -7, dtype=torch.int32, device="cuda"))


def bounds_of(c, b, h):
    p = c.p
    pool = c.pool[0].view(-1, p.n_kv_heads, ref.block_bytes(p))
    n = -(-c.lens_h[b] // p.page_tokens)
    x = pool[c.table[b, :n].long(), h, -512:].contiguous().view(dtype(p)).view(n, 2, D)
    return f64(x)


def wanted(c, q, T, top, sink, recent):
    p = c.p
    return [[[ref.select(p, f64(q[b, t, h * p.G : (h + 1) * p.G]), bounds_of(c, b, h), n - T + 1 + t, top, sink, recent)
              for h in range(p.n_kv_heads)] for t in range(T)] for b, n in enumerate(c.lens_h)]


def check_selection(sel, want):
    pages, count = sel.pages.cpu().numpy(), sel.count.cpu().numpy()
    for b, xs in enumerate(want):
        for t, ys in enumerate(xs):
            for h, kept in enumerate(ys):
                assert count[b, t, h] == len(kept)
                assert pages[b, t, h, : len(kept)].tolist() == kept
                assert np.all(pages[b, t, h, len(kept) :] == -1)


@pytest.mark.parametrize("page,group,half,rotate", CODECS)
@pytest.mark.parametrize("G,T,top,sink,recent", [(1, 1, 4, 1, 1), (4, 2, 7, 0, 1), (8, 1, 3, 1, 2), (3, 3, 40, 2, 3), (16, 1, 5, 0, 0)])
def test_selection_and_attention_over_it(page, group, half, rotate, G, T, top, sink, recent):
    p = params(2, G, page, group, half, rotate, bounds=True)
    c = Cache(p, [0, 1, 3 * page, 20 * page + 5, 33 * page - 1, 10 * page + 1], seed=top)
    c.fill()
    q = queries(c, T)
    sel = selection(c, T, top)
    akv.akv_paged_select(p, c.pages, q, sel, sink=sink, recent=recent)
    want = wanted(c, q, T, top, sink, recent)
    check_selection(sel, want)
    if page <= 64:
        check_attention(p, c, q, *attend(c, q, sel=sel), 1 / math.sqrt(D), kept=want)


def test_selection_ties_go_to_the_lower_page():
    """Equal pages, and more of them than are kept; scores above and below zero."""
    p = params(1, 2, 16, bounds=True)
    c = Cache(p, [64 * 16], seed=1)
    k, v = c.rows(1024)
    k[:] = k[:, :16].repeat(1, 64, 1, 1)
    k[:, 16 * 40 : 16 * 41] *= 0  # one page apart
    akv.akv_paged_append(p, c.pages, k, v)
    c.lens.fill_(1024)
    q = queries(c, 1)
    for top in (1, 2, 9, 63):
        sel = selection(c, 1, top)
        akv.akv_paged_select(p, c.pages, q, sel, sink=0, recent=0)
        check_selection(sel, wanted(c, q, 1, top, 0, 0))
        assert sel.pages[0, 0, 0, 0] == 0
    for bad in (math.nan, math.inf):  # a query row that is no number scores nothing: the lowest pages
        q[0, 0, 1, 5] = bad
        sel = selection(c, 1, 9)
        akv.akv_paged_select(p, c.pages, q, sel, sink=0, recent=0)
        assert sel.pages[0, 0, 0].tolist() == list(range(9))


def test_selection_of_infinite_and_missing_pages():
    p = params(1, 1, 16, bounds=True)
    c = Cache(p, [50 * 16], seed=2)
    k, v = c.rows(800)
    k[0, 16 * 33 + 4, 0, 9] = math.inf
    akv.akv_paged_append(p, c.pages, k, v)
    c.lens.fill_(800)
    q = queries(c, 1)
    sel = selection(c, 1, 6)
    akv.akv_paged_select(p, c.pages, q, sel)
    want = wanted(c, q, 1, 6, 1, 1)
    assert 33 in want[0][0][0]
    check_selection(sel, want)
    best = [j for j in want[0][0][0] if 0 < j < 49 and j != 33]
    c.table[0, best[0]] = -1  # no page: chosen last
    akv.akv_paged_select(p, c.pages, q, sel)
    assert best[0] not in sel.pages[0, 0, 0].tolist() and int(sel.count[0, 0, 0]) == 6


@pytest.mark.parametrize("pages", [3000, 9001])
def test_selection_among_many_pages(pages):
    p = params(1, 4, 16, bounds=True)
    c = Cache(p, [16 * pages - 3, 16 * 70], seed=pages)
    c.fill()
    q = queries(c, 1)
    sel = selection(c, 1, 64)
    akv.akv_paged_select(p, c.pages, q, sel, sink=1, recent=2)
    check_selection(sel, wanted(c, q, 1, 64, 1, 2))


def test_attention_over_a_selection_of_the_callers_own():
    """Entries past the table or the request, or negative, attend nothing; an empty selection gives zeros."""
    p = params(1, 4, 32)
    c = Cache(p, [320, 320], seed=13)
    c.fill()
    q = queries(c, 1)
    sel = selection(c, 1, 8)
    sel.pages[0, 0, 0] = torch.tensor([0, 3, 9, 10, 500, -1, -5, 2**31 - 1], dtype=torch.int32)
    sel.pages[1] = 1
    sel.count[0], sel.count[1] = 8, 0
    out, lse = attend(c, q, sel=sel)
    check_attention(p, c, q, out, lse, 1 / math.sqrt(D), kept=[[[[0, 3, 9]]], [[[]]]])
    sel.count[0] = 1000  # read as the eight there are
    again, _ = attend(c, q, sel=sel)
    assert torch.equal(again, out)


# ---- streams and graphs ------------------------------------------------------------------


def test_graph_of_a_step_on_another_stream():
    """Append, selection and attention of a step captured once and replayed as lengths advance."""
    p = params(2, 4, 16, 64, False, True, bounds=True)
    c, d = Cache(p, [200, 90], seed=14, room=40), Cache(p, [200, 90], seed=14, room=40)
    c.fill(), d.fill()
    k, v = (torch.empty((2, 1, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.empty((2, 1, 8, D), dtype=torch.bfloat16, device="cuda")
    out, lse, sel = torch.empty_like(q), torch.empty((2, 1, 8), device="cuda"), selection(c, 1, 6)
    ws = torch.empty(max(akv.akv_paged_attn_workspace_size(p, c.pages, 1, 6), akv.akv_paged_select_workspace_size(p, c.pages, 1)),
                     dtype=torch.uint8, device="cuda")

    def step(cc):
        akv.akv_paged_append(p, cc.pages, k, v)
        cc.lens += 1
        akv.akv_paged_select(p, cc.pages, q, sel, ws=ws)
        akv.akv_paged_attn(p, cc.pages, q, out, lse=lse, sel=sel, sm_scale=0.1, ws=ws)

    side = torch.cuda.Stream()
    k.zero_(), v.zero_(), q.zero_()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    before = [t.clone() for t in (c.lens, c.pool)]
    with torch.cuda.stream(side):
        step(c)
    torch.cuda.synchronize()
    c.lens.copy_(before[0]), c.pool.copy_(before[1])
    with torch.cuda.graph(graph):
        step(c)
    for i in range(20):
        g = torch.Generator(device="cuda").manual_seed(100 + i)
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        got = out.clone(), lse.clone(), sel.pages.clone()
        step(d)
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, sel.pages)))
    assert torch.equal(c.lens, d.lens) and torch.equal(c.pool, d.pool)


def test_calls_repeat_bit_for_bit():
    p = params(4, 8, 64, 64, False, True, bounds=True)
    c = Cache(p, [5000, 1200, 77], seed=15)
    c.fill()
    q = queries(c, 1)
    first = attend(c, q)
    for _ in range(5):
        again = attend(c, q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- rows that are not aligned -----------------------------------------------------------


@pytest.mark.parametrize("half,rotate", [(False, True), (True, False)])
def test_rows_at_odd_addresses(half, rotate):
    """Keys, values, queries and outputs two bytes off every alignment give what aligned ones give, bit for bit."""
    p = params(2, 4, 32, 64, half, rotate, bounds=True)
    c, d = Cache(p, [100, 45], seed=16), Cache(p, [100, 45], seed=16)

    def odd(t):
        wide = torch.zeros((*t.shape[:-1], D + 3), dtype=t.dtype, device="cuda")
        view = wide[..., 1 : D + 1]
        view.copy_(t)
        assert view.data_ptr() % 4 == 2
        return view

    k, v = c.rows(100)
    n = torch.tensor([100, 45], dtype=torch.int32, device="cuda")
    akv.akv_paged_append(p, c.pages, k, v, n_new=n)
    akv.akv_paged_append(p, d.pages, odd(k), odd(v), n_new=n)
    c.lens.copy_(n), d.lens.copy_(n)
    assert torch.equal(c.pool, d.pool)
    k2, v2, k3, v3 = torch.empty_like(k), torch.empty_like(v), odd(k), odd(v)
    akv.akv_paged_read(p, c.pages, k2, v2)
    akv.akv_paged_read(p, d.pages, k3, v3)
    assert torch.equal(k2, k3) and torch.equal(v2, v3)
    q = queries(c, 2)
    sel, sel2 = selection(c, 2, 2), selection(c, 2, 2)
    akv.akv_paged_select(p, c.pages, q, sel)
    akv.akv_paged_select(p, d.pages, odd(q), sel2)
    assert torch.equal(sel.pages, sel2.pages)
    out, out2 = torch.empty_like(q), odd(q)
    akv.akv_paged_attn(p, c.pages, q, out, sm_scale=0.1)
    akv.akv_paged_attn(p, d.pages, odd(q), out2, sm_scale=0.1)
    assert torch.equal(out, out2)


def test_many_tiles_per_cta_repeat_bit_for_bit():
    """Long requests with cold caches, one scale a row: copies that come out of order change nothing."""
    for group, G, T in ((128, 4, 1), (64, 8, 1), (128, 4, 4)):
        p = params(8, G, 64, group, False, False)
        n_pages = 4 * 1024
        gen = torch.Generator(device="cuda").manual_seed(17)
        pool = torch.zeros((1, n_pages, 8, 4, 2048 + 128 * (D // group)), dtype=torch.uint8, device="cuda")
        pool[..., :2048] = torch.randint(0, 256, pool[..., :2048].shape, generator=gen, device="cuda", dtype=torch.uint8)
        words = torch.rand(pool[..., 2048:].shape[:-1] + (64 * (D // group), ), generator=gen, device="cuda")
        words[..., 0::2] = 0.1 + 0.1 * words[..., 0::2]  # scales
        words[..., 1::2] = -1.0 - words[..., 1::2]  # minima
        pool[..., 2048:] = words.half().view(torch.uint8)
        table = torch.randperm(n_pages, generator=gen, device="cuda").int().view(4, 1024)
        lens = torch.tensor([65536, 65000, 40001, 65535], dtype=torch.int32, device="cuda")
        pages = akv.Pages(p, pool.view(1, n_pages, -1), table, lens)
        q = torch.randn((4, T, 8 * G, D), generator=gen, device="cuda").to(torch.bfloat16)
        flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
        first = None
        for _ in range(20):
            flush.zero_()
            out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
            akv.akv_paged_attn(p, pages, q, out, lse=lse, sm_scale=0.1)
            assert bool(torch.isfinite(lse).all())
            if first is None:
                first = out, lse
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
