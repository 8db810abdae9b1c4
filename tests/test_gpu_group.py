"""The MoE layer's operators on any number of tokens (routing and row maps,
grouped products with their gradients, fp8 blocks, combine) against plain
64-bit forms on the same inputs.  Each element's bound counts the roundings of
its own sum; nothing is measured first."""
import numpy as np
import pytest
import torch

import group_util as ref
from group_util import BF16, D, F32
from gpu_util import DEV

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None


def gen(*seed):
    return torch.Generator().manual_seed(int(np.random.SeedSequence(seed).generate_state(1)[0]))


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def dev(*ts_):
    out = [None if t is None else t.to(DEV) for t in ts_]
    return out[0] if len(out) == 1 else out


def within(got, want, bound, what=""):
    got = got.detach().to(want.device).double()
    assert got.shape == want.shape, (got.shape, want.shape)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((got - want).abs().max()), bad.nonzero()[:4].tolist())


def untouched(got, ok_rows, fill):
    rest = torch.ones(got.shape[0], dtype=torch.bool)
    rest[ok_rows] = False
    assert bool((got.cpu()[rest] == fill).all())


# --- routing -----------------------------------------------------------------

ROUTES = [(1, 8, 2), (1, 1, 1), (2, 64, 8), (37, 40, 6), (128, 8, 8), (500, 8, 2), (513, 16, 2), (777, 64, 6),
          (2500, 3, 3), (20000, 64, 8)]


def check_route(logits, K, got):
    idx, w, offsets, row_token, pair_row = [t.cpu() for t in got]
    ri, rw, ro, rt, rp = ref.route(logits, K)
    assert torch.equal(idx, ri)
    # exp of a difference rounded once, K of them added, one quotient
    assert bool(((w.double() - rw).abs() <= (12 + K + logits.nan_to_num(0, 0, 0).abs().max().item()) * 2.0 ** -23).all())
    assert torch.equal(offsets, ro) and torch.equal(row_token, rt) and torch.equal(pair_row, rp)


@pytest.mark.parametrize("T,E,K", ROUTES)
def test_route(T, E, K):
    logits = randn(gen(1, T, E), T, E)
    check_route(logits, K, ts.moe_route(dev(logits), K))
    i, w = ts.moe_route(dev(logits), K, maps=False)
    assert torch.equal(i.cpu(), ref.route(logits, K)[0])


@pytest.mark.parametrize("T", [3, 1200])
def test_route_ties_and_non_finite(T):
    """Exact ties, both zeros, masked experts (-inf, the lowest value), rows
    with nothing left, NaN, +inf."""
    E, K = 16, 4
    g = gen(2, T)
    logits = torch.randint(-2, 3, (T, E), generator=g).float()
    logits[0] = -float("inf")
    logits[1] = torch.finfo(F32).min
    logits[1, 5] = 0.0
    logits[2] = float("nan")
    if T > 8:
        logits[3] = 0.0
        logits[3, ::2] = -0.0
        logits[4, 3:] = -float("inf")
        logits[5, 7] = logits[5, 2] = float("inf")
        logits[6, 1::2] = float("nan")
        logits[7, 0], logits[7, 1:] = float("nan"), -float("inf")
    got = ts.moe_route(dev(logits), K)
    idx, w, offsets, row_token, pair_row = [t.cpu() for t in got]
    ri, rw, ro, rt, rp = ref.route(logits, K)
    assert torch.equal(idx, ri)
    assert torch.isfinite(w).all() and bool(((w.double() - rw).abs() <= 24 * 2.0 ** -23).all())
    assert bool((w[0] == 0).all()) and bool((w[2] == 0).all())
    assert torch.equal(offsets, ro) and torch.equal(row_token, rt) and torch.equal(pair_row, rp)


@pytest.mark.parametrize("T,E,K", [(1, 4, 2), (300, 8, 2), (5000, 64, 3)])
def test_group_of_given_choices(T, E, K):
    """Given choices, the same expert twice among them, some out of range:
    those get no row, and the rows behind the last stay as they were."""
    g = gen(3, T, E)
    idx = torch.randint(-1, E + 1, (T, K), generator=g, dtype=torch.int32)
    offsets, row_token, pair_row = ts.moe_group(dev(idx), E)
    ro, rt, rp = ref.group(idx, E)
    assert torch.equal(offsets.cpu(), ro) and torch.equal(pair_row.cpu(), rp)
    assert torch.equal(row_token.cpu()[:len(rt)], rt)


def test_route_no_tokens():
    i, w, o, t, p = ts.moe_route(torch.empty(0, 8, device=DEV), 2)
    assert o.cpu().tolist() == [0] * 9 and i.shape == (0, 2) and t.numel() == 0
    o, t, p = ts.moe_group(torch.empty(0, 2, dtype=torch.int32, device=DEV), 5)
    assert o.cpu().tolist() == [0] * 6


@pytest.mark.parametrize("T,E,K", [(1, 8, 2), (333, 64, 6), (4000, 40, 8)])
def test_route_grad(T, E, K):
    g = gen(4, T, E)
    logits, d_w = randn(g, T, E), randn(g, T, K)
    idx, w, *_ = ts.moe_route(dev(logits), K)
    got = ts.moe_route_grad(idx, w, dev(d_w), E)
    wl, il = w.cpu().double(), idx.cpu().long()
    dot = (wl * d_w.double()).sum(1, keepdim=True)
    want = torch.zeros(T, E, dtype=D).scatter_(1, il, wl * (d_w.double() - dot))
    mag = torch.zeros(T, E, dtype=D).scatter_(1, il, wl * (d_w.abs().double() + (wl * d_w.abs()).sum(1, keepdim=True)))
    within(got, want, ref.sum_bound(mag, K + 3))


def test_route_grad_against_differences():
    g = gen(5)
    T, E, K, h = 6, 12, 3, 1e-6
    logits, d_w = randn(g, T, E), randn(g, T, K)
    idx, w, *_ = ts.moe_route(dev(logits), K)
    got = ts.moe_route_grad(idx, w, dev(d_w), E).cpu().double()
    il = idx.cpu().long()

    def loss(l):
        return (torch.softmax(l.gather(1, il), 1) * d_w.double()).sum(1)
    for e in range(E):
        step = torch.zeros(T, E, dtype=D)
        step[:, e] = h
        diff = (loss(logits.double() + step) - loss(logits.double() - step)) / (2 * h)
        # differences: third derivative h^2 and 2^-53 / h; the kernel: fp32
        assert bool(((got[:, e] - diff).abs() <= 1e-5 * (1 + d_w.abs().sum(1))).all())


# --- grouped products -----------------------------------------------------------

# rows, groups, n, k: one row, fewer rows than groups, tiles that end inside,
# contractions shorter than a step, rows per group around every tile size
SHAPES = [(1, 1, 8, 8), (2, 8, 136, 72), (5, 64, 64, 128), (40, 3, 200, 264), (97, 4, 512, 8), (150, 4, 24, 520),
          (260, 4, 392, 136), (530, 3, 272, 328), (1100, 2, 520, 200), (900, 1, 128, 1032)]


def product(rows, G, n, k, dtype, w_kn=False, gather=False, lead=0, tail=0, seed=0):
    g = gen(10, rows, G, n, k, seed)
    offsets = ref.ragged(rows, G, g, lead, tail)
    src = torch.randint(0, max(rows // 2, 1), (rows,), generator=g, dtype=torch.int32) if gather else None
    S = max(rows // 2, 1) if gather else rows
    x = randn(g, S, k, dtype=dtype)
    w = randn(g, G, *((k, n) if w_kn else (n, k)), dtype=dtype, scale=k ** -0.5)
    return x, w, offsets, src, g


@pytest.mark.parametrize("rows,G,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w_kn", [False, True])
def test_grouped_mm(rows, G, n, k, dtype, w_kn):
    for gather, odt in ((False, F32), (True, BF16)):
        x, w, offsets, src, g = product(rows, G, n, k, dtype, w_kn, gather)
        y, mag = ref.mm(x, w, offsets, src, w_kn)
        got = ts.grouped_mm(*dev(x, w, offsets), row_src=dev(src), w_kn=w_kn, out_dtype=odt)
        assert got.dtype == odt
        within(got, y, ref.rounded(ref.sum_bound(mag, k), y, odt))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,lead,tail", [(50, 3, 7), (700, 130, 41), (64, 64, 0), (300, 0, 299)])
def test_rows_outside_the_groups_stay(dtype, rows, lead, tail):
    x, w, offsets, src, g = product(rows, 4, 136, 72, dtype, lead=lead, tail=tail)
    x[:lead], x[rows - tail:] = float("nan"), float("inf")
    y, mag = ref.mm(x, w, offsets)
    out = torch.full((rows, 136), 7.0, device=DEV)
    c, gt, up = (torch.full((rows, 136), 7.0, device=DEV) for _ in range(3))
    ts.grouped_mm(*dev(x, w, offsets), out=out)
    ts.grouped_drelu(dev(x), dev(w), dev(w), dev(offsets), out=c)
    mid = slice(lead, rows - tail)
    within(out[mid], y[mid], ref.sum_bound(mag[mid], 72))
    for t in (out, c):
        untouched(t, mid, 7.0)
    assert torch.isfinite(c).all()


def test_one_dense_group_without_offsets():
    x, w, _, _, g = product(333, 1, 264, 520, BF16)
    y, mag = ref.mm(x, w, torch.tensor([0, 333]))
    within(ts.grouped_mm(*dev(x, w)), y, ref.rounded(ref.sum_bound(mag, 520), y, BF16))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w_kn", [False, True])
@pytest.mark.parametrize("rows,G,n,k", [(7, 2, 40, 24), (300, 3, 264, 200), (640, 2, 256, 128)])
def test_two_products_in_one(dtype, w_kn, rows, G, n, k):
    x, w, offsets, src, g = product(rows, G, n, k, dtype, w_kn)
    x2, w2 = randn(g, rows, k, dtype=dtype), randn(g, *w.shape, dtype=dtype)
    (a, ma), (b, mb) = ref.mm(x, w, offsets, None, w_kn), ref.mm(x2, w2, offsets, None, w_kn)
    got = ts.grouped_mm(*dev(x, w, offsets), x2=dev(x2), w2=dev(w2), w_kn=w_kn)
    within(got, a + b, ref.rounded(ref.sum_bound(ma + mb, 2 * k), a + b, dtype))


@pytest.mark.parametrize("rows,G,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_grouped_drelu(rows, G, n, k, dtype):
    x, wg, offsets, src, g = product(rows, G, n, k, dtype, gather=True)
    wu = randn(g, *wg.shape, dtype=dtype, scale=k ** -0.5)
    (gt, mg), (up, mu) = ref.mm(x, wg, offsets, src), ref.mm(x, wu, offsets, src)
    eg, eu = ref.sum_bound(mg, k), ref.sum_bound(mu, k)
    c = ref.drelu(gt, up)
    bound = ref.drelu_bound(gt, up, eg, eu)
    args = dev(x, wg, wu, offsets)
    got = ts.grouped_drelu(*args, row_src=dev(src), out_dtype=F32)
    within(got, c, bound + 2.0 ** -23 * c.abs())
    got, g2, u2 = ts.grouped_drelu(*args, row_src=dev(src), keep=True)
    within(got, c, ref.rounded(bound + 2.0 ** -23 * c.abs(), c, dtype))
    within(g2, gt, ref.rounded(eg, gt, dtype))
    within(u2, up, ref.rounded(eu, up, dtype))


@pytest.mark.parametrize("rows,G,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_mm_dw(rows, G, n, k, dtype, gather):
    x, _, offsets, src, g = product(rows, G, n, k, dtype, gather=gather)
    d_y = randn(g, rows, n, dtype=dtype)
    y, mag = ref.dw(d_y, x, offsets, src)
    terms = max(b - a for _, a, b in ref.spans(offsets))
    got = ts.grouped_mm_dw(*dev(d_y, x, offsets), row_src=dev(src))
    within(got, y, ref.sum_bound(mag, terms))
    got = ts.grouped_mm_dw(*dev(d_y, x, offsets), row_src=dev(src), out_dtype=BF16)
    within(got, y, ref.rounded(ref.sum_bound(mag, terms), y, BF16))


def test_dw_rows_outside_and_empty():
    """NaN in rows of no group reaches nothing; groups without rows get zeros."""
    rows, G, n, k = 200, 5, 72, 136
    x, _, offsets, _, g = product(rows, G, n, k, BF16, lead=9, tail=20)
    d_y = randn(g, rows, n, dtype=BF16)
    y, mag = ref.dw(d_y, x, offsets)
    for t in (x, d_y):
        t[:9], t[180:] = float("nan"), float("inf")
    got = ts.grouped_mm_dw(*dev(d_y, x, offsets))
    within(got, y, ref.sum_bound(mag, rows))
    none = ts.grouped_mm_dw(torch.empty(0, 64, device=DEV), torch.empty(0, 72, device=DEV),
                            torch.zeros(4, dtype=torch.int32, device=DEV))
    assert none.shape == (3, 64, 72) and bool((none == 0).all())


def test_non_finite_rows_stay_in_their_rows():
    x, w, offsets, _, g = product(300, 3, 136, 264, BF16)
    a = ts.grouped_mm(*dev(x, w, offsets))
    x[17], x[200, 3] = float("nan"), float("inf")
    b = ts.grouped_mm(*dev(x, w, offsets))
    keep = [r for r in range(300) if r not in (17, 200)]
    assert torch.equal(a[keep].view(torch.int16), b[keep].view(torch.int16))
    assert torch.isnan(b[17]).all() and not torch.isfinite(b[200]).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n", [(1, 8), (3, 1792), (130, 72)])
def test_drelu_grad(dtype, rows, n):
    g = gen(20, rows, n)
    gt, up, dc = (randn(g, rows, n, dtype=dtype) for _ in range(3))
    gt[0, 0], up[0, 1], gt[0, 2], up[0, 3] = 0.0, -0.0, float("nan"), float("nan")
    dg, du = ts.drelu_grad(*dev(gt, up, dc))
    on = (gt > 0) & (up > 0)
    z = torch.zeros(())
    assert torch.equal(dg.cpu(), torch.where(on, dc.float() * up.float(), z).to(dtype))
    assert torch.equal(du.cpu(), torch.where(on, dc.float() * gt.float(), z).to(dtype))


# --- fp8 -------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 128), (7, 144), (65, 1792), (300, 272)])
def test_fp8_quant(dtype, rows, cols):
    g = gen(30, rows, cols)
    x = randn(g, rows, cols, dtype=dtype) * torch.logspace(-3, 3, rows).to(dtype)[:, None]
    x[0, :16] = 0.0
    q, s = ts.fp8_quant(dev(x))
    rq, rs = ref.quant_rows(x)
    assert torch.equal(s.cpu(), rs)
    assert torch.equal(q.cpu().view(torch.uint8), rq.view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_fp8_quant_edges(dtype):
    """Zeros, tiny and huge blocks, infinities and NaN: the scale, the codes."""
    x = torch.zeros(9, 256, dtype=dtype)
    x[1, 3] = 2.0 ** -120
    x[2] = torch.linspace(-3e38, 3e38, 256).to(dtype)  # (6e38 is beyond fp32: infinities and NaN only)
    x[8] = (torch.linspace(-1, 1, 256) * 3e38).to(dtype)
    x[3, 5] = float("inf")
    x[4, 7], x[4, 8] = float("nan"), 3.0
    x[5] = torch.linspace(-1e30, 1e30, 256).to(dtype)
    x[6, 130] = 2.0 ** -100
    x[7] = torch.arange(256).to(dtype)
    q, s = ts.fp8_quant(dev(x))
    v, s = q.cpu().float(), s.cpu()
    assert bool((v[0] == 0).all()) and bool((s[0] == 2.0 ** -100 / 448).all())
    assert bool((v[1] == 0).all()) and v[6, 130] == 448
    assert not torch.isfinite(x[2]).any() and torch.isinf(s[2]).all() and torch.isnan(v[2]).all()
    for r in (5, 7, 8):
        val = ref.row_values(q.cpu()[r:r + 1], s[r:r + 1])[0]
        # half a step of e4m3 relative to the value, or of its smallest step
        big = x[r].double().abs().view(2, 128).amax(1).repeat_interleave(128)
        assert bool(((val - x[r].double()).abs() <= 2.0 ** -4 * (1 + 2.0 ** -20) * x[r].double().abs()
                     + 2.0 ** -10 * big / 448).all()), r
    assert torch.isinf(s[3, 0]) and torch.isnan(v[3, :128]).all() and bool((v[3, 128:] == 0).all())
    assert torch.isnan(v[4, 7]) and v[4, 8] == 448 and int(torch.isnan(v[4]).sum()) == 1


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w_kn", [False, True])
@pytest.mark.parametrize("G,n,k", [(1, 16, 16), (3, 272, 144), (2, 128, 384)])
def test_fp8_quant_weights(dtype, w_kn, G, n, k):
    w = randn(gen(31, G, n, k), G, n, k, dtype=dtype)
    q, s = ts.fp8_quant_weights(dev(w.transpose(1, 2).contiguous() if w_kn else w), w_kn=w_kn)
    rq, rs = ref.quant_tiles(w)
    assert torch.equal(s.cpu(), rs)
    assert torch.equal(q.cpu().view(torch.uint8), rq.view(torch.uint8))


FP8_SHAPES = [(1, 1, 16, 16), (2, 8, 144, 272), (5, 64, 64, 128), (40, 3, 208, 400), (150, 4, 48, 528),
              (300, 3, 400, 144), (700, 2, 272, 336), (513, 1, 528, 1040)]


def fp8_product(rows, G, n, k, seed=0):
    x, w, offsets, src, g = product(rows, G, n, k, BF16, gather=True, seed=seed)
    xq, xs = ref.quant_rows(x)
    wq, wsc = ref.quant_tiles(w)
    return (xq, xs, wq, wsc, offsets, src), *fp8_want(xq, xs, wq, wsc, offsets, src), g


def fp8_want(xq, xs, wq, wsc, offsets, src=None):
    """The product and its bound: the sum's (per block also the two scales'
    product and its use) and the matrix instructions' own."""
    x, w = ref.row_values(xq, xs), ref.tile_values(wq, wsc)
    y, mag = ref.mm(x, w, offsets, src)
    return y, ref.sum_bound(mag, x.shape[1] + 4) + ref.fp8_bound(x, w, offsets, src)


@pytest.mark.parametrize("rows,G,n,k", FP8_SHAPES)
def test_fp8_mm(rows, G, n, k):
    (xq, xs, wq, wsc, offsets, src), y, bound, _ = fp8_product(rows, G, n, k)
    got = ts.fp8_mm(*dev(xq, xs, wq, wsc, offsets), row_src=dev(src), out_dtype=F32)
    within(got, y, bound)
    got = ts.fp8_mm(*dev(xq, xs, wq, wsc, offsets), row_src=dev(src))
    within(got, y, ref.rounded(bound, y, BF16))


@pytest.mark.parametrize("rows,G,n,k", FP8_SHAPES)
def test_fp8_drelu(rows, G, n, k):
    (xq, xs, wq, wsc, offsets, src), gt, eg, g = fp8_product(rows, G, n, k)
    uq, us = ref.quant_tiles(randn(g, G, n, k, dtype=BF16, scale=k ** -0.5))
    up, eu = fp8_want(xq, xs, uq, us, offsets, src)
    c = ref.drelu(gt, up)
    bound = ref.drelu_bound(gt, up, eg, eu) + 2.0 ** -23 * c.abs()
    got = ts.fp8_drelu(*dev(xq, xs, wq, wsc, uq, us, offsets), row_src=dev(src))
    within(got, c, ref.rounded(bound, c, BF16))


def test_fp8_block_exponents():
    """Rows and tiles whose scales span many powers of two."""
    g = gen(33)
    x = randn(g, 70, 512) * 2.0 ** torch.randint(-30, 30, (70, 4), generator=g).float().repeat_interleave(128, 1)
    w = randn(g, 1, 256, 512) * 2.0 ** torch.randint(-30, 30, (1, 256, 4), generator=g).float().repeat_interleave(128, 2)
    q, s = ts.fp8_quant(dev(x))
    wq, wsc = ts.fp8_quant_weights(dev(w))
    y, bound = fp8_want(q.cpu(), s.cpu(), wq.cpu(), wsc.cpu(), torch.tensor([0, 70]))
    within(ts.fp8_mm(q, s, wq, wsc, out_dtype=F32), y, bound)


@pytest.mark.parametrize("k", ref.EIGHTS_K)
def test_fp8_many_scale_blocks(k):
    """Each block of 128 its own powers of two, rows and weights: a scale of
    another block would show."""
    rows, G, n = ref.EIGHTS
    g = gen(34, k)
    nb = -(-k // 128)
    blocks = lambda *s: 2.0 ** torch.randint(-6, 7, (*s, nb), generator=g).float().repeat_interleave(128, len(s))[..., :k]  # noqa: E731
    gd = torch.Generator(device=DEV).manual_seed(k)
    x = torch.randn(rows // 2, k, generator=gd, device=DEV) * dev(blocks(rows // 2))
    wg, wu = (torch.randn(G, n, k, generator=gd, device=DEV) * dev(blocks(G, 1)) * k ** -0.5 for _ in range(2))
    offsets = ref.ragged(rows, G, g, lead=2, tail=3)
    src = torch.randint(0, rows // 2, (rows,), generator=g, dtype=torch.int32)
    off, sd = dev(offsets, src)
    (xq, xs), qg, qu = ts.fp8_quant(x), ts.fp8_quant_weights(wg), ts.fp8_quant_weights(wu)
    (gt, eg), (up, eu) = (fp8_want(xq, xs, *q, offsets, sd) for q in (qg, qu))
    mid = slice(2, rows - 3)
    within(ts.fp8_mm(xq, xs, *qg, off, row_src=sd, out_dtype=F32)[mid], gt[mid], eg[mid])
    c = ref.drelu(gt, up)
    bound = ref.drelu_bound(gt, up, eg, eu) + 2.0 ** -23 * c.abs()
    got = ts.fp8_drelu(xq, xs, *qg, *qu, off, row_src=sd, out_dtype=F32)
    within(got[mid], c[mid], bound[mid])


def test_fp8_products_that_cancel():
    """Large products that cancel across groups of 8, small ones beside them: the
    error is the stated share of the groups' largest products, whatever is left
    of the result."""
    rows, n, k = 70, 144, 512
    g = gen(35)
    half = k // 2
    x, w = randn(g, rows, half), randn(g, 1, n, half)
    at = torch.randperm(half, generator=g) + half  # (where the products come again, with the other sign)
    xx, ww = torch.empty(rows, k), torch.empty(1, n, k)
    xx[:, :half], ww[:, :, :half] = x, w
    xx[:, at], ww[:, :, at] = x, -w
    small = torch.rand(k, generator=g) < 0.3
    xx[:, small] *= 2.0 ** -8
    (xq, xs), (wq, wsc) = ref.quant_rows(xx), ref.quant_tiles(ww)
    y, bound = fp8_want(xq, xs, wq, wsc, [0, rows])
    for odt in (F32, BF16):
        got = ts.fp8_mm(*dev(xq, xs, wq, wsc), out_dtype=odt)
        within(got, y, ref.rounded(bound, y, odt))


# --- combine ---------------------------------------------------------------------

@pytest.mark.parametrize("ydt,odt", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("T,K,H", [(1, 2, 8), (1, 8, 4096), (33, 2, 520), (700, 3, 264), (5, 1, 12)])
def test_combine_and_gradients(ydt, odt, T, K, H):
    if H % 8 and BF16 in (ydt, odt):
        H = 16
    g = gen(40, T, K, H)
    y, w, d_out = randn(g, T * K + 3, H, dtype=ydt), torch.softmax(randn(g, T, K), 1), randn(g, T, H, dtype=odt)
    pair_row = torch.randperm(T * K, generator=g).to(torch.int32).view(T, K)
    if T > 8:
        pair_row[3] = -1          # a token without rows
        pair_row[5, 0] = T * K + 3  # past the rows
    ok = (pair_row >= 0) & (pair_row < T * K + 3)
    rows = torch.where(ok[:, :, None], y.double()[pair_row.clamp(0, T * K + 2).long()], torch.zeros((), dtype=D))
    wd = w.double()[:, :, None]
    for ww, wt in ((w, wd), (None, torch.ones_like(wd))):
        want, mag = (wt * rows).sum(1), (wt * rows.abs()).sum(1)
        got = ts.moe_combine(*dev(y, pair_row), w=dev(ww), out_dtype=odt)
        within(got, want, ref.rounded(ref.sum_bound(mag, K), want, odt))
    d_y = torch.full((T * K + 3, H), 7.0, dtype=ydt, device=DEV)
    _, d_w = ts.moe_combine_grad(*dev(d_out, y, pair_row, w), d_y=d_y)
    want = torch.full((T * K + 3, H), 7.0, dtype=D)
    want[pair_row[ok].long()] = (wd * d_out.double()[:, None]).expand(T, K, H)[ok]
    within(d_y, want, ref.rounded(2.0 ** -24 * want.abs(), want, ydt))
    dd = d_out.double()[:, None]
    within(d_w, (dd * rows).sum(2), ref.sum_bound((dd.abs() * rows.abs()).sum(2), H))


# --- every tile, long offsets, bad maps ---------------------------------------------

def big(rows, G, n, k, kind, w_kn=False):
    """Inputs on the device (drawn there), ragged groups that leave rows out at
    both ends, gathered rows."""
    g = gen(70, rows, G, n, k)
    gd = torch.Generator(device=DEV).manual_seed(rows * 7 + n)
    offsets = ref.ragged(rows, G, g, lead=2, tail=3) if G > 1 else torch.tensor([2, rows - 3], dtype=torch.int32)
    src = torch.randint(0, rows // 2, (rows,), generator=g, dtype=torch.int32)
    dt = F32 if kind == "f32" else BF16
    x = torch.randn(rows // 2, k, generator=gd, device=DEV).to(dt)
    ws = [(torch.randn(G, *((k, n) if w_kn else (n, k)), generator=gd, device=DEV) * k ** -0.5).to(dt) for _ in range(2)]
    return x, ws, offsets, dev(src), dev(offsets)


@pytest.mark.parametrize("rows,G,n", ref.TILE_SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
def test_every_tile(rows, G, n, kind):
    k = ref.TILE_K[kind]
    x, (wg, wu), offsets, src, off = big(rows, G, n, k, kind)
    mid = slice(2, rows - 3)

    def same_rows(got, want, bound, dt):
        assert got.dtype == dt
        within(got[mid], want[mid], ref.rounded(bound, want, dt)[mid])
        untouched(got, mid, 7.0)
    out = lambda dt: torch.full((rows, n), 7.0, dtype=dt, device=DEV)  # noqa: E731
    if kind == "fp8":
        (xq, xs), qg, qu = ts.fp8_quant(x), ts.fp8_quant_weights(wg), ts.fp8_quant_weights(wu)
        (gt, eg), (up, eu) = (fp8_want(xq, xs, *q, offsets, src) for q in (qg, qu))
        same_rows(ts.fp8_mm(xq, xs, *qg, off, row_src=src, out=out(F32)), gt, eg, F32)
        c = ts.fp8_drelu(xq, xs, *qg, *qu, off, row_src=src, out=out(BF16))
    else:
        (gt, mg), (up, mu) = ref.mm(x, wg, offsets, src), ref.mm(x, wu, offsets, src)
        eg, eu = ref.sum_bound(mg, k), ref.sum_bound(mu, k)
        same_rows(ts.grouped_mm(x, wg, off, row_src=src, out=out(F32)), gt, eg, F32)
        same_rows(ts.grouped_mm(x, wg.transpose(1, 2).contiguous(), off, row_src=src, w_kn=True, out=out(BF16)), gt, eg,
                  BF16)
        x2 = torch.randn_like(x.float()).to(x.dtype)
        y2, m2 = ref.mm(x2, wu, offsets, src)
        same_rows(ts.grouped_mm(x, wg, off, row_src=src, x2=x2, w2=wu, out=out(F32)), gt + y2,
                  ref.sum_bound(mg + m2, 2 * k), F32)
        c = ts.grouped_drelu(x, wg, wu, off, row_src=src, out=out(F32))
    want = ref.drelu(gt, up)
    same_rows(c, want, ref.drelu_bound(gt, up, eg, eu) + 2.0 ** -23 * want.abs(), c.dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,G,n,k", [(700, 5, 2064, 1736), (300, 3, 2576, 2312)])
def test_dw_large_tiles(dtype, rows, G, n, k):
    x, _, offsets, src, off = big(rows, G, 8, k, "f32" if dtype is F32 else "bf16")
    d_y = torch.randn(rows, n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)).to(dtype)
    for s in (src, None):
        xx = x if s is not None else torch.cat([x, x, x[:rows % 2]])
        y, mag = ref.dw(d_y, xx, offsets, s)
        within(ts.grouped_mm_dw(d_y, xx, off, row_src=s), y, ref.sum_bound(mag, rows))


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
def test_rows_of_x_past_4_gb(kind):
    """x of more than 4 GB: gathered rows on both sides of that offset."""
    k, n, rows, G = 8192, 144, 90, 3
    esz = {"bf16": 2, "f32": 4, "fp8": 1}[kind]
    S = (1 << 32) // (k * esz) + 70
    g = gen(80)
    src = torch.cat([torch.randint(0, 50, (rows // 2,), generator=g),
                     S - 1 - torch.randint(0, 60, (rows - rows // 2,), generator=g)])
    src = src[torch.randperm(rows, generator=g)].to(torch.int32)
    offsets = ref.ragged(rows, G, g)
    dt = F32 if kind == "f32" else BF16
    few, back = src.long().unique(return_inverse=True)
    xf = randn(g, len(few), k, dtype=dt)
    w = randn(g, G, n, k, dtype=dt, scale=k ** -0.5)
    small = back.to(torch.int32)
    if kind == "fp8":
        q, s = ref.quant_rows(xf)
        x = torch.empty(S, k, dtype=torch.uint8, device=DEV)
        xs = torch.empty(S, k // 128, device=DEV)
        x[few.to(DEV)], xs[few.to(DEV)] = dev(q.view(torch.uint8)), dev(s)
        wq = ts.fp8_quant_weights(dev(w))
        for f, more in ((ts.fp8_mm, ()), (ts.fp8_drelu, wq)):
            a = f(x.view(torch.float8_e4m3fn), xs, *wq, *more, dev(offsets), row_src=dev(src), out_dtype=F32)
            b = f(dev(q), dev(s), *wq, *more, dev(offsets), row_src=dev(small), out_dtype=F32)
            assert (a - b).norm() <= 1e-5 * b.norm()  # (another tile: another order of the same sums)
        return
    x = torch.empty(S, k, dtype=dt, device=DEV)
    x[few.to(DEV)] = dev(xf)
    y, mag = ref.mm(xf, w, offsets, small)
    wd, od, sd = dev(w, offsets, src)
    within(ts.grouped_mm(x, wd, od, row_src=sd, out_dtype=F32), y, ref.sum_bound(mag, k))
    kn = wd.transpose(1, 2).contiguous()
    within(ts.grouped_mm(x, kn, od, row_src=sd, w_kn=True, out_dtype=F32), y, ref.sum_bound(mag, k))
    e = ref.sum_bound(mag, k)
    c = ref.drelu(y, y)
    within(ts.grouped_drelu(x, wd, wd, od, row_src=sd, out_dtype=F32), c,
           ref.drelu_bound(y, y, e, e) + 2.0 ** -23 * c.abs())
    d_y = randn(g, rows, n, dtype=dt)
    y, mag = ref.dw(d_y, xf, offsets, small)
    within(ts.grouped_mm_dw(dev(d_y), x, od, row_src=sd), y, ref.sum_bound(mag, rows))


@pytest.mark.parametrize("kind,n,k", [("bf16", 131072, 16368), ("f32", 131072, 8176), ("fp8", 131056, 32752)])
def test_operands_just_below_4_gb(kind, n, k):
    """The largest weight matrix, and as many rows of x: their offsets need all
    of 32 bits."""
    g = gen(83)
    dt = F32 if kind == "f32" else BF16
    cols = torch.tensor([0, 1, n // 2 - 1, n // 2, 3 * n // 4, n - 17, n - 1], device=DEV)
    src = cols.to(torch.int32)
    long = torch.randn(n, k, generator=torch.Generator(device=DEV).manual_seed(83), device=DEV, dtype=dt)
    few = randn(g, 5, k, dtype=dt)
    if kind == "fp8":
        lq, ls = ts.fp8_quant_weights(long[None])
        fq, fs = ts.fp8_quant(dev(few))
        lv, fv = ref.row_values(lq[0][cols], ls[0][cols // 128]).cpu(), ref.row_values(fq, fs).cpu()
        y, mag = ref.mm(fv, lv[None], [0, 5])
        bound = ref.sum_bound(mag, k + 4) + ref.fp8_bound(fv, lv[None], [0, 5])
        within(ts.fp8_mm(fq, fs, lq, ls, out_dtype=F32)[:, cols], y, bound)
        del lq, ls
        lq, ls = ts.fp8_quant(long)
        fq, fs = ts.fp8_quant_weights(torch.cat([few, few, few, few[:1]]).to(DEV)[None])
        lv, fv = ref.row_values(lq[cols], ls[cols]).cpu(), ref.tile_values(fq, fs).cpu()
        y, mag = ref.mm(lv, fv, [0, 7])
        bound = ref.sum_bound(mag, k + 4) + ref.fp8_bound(lv, fv, [0, 7])
        within(ts.fp8_mm(lq, ls, fq, fs, row_src=src, out_dtype=F32), y, bound)
        return
    lv, few = long[cols].cpu(), torch.cat([few, few[:3]])
    y, mag = ref.mm(few, lv[None], [0, 8])
    within(ts.grouped_mm(dev(few), long[None], out_dtype=F32)[:, cols], y, ref.sum_bound(mag, k))
    y, mag = ref.mm(lv, few[None], [0, 7])
    within(ts.grouped_mm(long, dev(few)[None], row_src=src, out_dtype=F32), y, ref.sum_bound(mag, k))
    d_y = randn(g, 7, 16, dtype=dt)
    y, mag = ref.dw(d_y, lv, [0, 7])
    within(ts.grouped_mm_dw(dev(d_y), long, row_src=src), y, ref.sum_bound(mag, 7))


def test_outputs_past_2_31_elements():
    rows, n, k = 140000, 16384, 8
    g = gen(81)
    x, w = randn(g, rows, k, dtype=BF16), randn(g, 1, n, k, dtype=BF16)
    out = ts.grouped_mm(*dev(x, w))
    for r in (0, 65535, 131071, 131072, 131073, rows - 1):
        want = x[r].double() @ w[0].double().t()
        mag = x[r].double().abs() @ w[0].double().abs().t()
        within(out[r], want, ref.rounded(ref.sum_bound(mag, k), want, BF16))
    gate = torch.ones_like(out)
    dg, du = ts.drelu_grad(gate, gate, out)
    assert torch.equal(dg[-1], out[-1]) and torch.equal(du[131073], out[131073])
    del dg, du, gate
    q, s = ts.fp8_quant(out)
    rq, rs = ref.quant_rows(out[-2:].cpu())
    assert torch.equal(q[-2:].cpu().view(torch.uint8), rq.view(torch.uint8)) and torch.equal(s[-2:].cpu(), rs)
    pair = torch.tensor([[rows - 1, 131073]], dtype=torch.int32, device=DEV)
    got = ts.moe_combine(out, pair, out_dtype=F32)
    assert torch.equal(got[0], out[rows - 1].float() + out[131073].float())


def test_maps_out_of_range_stay_in_bounds():
    """Offsets out of order or range, sources out of range: clamped as stated
    (rows that no clamped group holds stay)."""
    rows, G, n, k = 60, 5, 72, 136
    g = gen(82)
    x, w = randn(g, 20, k, dtype=BF16), randn(g, G, n, k, dtype=BF16)
    bad = torch.tensor([-7, 10, 4, 33, 1 << 30, 12], dtype=torch.int32)
    src = torch.randint(-40, 60, (rows,), generator=g, dtype=torch.int32)
    src[0], src[1] = -(1 << 31), (1 << 31) - 1
    good = bad.clamp(0, rows).cummax(0).values
    y, mag = ref.mm(x, w, good, src.clamp(0, 19))
    out = torch.full((rows, n), 7.0, device=DEV)
    ts.grouped_mm(*dev(x, w, bad), row_src=dev(src), out=out)
    within(out, y, ref.sum_bound(mag, k))
    d_y = randn(g, rows, n, dtype=BF16)
    y, mag = ref.dw(d_y, x, good, src.clamp(0, 19))
    within(ts.grouped_mm_dw(*dev(d_y, x, bad), row_src=dev(src)), y, ref.sum_bound(mag, rows))


# --- together ---------------------------------------------------------------------

def layer(x, wr, wg, wu, wd, K, out_dtype=None):
    """The MoE layer on the framework's operators, with what backward needs."""
    logits = ts.grouped_mm(x, wr[None], out_dtype=F32)
    idx, w, off, tok, pair = ts.moe_route(logits, K)
    c, gt, up = ts.grouped_drelu(x, wg, wu, off, row_src=tok, keep=True)
    y = ts.grouped_mm(c, wd, off, w_kn=True)
    return ts.moe_combine(y, pair, w, out_dtype=out_dtype), (idx, w, off, tok, pair, c, gt, up, y)


def backward(x, wr, wg, wu, wd, d_out, kept):
    idx, w, off, tok, pair, c, gt, up, y = kept
    d_y, d_w = ts.moe_combine_grad(d_out, y, pair, w)
    d_c = ts.grouped_mm(d_y, wd, off)
    d_wd = ts.grouped_mm_dw(c, d_y, off)
    dg, du = ts.drelu_grad(gt, up, d_c)
    d_wg = ts.grouped_mm_dw(dg, x, off, row_src=tok)
    d_wu = ts.grouped_mm_dw(du, x, off, row_src=tok)
    d_x = ts.moe_combine(ts.grouped_mm(dg, wg, off, x2=du, w2=wu, w_kn=True), pair, out_dtype=F32)
    d_l = ts.moe_route_grad(idx, w, d_w, wr.shape[0])
    d_x = d_x + ts.grouped_mm(d_l, wr[None].float(), w_kn=True)
    d_wr = ts.grouped_mm_dw(d_l, x.float())[0]
    return d_x, d_wr, d_wg, d_wu, d_wd


def layer64(x, wr, wg, wu, wd, idx):
    w = torch.softmax((x @ wr.t()).gather(1, idx), 1)
    out = torch.zeros_like(x)
    for k in range(idx.shape[1]):
        h = [torch.einsum("th,tih->ti", x, m[idx[:, k]]) for m in (wg, wu)]
        out = out + w[:, k:k + 1] * torch.einsum("ti,tih->th", h[0].relu() * h[1].relu(), wd[idx[:, k]])
    return out


@pytest.mark.parametrize("dtype,T", [(F32, 1), (F32, 50), (BF16, 1), (BF16, 130)])
def test_layer_forward_and_backward(dtype, T):
    """The layer as a model runs it, both passes, against 64-bit autograd; and
    its gradients against differences of the 64-bit layer."""
    E, K, H, I = 8, 2, 64, 136
    g = gen(50, T)
    x = randn(g, T, H, dtype=dtype)
    wr, wg, wu, wd = (randn(g, *s, dtype=dtype, scale=H ** -0.5) for s in ((E, H), (E, I, H), (E, I, H), (E, I, H)))
    d_out = randn(g, T, H, dtype=dtype)
    args = dev(x, wr, wg, wu, wd)
    out, kept = layer(*args, K)
    grads = backward(*args, dev(d_out), kept)
    leaves = [t.double().requires_grad_() for t in (x, wr, wg, wu, wd)]
    idx = kept[0].cpu().long()
    want = layer64(*leaves, idx)
    want.backward(d_out.double())
    # bf16: five stages round to 2^-8 each; fp32: sums of up to 200 terms.
    # (2-norms: a gate next to 0 may close on one side only)
    tol = 5 * 2.0 ** -8 if dtype == BF16 else 200 * 2.0 ** -24
    for got, ref_ in zip((out, *grads), (want.detach(), *(l.grad for l in leaves))):
        err = (got.cpu().double() - ref_).norm() / ref_.norm()
        assert err <= tol, (err, got.shape)
    # differences along a random direction of everything
    if dtype == F32 and T > 1:
        dirs = [torch.randn(l.shape, generator=g, dtype=D) for l in leaves]
        h = 1e-6
        f = lambda s: (layer64(*[l.detach() + s * d for l, d in zip(leaves, dirs)], idx) * d_out.double()).sum()  # noqa: E731
        diff = (f(h) - f(-h)) / (2 * h)
        got = sum((gr.cpu().double() * d).sum() for gr, d in zip(grads, dirs))
        mag = sum((gr.cpu().double() * d).abs().sum() for gr, d in zip(grads, dirs))
        assert abs(diff - got) <= 1e-5 * mag


def test_layer_fp8_forward():
    """The 8-bit layer: routing, quantised gate + up and down, combine."""
    T, E, K, H, I = 90, 8, 2, 256, 400
    g = gen(51)
    x = randn(g, T, H, dtype=BF16)
    wr, wg, wu, wd = (randn(g, *s, dtype=BF16, scale=H ** -0.5) for s in ((E, H), (E, I, H), (E, I, H), (E, I, H)))
    xd, wrd, wgd, wud, wdd = dev(x, wr, wg, wu, wd)
    qg, qu, qd = ts.fp8_quant_weights(wgd), ts.fp8_quant_weights(wud), ts.fp8_quant_weights(wdd, w_kn=True)
    idx, w, off, tok, pair = ts.moe_route(ts.grouped_mm(xd, wrd[None], out_dtype=F32), K)
    c = ts.fp8_drelu(*ts.fp8_quant(xd), *qg, *qu, off, row_src=tok)
    out = ts.moe_combine(ts.fp8_mm(*ts.fp8_quant(c), *qd, off), pair, w)
    want = layer64(*(t.double() for t in (x, wr, wg, wu, wd)), idx.cpu().long())
    # x, the three weights and Combined rounded to e4m3 (2^-4 each at most);
    # gate and up are both of the first two
    assert (out.cpu().double() - want).norm() / want.norm() <= 6 * 2.0 ** -4


@pytest.mark.parametrize("T,E,K,H,I", ref.FP8_LAYERS)
def test_layer_fp8_forward_from_its_codes(T, E, K, H, I):
    """The 8-bit layer, each element against the 64-bit layer on the same codes
    and scales: every block's scale, expert and weight in its place."""
    x, wr, wg, wu, wd = ref.fp8_layer_inputs(T, E, H, I, gen(52, T))
    xd, wrd, wgd, wud, wdd = dev(x, wr, wg, wu, wd)
    logits = ts.grouped_mm(xd, torch.nn.functional.pad(wrd, (0, 0, 0, -E % 8))[None], out_dtype=F32)[:, :E].contiguous()
    want = x.double() @ wr.double().t()
    within(logits, want, ref.sum_bound(x.double().abs() @ wr.double().abs().t(), H))
    qg, qu, qd = ts.fp8_quant_weights(wgd), ts.fp8_quant_weights(wud), ts.fp8_quant_weights(wdd, w_kn=True)
    idx, w, off, tok, pair = ts.moe_route(logits, K)
    c = ts.fp8_drelu(*ts.fp8_quant(xd), *qg, *qu, off, row_src=tok)
    out = ts.moe_combine(ts.fp8_mm(*ts.fp8_quant(c), *qd, off), pair, w)
    codes = [ref.quant_tiles(m) for m in (wg, wu, wd.transpose(1, 2))]
    comb, comb_bound, want, bound = ref.fp8_layer(x, *codes, logits.cpu(), K, c.cpu())
    within(c, comb, comb_bound)
    within(out, want, bound)


# --- streams, graphs, determinism ---------------------------------------------------

def everything(x, wr, wg, wu, wd, K, d_out):
    out, kept = layer(x, wr, wg, wu, wd, K)
    grads = backward(x, wr, wg, wu, wd, d_out, kept)
    q = ts.fp8_quant(x)
    c8 = ts.fp8_drelu(*q, *ts.fp8_quant_weights(wg), *ts.fp8_quant_weights(wu), kept[2], row_src=kept[3])
    return (out, c8, kept[0], kept[4], *grads)


def small_layer(T, seed):
    E, K, H, I = 8, 2, 128, 208
    g = gen(60, seed)
    ws = dev(*(randn(g, *s, dtype=BF16, scale=H ** -0.5) for s in ((E, H), (E, I, H), (E, I, H), (E, I, H))))
    return dev(randn(g, T, H, dtype=BF16)), ws, K, dev(randn(g, T, H, dtype=BF16))


def same(a, b):
    return all(torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8)) for p, q in zip(a, b))


def test_repeats_and_streams_give_the_same_bits():
    calls = [small_layer(T, s) for s, T in enumerate((1, 90, 700))]
    serial = [everything(x, *w, K, d) for x, w, K, d in calls]
    torch.cuda.synchronize()
    for (x, w, K, d), r in zip(calls, serial):
        assert same(everything(x, *w, K, d), r)
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for s, (x, w, K, d) in zip(streams, calls):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(everything(x, *w, K, d))
    torch.cuda.synchronize()
    for a, b in zip(got, serial):
        assert same(a, b)


def test_a_given_stream_owns_what_the_call_makes(monkeypatch):
    """Outputs and workspaces come from the memory of the stream that the call
    runs on: from the current stream's, blocks whose last readers still run there
    could be handed out, and a workspace handed on while the call runs."""
    x, (wr, wg, wu, wd), K, d = small_layer(1500, 3)  # (two launches and a workspace to route)

    def run(stream):
        kw = {} if stream is None else {"stream": stream}
        logits = ts.grouped_mm(x, wr[None], out_dtype=F32, **kw)
        idx, w, off, tok, pair = ts.moe_route(logits, K, **kw)
        off2, tok2, pair2 = ts.moe_group(idx, 8, **kw)
        c, gate, up = ts.grouped_drelu(x, wg, wu, off, row_src=tok, keep=True, **kw)
        y = ts.grouped_mm(c, wd, off, w_kn=True, **kw)
        out = ts.moe_combine(y, pair, w, **kw)
        d_y, d_w = ts.moe_combine_grad(d, y, pair, w, **kw)
        d_l = ts.moe_route_grad(idx, w, d_w, 8, **kw)
        d_g, d_u = ts.drelu_grad(gate, up, ts.grouped_mm(d_y, wd, off, **kw), **kw)
        d_wg = ts.grouped_mm_dw(d_g, x, off, row_src=tok, **kw)
        qx, qg = ts.fp8_quant(x, **kw), ts.fp8_quant_weights(wg, **kw)
        qu, qd = ts.fp8_quant_weights(wu, **kw), ts.fp8_quant_weights(wd, w_kn=True, **kw)
        c8 = ts.fp8_drelu(*qx, *qg, *qu, off, row_src=tok, **kw)
        y8 = ts.fp8_mm(*ts.fp8_quant(c8, **kw), *qd, off, **kw)
        return out, w, off2, tok2, pair2, d_y, d_l, d_u, d_wg, y8

    want = run(None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    made, empty = [], torch.empty

    def watched(*args, **kw):
        made.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", watched)
    got = run(s)
    monkeypatch.undo()
    s.synchronize()
    assert len(made) > 20 and all(m == s for m in made)
    assert same(got, want)


@pytest.mark.parametrize("T", [1, 600])
def test_graph_replays(T):
    """Forward and backward captured into one graph: replays with new inputs,
    eager work between them, equal eager calls bit for bit."""
    x, w, K, d = small_layer(T, 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        everything(x, *w, K, d)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(x, *w, K, d)
    for i in range(4):
        x.copy_(dev(randn(gen(61, i), *x.shape, dtype=BF16)))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        assert same(got, everything(x.clone(), *w, K, d)), i
        torch.cuda.synchronize()
