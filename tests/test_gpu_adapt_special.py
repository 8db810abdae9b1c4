"""Adapters of whole numbers, and of infinities and NaN among them: each value of the
result is the definition's, signs included, and other requests' rows keep theirs.
All finite values are small whole numbers (times powers of two), so that every sum is
exact in any order, a step that is left out or taken twice shows, and results are
compared for equality."""
import math
import random

import pytest
import torch

import adapt_util as ref
import group_util as gref
from adapt_util import BF16, F32
from gpu_util import DEV
from test_gpu_group import dev

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None

INF, NAN = float("inf"), float("nan")
N, BAD = 6, 2  # adapters, the broken one

# rows, segments, rank, n, k: a single row, one row a request, a split contraction (its
# last three), prompts, the large tiles (the last with more of t than LDS holds)
SHAPES = [(1, 1, 16, 264, 136), (40, 40, 16, 264, 136), (300, 7, 64, 264, 136), (2500, 40, 24, 1552, 136), (3000, 33, 128, 4112, 136),
          (1, 1, 8, 144, 4104), (33, 5, 24, 144, 4104), (300, 300, 40, 144, 4104)]


def whole(g, *shape, top=2, keep=1.0):
    v = torch.randint(-top, top + 1, shape, generator=g).float()
    return v * (torch.rand(shape, generator=g) < keep)


def inputs(rows, S, rank, n, k, products, seed):
    """x [rows][k], per product (w [n][k], a [N][rank][k], b [N][rank][n]), offsets,
    adapters, scales: whole numbers, products of x with a below 2^8 (so that t is exact
    in one bf16 part)."""
    g = torch.Generator().manual_seed(1000 * seed + rows + k)
    off, ad = ref.segments(rows, S, N, g)
    ad[::3] = BAD
    x = whole(g, rows, k)
    mats = [(whole(g, n, k), whole(g, N, rank, k, keep=min(1.0, 100 / k)), whole(g, N, rank, n)) for _ in range(products)]
    for _, a, _ in mats:
        assert float((x @ a.view(-1, k).t()).abs().max()) <= 256
    return x, mats, off, ad, torch.exp2(torch.randint(-1, 3, (N,), generator=g).float())


def break_b(b):
    """Infinities and NaN in [rank][n], one a column or two of one step's."""
    rank, n = b.shape
    j = torch.arange(n)
    for every, at, value in ((5, 0, INF), (5, 1, -INF), (13, 3, NAN)):
        c = j[j % every == at]
        b[c % rank, c] = value
    c = j[j % 11 == 2]
    b[0, c], b[1, c] = INF, -INF
    c = j[j % 17 == 4]
    b[rank - 1, c], b[0, c] = INF, INF


def projected(x, w, a, b, off, ad, scale):
    """x w^T + scale (x a^T) b, term by term in 64 bits."""
    x, y = x.double(), x.double() @ w.double().t()
    for s, p, q in gref.spans(off):
        i = int(ad[s])
        if q > p and 0 <= i < N:
            # (term by term: a library product may pad with zeros, and 0 x inf is NaN)
            t = (x[p:q, :, None].expand(-1, -1, 1) * 0).sum(1).expand(-1, a.shape[1]).clone()
            fin = torch.isfinite(a[i])
            t += x[p:q] @ torch.where(fin, a[i], 0.0).double().t()
            for r, c in (~fin).nonzero().tolist():
                t[:, r] += x[p:q, c] * float(a[i, r, c])
            t *= float(scale[i])
            for r in range(a.shape[1]):
                y[p:q] += t[:, r:r + 1] * b[i, r].double()
    return y


def equal(got, want):
    nan = torch.isnan(want)
    return torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


def compare(x, mats, off, ad, scale, dtype, odt):
    d = lambda t: t.to(DEV)  # noqa: E731
    o = dev(off, ad)
    ys = [projected(d(x), d(w), d(a), d(b), off, ad, scale) for w, a, b in mats]
    ops = [[t.to(dtype) for t in m] for m in mats]
    if len(mats) == 1:
        want = ys[0].to(odt)
        (w, a, b), = ops
        for kn in (False, True):
            wk, bk = (w.t().contiguous(), b) if kn else (w, b.transpose(1, 2).contiguous())
            got = ts.adapter_mm(*dev(x.to(dtype), wk, a, bk), *o, scale=dev(scale), w_kn=kn, out_dtype=odt)
            assert equal(got, want), kn
        return want
    # (projections exact in fp32, one rounding of their product; a NaN closes)
    want = gref.drelu(*[y.float() for y in ys]).to(odt)
    (wg, ag, bg), (wu, au, bu) = ops
    bg, bu = (b.transpose(1, 2).contiguous() for b in (bg, bu))
    got = ts.adapter_drelu(*dev(x.to(dtype), wg, wu, ag, bg, au, bu), *o, scale=dev(scale), out_dtype=odt)
    assert equal(got, want)
    return want


@pytest.mark.parametrize("dtype,odt", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,S,rank,n,k", SHAPES)
def test_infinities_and_nan_of_b(rows, S, rank, n, k, dtype, odt):
    if k > 4000:  # (the sums of two parts at least)
        assert ts.adapter_workspace_bytes(rows, rank, 1, False, n, k, dtype, odt) > 2 * rows * n * 4
    x, mats, off, ad, scale = inputs(rows, S, rank, n, k, 1, 1)
    break_b(mats[0][2][BAD])
    want = compare(x, mats, off, ad, scale, dtype, odt)
    assert all(bool(v.any()) for v in (want == INF, want == -INF, torch.isnan(want)))
    for broken in ((0,), (1,), (0, 1)):
        x, mats, off, ad, scale = inputs(rows, S, rank, n, k, 2, 2)
        for i in broken:
            break_b(mats[i][2][BAD])
        want = compare(x, mats, off, ad, scale, dtype, odt)
        assert bool((want == INF).any())


@pytest.mark.parametrize("dtype,odt", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,S,rank,n,k", SHAPES)
def test_infinite_t_beside_infinities_of_b(rows, S, rank, n, k, dtype, odt):
    """A's infinity makes t infinite at one rank; B has infinities, NaN and zeros
    there and at other ranks of the same step."""
    for broken in ((0,), (1,), (0, 1)):
        for products in (1, 2):
            if broken[-1] >= products:
                continue
            x, mats, off, ad, scale = inputs(rows, S, rank, n, k, products, 3)
            x[:, 5] = torch.where(torch.arange(rows) % 2 == 0, 1.0, -1.0)
            for i in broken:
                _, a, b = mats[i]
                a[BAD, 1, 5] = -INF
                break_b(b[BAD])
                b[BAD, 1, 8::23], b[BAD, 1, 9::23], b[BAD, 1, 10::23] = INF, NAN, 0.0
                b[BAD, 2, 8::46] = INF
            want = compare(x, mats, off, ad, scale, dtype, odt)
            assert bool((want == INF).any())


@pytest.mark.parametrize("rows,n,k", ref.TILES + ref.SPLITS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_step_counts_once(rows, n, k, dtype):
    """Every tile and split: each step of the contraction is in the sums, once (a bound
    of the sums' rounding is wider than a step's share where the contraction is long)."""
    g = torch.Generator(device=DEV).manual_seed(rows + n + k)
    r = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV, dtype=torch.int8)  # noqa: E731
    x = r(rows, k).to(dtype)
    for S, rank in ((rows, 16), (max(rows // 60, 1), 24)):
        off, ad = ref.segments(rows, S, N, torch.Generator().manual_seed(k))
        scale = torch.exp2(torch.randint(-1, 3, (N,), generator=torch.Generator().manual_seed(n)).float())
        # (few values of a, so that t is a whole number below 2^8)
        mats = [(r(n, k).to(dtype), (r(N, rank, k) * (torch.rand(N, rank, k, generator=g, device=DEV) < 100 / k)).to(dtype),
                 r(N, n, rank).to(dtype)) for _ in range(2)]
        for _, a, _ in mats:
            assert float((x.float() @ a.float().view(-1, k).t()).abs().max()) <= 256
        ys = [ref.adapted(x, *m, off, ad, scale, False, 0)[0] for m in mats]
        assert all(bool((y.abs() < 2 ** 22).all()) for y in ys)
        o = dev(off, ad)
        (w, a, b), (v, c, d) = mats
        for kn in (False, True):
            m = (w.t().contiguous(), a, b.transpose(1, 2).contiguous()) if kn else (w, a, b)
            assert torch.equal(ts.adapter_mm(x, *m, *o, scale=dev(scale), w_kn=kn, out_dtype=F32).double(), ys[0]), (S, kn)
        got = ts.adapter_drelu(x, w, v, a, b, c, d, *o, scale=dev(scale), out_dtype=F32)
        assert torch.equal(got, gref.drelu(*[y.float() for y in ys])), S


@pytest.mark.parametrize("odt", [BF16, F32])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,S,rank,n,k", SHAPES)
def test_the_ranks_values_keep_their_bits(rows, S, rank, n, k, dtype, odt):
    """t of 16 bits (bf16 output; differences of two that leave 8) and of 22 (fp32
    output): what the output can hold of them is exact."""
    g = torch.Generator().manual_seed(7 + rows + k)
    off, ad = ref.segments(rows, S, N, g)
    scale = torch.exp2(torch.randint(-1, 3, (N,), generator=g).float())
    top = 15 if odt == BF16 else 120
    x = whole(g, rows, k, top=top)
    mats, r = [], torch.arange(rank)
    for _ in range(2):
        a = whole(g, N, 1, k, top=top, keep=min(1.0, 136 / k)).repeat(1, rank, 1)
        a[:, r, r] += r % 4 + 1.0  # ranks differ in one place each
        b = torch.zeros(N, rank, n)
        j = torch.arange(n)
        b[:, j % rank, j] = 1
        if odt == BF16:
            b[:, (j + 1) % rank, j] = -1
        mats.append((torch.zeros(n, k), a, b))
        t = (x @ a.view(-1, k).t()).abs()
        assert float(t.max()) < (1 << 16 if odt == BF16 else 1 << 22)
        assert rows == 1 or float(t.max()) > (1 << 11 if odt == BF16 else 1 << 17)
    compare(x, mats[:1], off, ad, scale, dtype, odt)
    compare(x, mats, off, ad, scale, dtype, odt)


@pytest.mark.parametrize("dtype,odt", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rows", [1, 40])
def test_finite_t_above_the_largest_bf16(rows, dtype, odt):
    """t between the largest finite values of bf16 and of fp32 stays finite."""
    n, k, rank = 144, 136, 16
    x, mats, off, ad, _ = inputs(rows, rows, rank, n, k, 1, 5)
    w, a, b = (torch.zeros_like(t) for t in mats[0])
    x[:, 0], x[:, 1] = 255 * 2.0 ** 120, 2.0 ** 119 * (1 + 2.0 ** -7)
    ad[:] = BAD
    a[BAD, 3, :2], a[BAD, 7, :2] = 1, -1  # t = +-(2^128 - 2^119 + 2^112)
    b[BAD, 3, ::2], b[BAD, 7, 1::2] = 2.0 ** -20, 2.0 ** -2
    assert float(torch.tensor(float(x[0, 0]) + float(x[0, 1])).bfloat16()) == INF
    want = compare(x, [(w, a, b)], off, ad, torch.ones(N), dtype, odt)
    assert bool(torch.isfinite(want).all()) and bool((want.abs() > 2.0 ** 107).all())


@pytest.mark.parametrize("seed", range(8))
def test_random_shapes(seed):
    """Sizes over their ranges, types, layouts and broken values as they come."""
    rng = random.Random(seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    for i in range(12):
        dtype, odt, q = *rng.choice([(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)]), 8
        rows, rank, n, k = log(1, 3000), log(8, 128) // q * q, log(8, 4200) // q * q, log(8, 6000) // q * q
        S, products, what = rng.choice([min(rows, log(1, 300)), log(1, 100)]), rng.choice([1, 2]), rng.choice(["", "b", "t"])
        x, mats, off, ad, scale = inputs(rows, S, rank, n, k, products, 100 + 12 * seed + i)
        if what == "t":
            x[:, 5] = torch.where(torch.arange(rows) % 2 == 0, 1.0, -1.0)
            mats[0][1][BAD, 1, 5] = -INF
        if what:
            break_b(mats[-1][2][BAD])
        compare(x, mats, off, ad, scale, dtype, odt)
