"""Low-rank adapters of many requests beside a shared projection, and in front of
dReLU, against 64 bits."""
import pytest
import torch

import adapt_util as ref
import group_util as gref
from adapt_util import BF16, F32
from gpu_util import DEV
from test_gpu_group import dev, gen, randn, within

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None

# rows, segments, adapters, rank, n, k
CASES = [(1, 1, 1, 8, 8, 8), (1, 1, 3, 16, 264, 1032), (7, 7, 2, 8, 136, 72), (32, 32, 64, 16, 392, 520),
         (40, 3, 5, 24, 200, 264), (70, 64, 2, 128, 512, 136), (97, 97, 200, 32, 24, 520), (150, 9, 4, 64, 272, 8),
         (260, 2, 1, 16, 520, 200), (300, 300, 7, 40, 392, 136), (1100, 5000, 9, 8, 128, 104), (530, 17, 6, 104, 272, 328)]


def parts_of(dtype, odt):
    return 0 if dtype == F32 else 2 if odt == F32 else 1


def check(x, mats, off, ad, scale, w_kn, odt, out=None):
    parts = parts_of(x.dtype, odt)
    o = dev(off, ad)
    p, q = int(off[0]), int(off[-1])
    ys = [ref.adapted(*dev(x, w, a, b), off, ad, scale, w_kn, parts) for w, a, b in mats]
    if len(mats) == 1:
        (w, a, b), (want, bound) = mats[0], ys[0]
        got = ts.adapter_mm(*dev(x, w, a, b), *o, scale=dev(scale), w_kn=w_kn, out=out, out_dtype=odt)
    else:
        (w, a, b), (v, c, d) = mats
        (g, eg), (u, eu) = ys
        got = ts.adapter_drelu(*dev(x, w, v, a, b, c, d), *o, scale=dev(scale), out=out, out_dtype=odt)
        want, bound = gref.drelu(g, u), gref.drelu_bound(g, u, eg, eu)
        bound = bound + 2.0 ** -23 * (want + bound)
    assert got.dtype == odt
    within(got[p:q], want[p:q], gref.rounded(bound, want, odt)[p:q])
    return got


@pytest.mark.parametrize("rows,S,N,rank,n,k", CASES + [(33, 5, 3, 4, 20, 12), (9, 9, 4, 12, 36, 516)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w_kn", [False, True])
def test_mm(rows, S, N, rank, n, k, dtype, w_kn):
    if dtype == BF16 and (rank % 8 or n % 8 or k % 8):
        pytest.skip("bf16 sizes come in eights")
    g = gen(80, rows, S, N, rank, n, k)
    for odt, scaled in ((dtype, True), (F32 if dtype == BF16 else BF16, False)):
        check(*ref.case(rows, S, N, rank, n, k, dtype, w_kn, g, scaled=scaled), w_kn, odt)


@pytest.mark.parametrize("rows,S,N,rank,n,k", CASES + [(33, 5, 3, 4, 20, 12), (9, 9, 4, 12, 36, 516)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_drelu(rows, S, N, rank, n, k, dtype):
    if dtype == BF16 and (rank % 8 or n % 8 or k % 8):
        pytest.skip("bf16 sizes come in eights")
    g = gen(81, rows, S, N, rank, n, k)
    for odt, scaled in ((dtype, True), (F32 if dtype == BF16 else BF16, False)):
        check(*ref.case(rows, S, N, rank, n, k, dtype, False, g, products=2, scaled=scaled), False, odt)


@pytest.mark.parametrize("rows,n,k", ref.TILES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_tile(rows, n, k, dtype):
    """Every tile, with a segment a row and with ragged ones."""
    g = torch.Generator(device=DEV).manual_seed(82)
    for S, rank in ((rows, 16), (max(rows // 60, 1), 24)):
        for w_kn in (False, True):
            check(*ref.case(rows, S, 9, rank, n, k, dtype, w_kn, g), w_kn, dtype)
        check(*ref.case(rows, S, 9, rank, n, k, dtype, False, g, products=2), False, dtype)


@pytest.mark.parametrize("products", [1, 2])
def test_no_segment_has_an_adapter(products):
    """Then it is the projection, bit for bit."""
    g = gen(83)
    x, mats, off, ad, scale = ref.case(90, 8, 3, 16, 264, 136, BF16, False, g, products)
    ad[:] = -1
    got = check(x, mats, off, ad, scale, False, BF16)
    ws = dev(*[m[0][None] for m in mats]) if products == 2 else [dev(mats[0][0][None])]
    want = ts.grouped_mm(dev(x), *ws) if products == 1 else ts.grouped_drelu(dev(x), *ws)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,lead,tail", [(50, 3, 7), (700, 130, 41), (64, 64, 0), (300, 0, 299)])
def test_rows_outside_the_segments_stay(dtype, rows, lead, tail):
    for products in (1, 2):
        x, mats, off, ad, scale = ref.case(rows, 4, 3, 16, 136, 72, dtype, False, gen(84, rows), products, lead, tail)
        x[:lead], x[rows - tail:] = float("nan"), float("inf")
        out = torch.full((rows, 136), 7.0, device=DEV)
        xx = x.clone()
        xx[:lead], xx[rows - tail:] = 0, 0
        got = check(xx, mats, off, ad, scale, False, F32)
        o = dev(off, ad)
        if products == 1:
            ts.adapter_mm(*dev(x, *mats[0]), *o, scale=dev(scale), out=out)
        else:
            (w, a, b), (v, c, d) = mats
            ts.adapter_drelu(*dev(x, w, v, a, b, c, d), *o, scale=dev(scale), out=out)
        assert torch.equal(out[lead:rows - tail], got[lead:rows - tail])
        rest = torch.ones(rows, dtype=torch.bool)
        rest[lead:rows - tail] = False
        assert bool((out.cpu()[rest] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,rank", [(40, 8), (40, 16), (300, 64), (2500, 24)])
def test_broken_adapters_reach_their_own_rows_only(dtype, rows, rank):
    """Infinities and NaN in one adapter's matrices, and in one request's x."""
    n, k, N = 1552 if rows == 2500 else 264, 136, 6
    for w_kn in (False, True):
        x, mats, off, ad, scale = ref.case(rows, min(rows, 40), N, rank, n, k, dtype, w_kn, gen(85, rows, rank))
        w, a, b = mats[0]
        ad[::3] = 2
        o = dev(off, ad)
        want = ts.adapter_mm(*dev(x, w, a, b), *o, scale=dev(scale), w_kn=w_kn)
        row = torch.repeat_interleave(ad, (off[1:] - off[:-1]).long())
        mine = (row == 2).to(DEV)
        for where in ("b", "a"):
            a2, b2 = a.clone(), b.clone()
            if where == "b":
                b2.view(N, -1)[2, ::7] = float("inf")
                b2.view(N, -1)[2, 3::11] = float("nan")
            else:
                a2[2, 1, 5] = float("inf")
            got = ts.adapter_mm(*dev(x, w, a2, b2), *o, scale=dev(scale), w_kn=w_kn)
            assert torch.equal(got[~mine], want[~mine])
            y = ref.adapted(*dev(x, w, a2, b2), off, ad, scale, w_kn, 0)[0]
            clean = torch.isfinite(y) & mine[:, None]
            assert bool((~torch.isfinite(got[~torch.isfinite(y)])).all())
            assert torch.equal(got[clean], want[clean])
        x2 = x.clone()
        x2[0] = float("nan")
        got = ts.adapter_mm(*dev(x2, w, a, b), *o, scale=dev(scale), w_kn=w_kn)
        assert torch.equal(got[1:], want[1:]) and not bool(torch.isfinite(got[0]).any())


def test_offsets_out_of_order_stay_in_bounds():
    """Which rows are computed is unspecified; nothing outside is written."""
    x, mats, off, ad, scale = ref.case(60, 6, 3, 16, 136, 72, BF16, False, gen(86))
    room = torch.full((62, 136), 7.0, device=DEV, dtype=BF16)
    for bad in ([0, 50, 20, 70, -5, 30, 60], [60, 50, 40, 30, 20, 10, 0], [-9, -8, -7, 99, 99, 99, 2 ** 31 - 1]):
        o = torch.tensor(bad, dtype=torch.int32)
        ts.adapter_mm(*dev(x, *mats[0], o, ad), out=room[1:61])
        assert bool((room[0] == 7).all() and (room[61] == 7).all())


def test_nothing_to_do():
    x, mats, off, ad, scale = ref.case(6, 2, 3, 16, 136, 72, BF16, False, gen(87))
    w, a, b = mats[0]
    out = torch.full((6, 136), 7.0, device=DEV, dtype=BF16)
    ts.adapter_mm(*dev(x, w, a, b), dev(off[:1]), dev(ad[:0]), out=out)
    assert bool((out == 7).all())
    assert ts.adapter_mm(dev(x[:0]), *dev(w, a, b, off * 0, ad)).shape == (0, 136)


def test_many_segments_and_a_far_piece():
    """More segments than two rounds of 64 probes tell apart, most of them empty."""
    S, rows = 70001, 900
    g = gen(88)
    off = torch.sort(torch.randint(0, rows + 1, (S + 1,), generator=g)).values.to(torch.int32)
    off[0], off[-1] = 0, rows
    x, mats, _, _, scale = ref.case(rows, 3, 8, 16, 136, 72, BF16, False, g)
    ad = torch.randint(-1, 9, (S,), generator=g, dtype=torch.int32)
    check(x, mats, off, ad, scale, False, BF16)
