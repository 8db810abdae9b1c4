"""dReLU's activations kept in 8 bits and the backward product that reads them,
against 64-bit forms of the same inputs; codes bit for bit."""
import pytest
import torch

import group_util as gref
import keep_util as ref
from group_util import BF16, D, F32
from gpu_util import DEV
from test_gpu_group import dev, gen, randn, within

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None

# rows, groups, n, k: one row; blocks of 16 that end inside (n 8, 136, 520; fp32 also 4)
SHAPES = [(1, 1, 8, 8), (2, 8, 136, 72), (40, 3, 200, 264), (97, 4, 512, 8), (260, 4, 392, 136), (530, 3, 272, 328)]


def inputs(rows, G, n, k, dtype, gather, seed, lead=0, tail=0):
    g = gen(60, rows, G, n, k, seed)
    off = gref.ragged(rows, G, g, lead, tail)
    S = max(rows // 2, 1) if gather else rows
    src = torch.randint(0, S, (rows,), generator=g, dtype=torch.int32) if gather else None
    x = randn(g, S, k, dtype=dtype)
    wg, wu = (randn(g, G, n, k, dtype=dtype, scale=k ** -0.5) for _ in range(2))
    return g, off, src, x, wg, wu


def check_pack(x, wg, wu, off, src, odt):
    args = dev(x, wg, wu, off)
    c, codes, exps = ts.grouped_drelu_pack(*args, row_src=dev(src), out_dtype=odt)
    # the same products in the same order, in fp32
    c32, g32, u32 = ts.grouped_drelu(*args, row_src=dev(src), keep=True, out_dtype=F32)
    a, b = int(off[0]), int(off[-1])
    wc, we = ref.pack2(g32[a:b].cpu(), u32[a:b].cpu())
    assert torch.equal(codes[a:b].cpu(), wc) and torch.equal(exps[a:b].cpu(), we)
    assert torch.equal(c[a:b], c32[a:b].to(odt))
    gate, up = ts.drelu_unpack(codes, exps)
    assert gate.dtype == BF16
    for got, want in zip((gate, up), ref.values2(wc, we)):
        assert torch.equal(got[a:b].cpu().double(), want)
    # and against 64 bits: half a step of 5 significant bits, the block's floor
    for got, w in ((gate, wg), (up, wu)):
        y, mag = gref.mm(dev(x), dev(w), off, dev(src))
        y, e = y[a:b], gref.sum_bound(mag, x.shape[1])[a:b]
        want = y.clamp(min=0)
        big = torch.nn.functional.pad(want + e, (0, -y.shape[1] % 16)).view(y.shape[0], -1, 16).amax(2)
        floor = big.repeat_interleave(16, 1)[:, :y.shape[1]] * 2.0 ** -15 * 17 / 16
        within(got[a:b], want, e + 2.0 ** -5 * (want + e) + floor)
        assert bool(((got[a:b] > 0) == (y > 0))[y.abs() > e].all())
    return codes, exps


@pytest.mark.parametrize("rows,G,n,k", SHAPES + [(33, 2, 20, 12)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pack(rows, G, n, k, dtype):
    if dtype == BF16 and n % 8:
        pytest.skip("bf16 columns come in eights")
    for gather, odt in ((False, dtype), (True, F32 if dtype == BF16 else BF16)):
        _, off, src, x, wg, wu = inputs(rows, G, n, k, dtype, gather, 0)
        check_pack(x, wg, wu, off, src, odt)


@pytest.mark.parametrize("rows,G,n", gref.TILE_SHAPES)
def test_pack_and_grad_every_tile(rows, G, n):
    for dtype in (BF16, F32):
        g, off, src, x, wg, wu = inputs(rows, G, n, gref.TILE_K["bf16"], dtype, False, 1)
        codes, exps = check_pack(x, wg, wu, off, src, dtype)
        check_grad(x, wg, codes, exps, off, None, dtype)


def check_grad(d_y, w, codes, exps, off, src, odt):
    dg, du, c = ts.grouped_drelu_grad(*dev(d_y, w), codes, exps, dev(off), row_src=dev(src), out_dtype=odt)
    dg2, du2 = ts.grouped_drelu_grad(*dev(d_y, w), codes, exps, dev(off), row_src=dev(src), out_dtype=odt, want_c=False)
    a, b = int(off[0]), int(off[-1])
    y, mag = gref.mm(dev(d_y), dev(w), off, dev(src))
    e = gref.sum_bound(mag, d_y.shape[1])
    g, u = (v.to(DEV) for v in ref.values2(codes.cpu(), exps.cpu()))
    on = ((g > 0) & (u > 0)).double()
    for got, again, f in ((dg, dg2, u * on), (du, du2, g * on)):
        want = y * f
        # the product with the fp32 value is rounded once more
        bound = e * f + 2.0 ** -23 * (want.abs() + e * f)
        within(got[a:b], want[a:b], gref.rounded(bound, want, odt)[a:b])
        assert torch.equal(got[a:b], again[a:b])
        assert bool((got[a:b][on[a:b] == 0] == 0).all())
    # two values of 5 significant bits: exact in fp32
    assert torch.equal(c[a:b], (g * u)[a:b].float().to(odt))


@pytest.mark.parametrize("rows,G,n,k", SHAPES + [(33, 2, 20, 12)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_grad(rows, G, n, k, dtype):
    if dtype == BF16 and n % 8:
        pytest.skip("bf16 columns come in eights")
    for gather, odt in ((False, dtype), (True, F32 if dtype == BF16 else BF16)):
        g, off, src, d_y, w, _ = inputs(rows, G, n, k, dtype, gather, 2)
        codes, exps = dev(*ref.pack2(randn(g, rows, n), randn(g, rows, n)))
        check_grad(d_y, w, codes, exps, off, src, odt)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,lead,tail", [(50, 3, 7), (700, 130, 41), (64, 64, 0), (300, 0, 299)])
def test_rows_outside_the_groups_stay(dtype, rows, lead, tail):
    g, off, src, x, wg, wu = inputs(rows, 4, 136, 72, dtype, False, 3, lead, tail)
    x[:lead], x[rows - tail:] = float("nan"), float("inf")
    out = torch.full((rows, 136), 7.0, device=DEV)
    codes = torch.full((rows, 136, 2), 9, dtype=torch.uint8, device=DEV)
    exps = torch.full((rows, 9, 2), 9, dtype=torch.uint8, device=DEV)
    ts.grouped_drelu_pack(*dev(x, wg, wu, off), out=out, codes=codes, exps=exps)
    rest = torch.ones(rows, dtype=torch.bool)
    rest[lead:rows - tail] = False
    assert bool((out.cpu()[rest] == 7).all() and (codes.cpu()[rest] == 9).all() and (exps.cpu()[rest] == 9).all())


def as_gate(v, dtype=F32):
    """x, w with x w^T = v in every one of 3 rows: v's elements are the weights."""
    w = torch.zeros(1, v.numel(), 8)
    w[0, :, 0] = v
    x = torch.zeros(3, 8)
    x[:, 0] = 1
    return x.to(dtype), w.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pack_edges(dtype):
    """Infinities, NaN, halves, the largest finite, both zeros, beside each other
    and alone in their blocks of 16 (fp32's subnormals are left to the unpacking:
    the matrix cores may take them as zeros)."""
    v = torch.tensor([e for e in ref.EDGES if not 0 < abs(e) < 2.0 ** -126] + [1.0] * 8)
    v = v[:v.numel() // 8 * 8].to(dtype).float()
    v = torch.cat([v, *(torch.nn.functional.pad(e.view(1), (0, 15)) for e in v)])
    x, w = as_gate(v, dtype)
    u = torch.rand(v.numel(), generator=gen(61)).to(dtype).float()
    _, wu = as_gate(u, dtype)
    _, codes, exps = ts.grouped_drelu_pack(*dev(x, w, wu))
    wc, we = ref.pack2(v.expand(3, -1), u.expand(3, -1))
    assert torch.equal(codes.cpu(), wc) and torch.equal(exps.cpu(), we)


@pytest.mark.parametrize("n", [4, 8, 20, 24, 136])
def test_unpack_every_code(n):
    """Every code next to every exponent byte that a block can have."""
    e = torch.arange(15, 256, dtype=torch.uint8)
    rows = 256
    q = (torch.arange(rows * n).view(rows, n) * 7 % 256).to(torch.uint8)
    for lo in range(0, 241, 48):
        ex = e[(torch.arange(rows * ((n + 15) // 16)).view(rows, -1) % 48 + lo).clamp(max=240)]
        full = ex.repeat_interleave(16, 1)[:, :n]
        qq = torch.where((full == 255) & (q > 240), torch.full_like(q, 240), q)
        codes, exps = torch.stack([qq, qq.flip(0)], 2), torch.stack([ex, ex.flip(0)], 2)
        gate, up = ts.drelu_unpack(*dev(codes.contiguous(), exps.contiguous()))
        for got, want in zip((gate, up), ref.values2(codes, exps)):
            assert torch.equal(got.cpu().double(), want)


def test_no_rows():
    x, w = torch.empty(0, 64, device=DEV), torch.zeros(4, 32, 64, device=DEV)
    off = torch.zeros(5, dtype=torch.int32, device=DEV)
    c, codes, exps = ts.grouped_drelu_pack(x, w, w, off)
    assert c.shape == (0, 32) and codes.shape == (0, 32, 2) and exps.shape == (0, 2, 2)
    assert ts.drelu_unpack(codes, exps)[0].shape == (0, 32)
    assert ts.grouped_drelu_grad(x, w, codes, exps, off)[2].shape == (0, 32)
