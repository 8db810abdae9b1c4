"""Adapters at the limits of what a call may hold: offsets that descend, more
workgroups than one launch takes."""
import pytest
import torch

import adapt_util as ref
import group_util as gref
from adapt_util import BF16, F32
from gpu_util import DEV
from test_gpu_adapt import check
from test_gpu_group import dev, gen, randn, within

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None


def descending(off, how):
    off = off.clone()
    S = len(off) - 1
    if how == "front":
        off[0] = off[1] + 1
    elif how == "last":
        off[S] = off[S - 1] - 1
    elif how == "swapped":
        off[S // 2], off[S // 2 + 1] = off[S // 2 + 1].clone() + 3, off[S // 2].clone()
    else:
        off = off[torch.randperm(S + 1, generator=torch.Generator().manual_seed(S))]
        off[0], off[S] = 2, off.max()
        off[1] = off.max() + 1
    return off


@pytest.mark.parametrize("how", ["front", "last", "swapped", "shuffled"])
@pytest.mark.parametrize("rows,S", [(200, 6), (200, 64), (200, 65), (300, 5000), (2500, 40), (2500, 100)])
def test_descending_offsets_leave_no_adapter(rows, S, how):
    """The projections alone, bit for bit, whatever the workspace held."""
    n, k, rank, N = 136, 72, 16, 3
    x, mats, off, ad, scale = ref.case(rows, S, N, rank, n, k, BF16, False, gen(110, rows, S), 2)
    off = descending(off, how)
    b, e = max(int(off[0]), 0), min(int(off[-1]), rows)
    inside = off.clamp(0, rows)
    assert b < e and bool((inside[1:] < inside[:-1]).any())
    (w, a, bm), (v, c, d) = [dev(*m) for m in mats]
    x, o, ad, scale = dev(x, off, ad, scale)
    plain, none = dev(torch.tensor([b, e], dtype=torch.int32), torch.tensor([-1], dtype=torch.int32))

    def run(offsets, adapter, fill):
        ws = torch.full((1 << 24,), fill, dtype=torch.uint8, device=DEV)
        outs = [torch.full((rows, n), 7.0, device=DEV, dtype=BF16) for _ in range(2)]
        ts.adapter_mm(x, w, a, bm, offsets, adapter, scale=scale, out=outs[0], ws=ws)
        ts.adapter_drelu(x, w, v, a, bm, c, d, offsets, adapter, scale=scale, out=outs[1], ws=ws)
        return outs
    want = run(plain, none, 0)
    for fill in (0, 0x3F, 0xFF):
        for g, t in zip(run(o, ad, fill), want):
            assert torch.equal(g, t)


# rows, segments, rank, products, dtype: more workgroups of the ranks' values than a launch
# takes (2^32 threads), by rows and ranks and by segments
@pytest.mark.parametrize("rows,S,rank,products,dtype", [(270000, 270000, 128, 2, BF16), (530001, 530001, 128, 1, F32),
                                                        (3, 1 << 23, 8, 1, BF16)])
def test_more_workgroups_than_a_launch_takes(rows, S, rank, products, dtype):
    n, k, N = 16, 8, 5
    g = gen(111, rows)
    d = lambda *s: randn(g, *s, dtype=dtype, scale=0.5)  # noqa: E731
    x, mats = d(rows, k), [(d(n, k), d(N, rank, k), d(N, n, rank)) for _ in range(products)]
    if S == rows:
        off = torch.arange(S + 1, dtype=torch.int32)
    else:
        off = torch.full((S + 1,), rows, dtype=torch.int32)
        off[0], off[1:S // 2], off[S // 2:S - 1] = 0, 1, 2  # rows of segments 0, S / 2 - 1, S - 2
    ad = torch.randint(0, N, (S,), generator=g, dtype=torch.int32)
    o = dev(off, ad)
    (w, a, b), (v, c, e) = mats[0], mats[-1]
    if products == 1:
        got = ts.adapter_mm(*dev(x, w, a, b), *o, out_dtype=F32)
    else:
        got = ts.adapter_drelu(*dev(x, w, v, a, b, c, e), *o, out_dtype=F32)
    parts = 2 if dtype == BF16 else 0
    if S == rows:
        at = torch.cat([torch.randint(0, rows, (200,), generator=g), torch.tensor([0, rows - 1]),
                        torch.arange(rows // 2 - 20, rows // 2 + 20), torch.arange(262100, 262200)])
        own = ad[at]
    else:
        at, own = torch.arange(3), ad[torch.tensor([0, S // 2 - 1, S - 2])]
    ys = [ref.adapted(x[at], *m, torch.arange(len(at) + 1), own, None, False, parts) for m in mats]
    want, bound = ys[0]
    if products == 2:
        (p, ep), (q, eq) = ys
        want, bound = gref.drelu(p, q), gref.drelu_bound(p, q, ep, eq)
        bound = bound + 2.0 ** -23 * (want + bound)
    within(got[at.to(DEV)], want, bound)


# rows, segments, rank: the ranks' values by workgroups of 16 x 16, 32 x 64 and (bf16) 64
# x 64 rows x ranks, on both sides of the sizes where one gives way to the next
@pytest.mark.parametrize("rows,S,rank,products,shape", [
    (2500, 40, 48, 1, 0), (1365, 1, 48, 2, 0), (1366, 1, 48, 2, 1), (9001, 30, 16, 1, 0), (9001, 30, 24, 1, 1),
    (3001, 370, 128, 1, 1), (3001, 380, 128, 1, 0), (4095, 40, 128, 1, 1), (4097, 40, 128, 1, 2), (4097, 130, 128, 1, 1),
    (2500, 7, 120, 2, 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_shape_of_the_ranks_workgroups(rows, S, rank, products, shape, dtype):
    each = rows * rank * products
    small = rank * products <= 16 or each < 1 << 17 or rows < 8 * S
    assert shape == (0 if small else 2 if each >= 1 << 19 and rows >= 32 * S else 1)
    n, k, N = 40, 1144, 6
    g = torch.Generator(device=DEV).manual_seed(rows + rank)
    x, mats, off, ad, scale = ref.case(rows, S, N, rank, n, k, dtype, False, g, products, lead=3, tail=2)
    check(x, mats, off, ad, scale, False, F32)
    check(x, mats, off, ad, scale, False, dtype)
