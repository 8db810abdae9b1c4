"""Adapters at the limits of what a call may hold: offsets that descend, more
workgroups than one launch takes."""
import pytest
import torch

import adapt_util as ref
from adapt_util import BF16, F32
from gpu_util import DEV
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
