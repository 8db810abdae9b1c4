"""Projections with adapters in 64 bits, and what the results may be off by
(results on the inputs' device)."""
import torch

import group_util as ref
from group_util import BF16, D, F32

# (rows, n) that take every tile at this contraction, for one product and for gate + up
TILE_K = 336
TILES = [(1, 144), (41, 4112), (41, 6160), (41, 8208), (300, 1552), (700, 1040), (100, 8208), (300, 8208), (700, 6160),
         (1000, 2064), (2500, 1552), (2500, 6160), (700, 8208), (1000, 6160), (1000, 8208), (2000, 4112)]


def segments(rows, S, N, gen, lead=0, tail=0):
    """Ascending offsets over [lead, rows - tail) (one row each where rows == S,
    else ragged with empty ones), adapters of the segments, some without one."""
    m = rows - lead - tail
    if m == S:
        off = torch.arange(S + 1)
    else:
        cuts = (torch.rand(S - 1, generator=gen) ** 2 * (m + 1)).long().clamp(max=m)
        if S > 3:
            cuts[1] = cuts[0]
        off = torch.cat([torch.zeros(1, dtype=torch.int64), cuts.sort().values, torch.tensor([m])])
    ad = torch.randint(0, N, (S,), generator=gen, dtype=torch.int32)
    none = torch.rand(S, generator=gen)
    ad[none < 0.1] = -1
    ad[none > 0.95] = N
    if S == 1:
        ad[0] = N - 1
    return (off + lead).to(torch.int32), ad


def adapted(x, w, a, b, offsets, adapter, scale, w_kn, parts):
    """(y, bound): fp32 sums of the product and of the ranks' values, t, which are
    scaled (one rounding) and rounded to `parts` bf16 parts (0: kept in fp32)."""
    x, w, a, b = x.double(), w.double(), a.double(), b.double()
    R, k = x.shape
    w = w if w_kn else w.t()
    b = b if w_kn else b.transpose(1, 2)
    y, mag = x @ w, x.abs() @ w.abs()
    extra = torch.zeros_like(y)
    N, rank = a.shape[:2]
    for s, p, q in ref.spans(offsets):
        i = int(adapter[s])
        if q <= p or not 0 <= i < N:
            continue
        f = float(scale[i]) if scale is not None else 1.0
        t = f * (x[p:q] @ a[i].t())
        e = abs(f) * ref.sum_bound(x[p:q].abs() @ a[i].abs().t(), k) + 2.0 ** -24 * t.abs()
        if parts:
            e = e + ref.half_step(BF16) ** parts * (t.abs() + e)
        y[p:q] += t @ b[i]
        mag[p:q] += (t.abs() + e) @ b[i].abs()
        extra[p:q] = e @ b[i].abs()
    return y, extra + ref.sum_bound(mag, k + 2 * rank)


def case(rows, S, N, rank, n, k, dtype, w_kn, g, products=1, lead=0, tail=0, scaled=True):
    off, ad = segments(rows, S, N, g, lead, tail)
    x = torch.randn(rows, k, generator=g).to(dtype)
    scale = torch.rand(N, generator=g) + 0.5 if scaled else None
    mats = []
    for _ in range(products):
        w = torch.randn(*((k, n) if w_kn else (n, k)), generator=g) * k ** -0.5
        a = torch.randn(N, rank, k, generator=g) * k ** -0.5
        b = torch.randn(N, *((rank, n) if w_kn else (n, rank)), generator=g) * rank ** -0.5
        mats.append([m.to(dtype) for m in (w, a, b)])
    return x, mats, off, ad, scale
