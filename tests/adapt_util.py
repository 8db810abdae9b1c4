"""Projections with adapters in 64 bits, and what the results may be off by
(results on the inputs' device)."""
import torch

import group_util as ref
from group_util import BF16, D, F32

# (rows, n, k) that between them take every tile of both types and modes, with the
# contraction in one workgroup and shared by several
TILES = [(1, 144, 136), (1, 144, 2056), (1500, 528, 136), (1500, 1040, 136), (1, 144, 4104), (200, 144, 4104),
         (1500, 4112, 136), (2500, 144, 136), (300, 144, 4104), (130, 528, 4104), (1000, 8208, 136), (200, 528, 4104),
         (700, 2064, 4104), (200, 1040, 4104), (700, 4112, 4104), (700, 1040, 4104), (1000, 1040, 4104), (500, 2064, 8192),
         (500, 4112, 8192), (1700, 528, 28672), (1700, 1040, 28672)]

# ... and every tile with every split that a grid of sizes chooses for it
SPLITS = [(1, 8, 136), (1, 8, 2056), (1, 8, 8200), (33, 14336, 136), (1500, 8, 4104), (1500, 1040, 136), (33, 2064, 4104),
          (1, 2064, 8200), (700, 144, 8200), (1500, 4112, 136), (1, 2064, 2056), (700, 8, 8200), (1, 8, 4104), (3000, 8, 4104),
          (2000, 4112, 136), (200, 1040, 14344), (700, 528, 136), (1, 1040, 28672), (130, 528, 14344), (700, 2064, 8200),
          (6000, 8, 8200), (33, 8208, 14344), (700, 1040, 8200), (1, 4112, 4104), (300, 1040, 28672), (1, 8208, 14344),
          (130, 264, 14344), (2000, 144, 4104), (1000, 144, 8200), (700, 4112, 8200), (33, 4112, 8200),
          (500, 4112, 14344), (1000, 144, 14344), (1000, 1040, 28672), (1000, 528, 57352), (200, 4112, 8200), (200, 1040, 57352)]


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
    of_row = torch.full((R,), -1, dtype=torch.int64)
    for s, p, q in ref.spans(offsets):
        of_row[p:q] = int(adapter[s])
    for i in range(N):
        at = (of_row == i).nonzero()[:, 0].to(x.device)
        if not at.numel():
            continue
        f = float(scale[i]) if scale is not None else 1.0
        t = f * (x[at] @ a[i].t())
        e = abs(f) * ref.sum_bound(x[at].abs() @ a[i].abs().t(), k) + 2.0 ** -24 * t.abs()
        if parts:
            e = e + ref.half_step(BF16) ** parts * (t.abs() + e)
        y[at] += t @ b[i]
        mag[at] += (t.abs() + e) @ b[i].abs()
        extra[at] = e @ b[i].abs()
    return y, extra + ref.sum_bound(mag, k + 2 * rank)


def case(rows, S, N, rank, n, k, dtype, w_kn, g, products=1, lead=0, tail=0, scaled=True):
    """x, the products' (w, a, b), offsets, adapters, scales; matrices on g's device."""
    off, ad = segments(rows, S, N, torch.Generator().manual_seed(g.initial_seed() % 2 ** 31 + products), lead, tail)

    def draw(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=g.device) * scale).to(dtype)
    x = draw(rows, k)
    scale = torch.rand(N, generator=g, device=g.device).cpu() + 0.5 if scaled else None
    mats = [(draw(*((k, n) if w_kn else (n, k)), scale=k ** -0.5), draw(N, rank, k, scale=k ** -0.5),
             draw(N, *((rank, n) if w_kn else (n, rank)), scale=rank ** -0.5)) for _ in range(products)]
    return x, mats, off, ad, scale
