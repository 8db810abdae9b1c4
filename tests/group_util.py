"""Plain 64-bit forms of the grouped operators, and what their results may be
off by (results on the inputs' device)."""
import torch

F32, BF16, D = torch.float32, torch.bfloat16, torch.float64
E4M3 = torch.float8_e4m3fn


def half_step(dtype):
    """Largest relative error of one rounding to `dtype`."""
    return torch.finfo(dtype).eps / 2


def spans(offsets):
    return [(g, int(a), int(b)) for g, (a, b) in enumerate(zip(offsets[:-1], offsets[1:]))]


def ragged(rows, groups, gen, lead=0, tail=0):
    """Ascending offsets over rows [lead, rows - tail), some groups empty."""
    n = rows - lead - tail
    cuts = torch.randint(0, n + 1, (groups - 1,), generator=gen)
    if groups > 3:
        cuts[1] = cuts[0]  # an empty group
    o = torch.cat([torch.zeros(1, dtype=torch.int64), cuts.sort().values, torch.tensor([n])])
    return (o + lead).to(torch.int32)


# (rows, groups, n) that between them take every tile of every kind and mode at
# these contractions: several whole blocks (the stages' rings wrap) and a partial one
TILE_SHAPES = [(41, 1, 144), (41, 1, 6160), (41, 1, 8208), (41, 5, 4112), (41, 5, 8208), (100, 5, 6160), (300, 5, 4112),
               (300, 5, 6160), (300, 5, 8208), (700, 5, 4112), (700, 5, 6160), (700, 5, 8208), (1000, 1, 2064),
               (2500, 1, 1552), (4000, 1, 144), (300, 5, 2064), (700, 5, 2064), (2300, 1, 1552)]
TILE_K = {"bf16": 336, "f32": 336, "fp8": 720}
# the fp8 tile that fetches the rows' scales of 8 blocks at a time: 9 to 23 blocks
EIGHTS = (1500, 3, 8208)
EIGHTS_K = (1152, 1168, 2176, 2832)


def mm(x, w, offsets, row_src=None, w_kn=False):
    """(y, sum of |products|) in 64 bits; NaN where no group has the row."""
    x = x.double() if row_src is None else x.double()[row_src.long()]
    w = w.double() if w_kn else w.double().transpose(1, 2)
    y = torch.full((x.shape[0], w.shape[2]), float("nan"), dtype=D, device=x.device)
    mag = y.clone()
    for g, a, b in spans(offsets):
        y[a:b] = x[a:b] @ w[g]
        mag[a:b] = x[a:b].abs() @ w[g].abs()
    return y, mag


def dw(d_y, x, offsets, row_src=None):
    x = x.double() if row_src is None else x.double()[row_src.long()]
    d_y = d_y.double()
    G = len(offsets) - 1
    y = torch.zeros(G, d_y.shape[1], x.shape[1], dtype=D, device=x.device)
    mag = y.clone()
    for g, a, b in spans(offsets):
        y[g] = d_y[a:b].t() @ x[a:b]
        mag[g] = d_y[a:b].abs().t() @ x[a:b].abs()
    return y, mag


def sum_bound(mag, terms):
    """An fp32 sum of `terms` exact products in any order, each addition off by
    at most a whole step (the matrix cores may cut instead of round)."""
    return (terms + 2) * 2.0 ** -23 * mag


def fp8_bound(x, w, offsets, row_src=None):
    """What the fp8 matrix instructions leave out: they add products in groups
    of 8 consecutive contraction indices, aligned to the group's largest
    exponent, and cut what lies below 2^-13 of it (a power of two 2^-13 of the
    largest is kept, 2^-14 is lost).  So each of the 7 others is off by less
    than 2^-13 of the group's largest product."""
    x = x.double() if row_src is None else x.double()[row_src.long()]
    w, x = w.double().abs(), x.abs()
    out = torch.zeros(x.shape[0], w.shape[1], dtype=D, device=x.device)
    for g, a, b in spans(offsets):
        for k in range(0, x.shape[1], 8):
            top = torch.zeros(b - a, w.shape[1], dtype=D, device=x.device)
            for i in range(k, k + 8):
                top = torch.maximum(top, x[a:b, i, None] * w[g, None, :, i])
            out[a:b] += 7 * 2.0 ** -13 * top
    return out


def drelu(g, u):
    return torch.where((g > 0) & (u > 0), g * u, torch.zeros_like(g))


def drelu_bound(g, u, eg, eu):
    return g.abs() * eu + u.abs() * eg + eg * eu


def rounded(bound, y, dtype):
    """The bound with one rounding to dtype behind it (and its smallest values)."""
    return bound + half_step(dtype) * (y.abs() + bound) + 2.0 ** -126


def quant_rows(x):
    """Codes (as values) and scales of blocks of 128 along rows."""
    R, C = x.shape
    nb = -(-C // 128)
    p = torch.nn.functional.pad(x.float(), (0, nb * 128 - C)).view(R, nb, 128)
    amax = p.abs().amax(2).clamp(min=2.0 ** -100)
    q = (p * 448.0 / amax[:, :, None]).to(E4M3)
    return q.view(R, nb * 128)[:, :C].contiguous(), amax / 448.0


def quant_tiles(w):
    G, n, k = w.shape
    nb, kb = -(-n // 128), -(-k // 128)
    p = torch.nn.functional.pad(w.float(), (0, kb * 128 - k, 0, nb * 128 - n)).view(G, nb, 128, kb, 128)
    amax = p.abs().amax(dim=(2, 4)).clamp(min=2.0 ** -100)
    q = (p * 448.0 / amax[:, :, None, :, None]).to(E4M3).view(G, nb * 128, kb * 128)
    return q[:, :n, :k].contiguous(), amax / 448.0


def row_values(q, s):
    return q.float().double() * s.double().repeat_interleave(128, 1)[:, :q.shape[1]]


def tile_values(q, s):
    G, n, k = q.shape
    return q.float().double() * s.double().repeat_interleave(128, 1)[:, :n].repeat_interleave(128, 2)[:, :, :k]


def route(logits, K):
    """idx, w, offsets, row_token, pair_row by sorting, in 64 bits."""
    T, E = logits.shape
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -float("inf")), logits).double()
    val, idx = torch.sort(l, dim=1, descending=True, stable=True)
    val, idx = val[:, :K], idx[:, :K]
    m = val[:, :1]
    e = torch.where(val == m, torch.ones_like(val), torch.exp(val - m))
    e = torch.where(m == -float("inf"), torch.zeros_like(e), e)
    s = e.sum(1, keepdim=True)
    w = torch.where(s > 0, e / s, torch.zeros_like(e))
    return idx.to(torch.int32), w, *group(idx, E)


def group(idx, E):
    T, K = idx.shape
    flat = idx.reshape(-1).long()
    ok = (flat >= 0) & (flat < E)
    order = torch.sort(torch.where(ok, flat, torch.full_like(flat, E)), stable=True).indices
    n = int(ok.sum())
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    for e in range(E):
        offsets[e + 1] = offsets[e] + int((flat == e).sum())
    pair_row = torch.full((T * K,), -1, dtype=torch.int32)
    pair_row[order[:n]] = torch.arange(n, dtype=torch.int32)
    return offsets, (order[:n] // K).to(torch.int32), pair_row.view(T, K)


def fp8_layer(x, gate, up, down, logits, K, c):
    """The 8-bit layer from its own codes: Combined and the output in 64 bits and
    what bf16 results may be off by.  gate, up, down: (codes, scales) of the
    weights, [E][n][k] each; c: the Combined that the down product was given."""
    idx, w, off, tok, pair = route(logits, K)

    def product(v, q, src=None):
        wv = tile_values(*q)
        y, mag = mm(v, wv, off, src)
        # (a block's two scales are multiplied first, and the sum by them)
        return y, sum_bound(mag, v.shape[1] + 4) + fp8_bound(v, wv, off, src)

    xv = row_values(*quant_rows(x))
    (g, eg), (u, eu) = product(xv, gate, tok), product(xv, up, tok)
    comb = drelu(g, u)
    comb_bound = rounded(drelu_bound(g, u, eg, eu) + 2.0 ** -23 * comb, comb, BF16)
    y, ey = product(row_values(*quant_rows(c)), down)
    ey = rounded(ey, y, BF16)
    # weights: exp of a difference rounded once, K of them added, one quotient
    ew = (12 + K + float(logits.abs().max())) * 2.0 ** -23
    y, ey, w = y[pair.long()], ey[pair.long()], w[:, :, None]
    out, mag = (w * y).sum(1), (w * (y.abs() + ey)).sum(1)
    bound = (w * ey).sum(1) + ew * (y.abs() + ey).sum(1) + sum_bound(mag, K)
    return comb, comb_bound, out, rounded(bound, out, BF16)


# tokens, experts, top k, hidden, inter: two and four blocks of 128, one of them partial
FP8_LAYERS = [(1, 4, 2, 144, 272), (90, 8, 2, 256, 400), (700, 4, 3, 400, 256)]


def fp8_layer_inputs(T, E, H, I, gen):
    """x, router, gate, up, down_t as the layer's weights are laid out."""
    x = torch.randn(T, H, generator=gen).to(BF16)
    return x, *((torch.randn(*s, generator=gen) * H ** -0.5).to(BF16)
                for s in ((E, H), (E, I, H), (E, I, H), (E, I, H)))
