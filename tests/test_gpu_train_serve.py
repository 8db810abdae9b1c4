"""The layer's training step with its balance loss and 8-bit activations, and the
feed-forward layer with adapters, as they run together: each stage against 64 bits
on what it was given, gradients against differences, streams, graphs, the largest
sizes."""
import pytest
import torch

import adapt_util as aref
import balance_util as bref
import group_util as gref
import keep_util as kref
from group_util import BF16, D, F32
from gpu_util import DEV
from test_gpu_group import dev, gen, randn, same, within

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None


def step(x, logits, wg, wu, wd, K, d_out, d_loss, mask=None, kw={}):
    """One training step of the MoE layer; its intermediate results."""
    E = wg.shape[0]
    r = {}
    r["idx"], r["w"], r["off"], r["tok"], r["pair"] = ts.moe_route(logits, K, **kw)
    r["loss"], r["counts"] = ts.moe_balance(logits, r["idx"], mask=mask, **kw)
    r["c"], r["codes"], r["exps"] = ts.grouped_drelu_pack(x, wg, wu, r["off"], row_src=r["tok"], **kw)
    r["y"] = ts.grouped_mm(r["c"], wd, r["off"], w_kn=True, **kw)
    r["out"] = ts.moe_combine(r["y"], r["pair"], r["w"], **kw)
    # backward: Combined comes out of the codes again
    r["d_y"], r["d_w"] = ts.moe_combine_grad(d_out, r["y"], r["pair"], r["w"], **kw)
    route = ts.moe_route_grad(r["idx"], r["w"], r["d_w"], E, **kw)
    r["d_route"] = route.clone()
    r["d_logits"] = ts.moe_balance_grad(logits, r["counts"], d_loss, K, mask=mask, add=route, out=route, **kw)
    r["d_gate"], r["d_up"], r["c2"] = ts.grouped_drelu_grad(r["d_y"], wd, r["codes"], r["exps"], r["off"], **kw)
    r["d_wd"] = ts.grouped_mm_dw(r["c2"], r["d_y"], r["off"], **kw)
    r["d_wg"] = ts.grouped_mm_dw(r["d_gate"], x, r["off"], row_src=r["tok"], **kw)
    r["d_wu"] = ts.grouped_mm_dw(r["d_up"], x, r["off"], row_src=r["tok"], **kw)
    r["d_x"] = ts.moe_combine(ts.grouped_mm(r["d_gate"], wg, r["off"], x2=r["d_up"], w2=wu, w_kn=True, **kw), r["pair"], **kw)
    r["gate"], r["up"] = ts.drelu_unpack(r["codes"], r["exps"], **kw)
    return r


def inputs(T, E, K, H, I, dtype, seed):
    g = gen(90, T, seed)
    x, d_out = randn(g, T, H, dtype=dtype), randn(g, T, H, dtype=dtype)
    wg, wu, wd = (randn(g, E, I, H, dtype=dtype, scale=H ** -0.5) for _ in range(3))
    return x, randn(g, T, E), wg, wu, wd, K, d_out, torch.tensor([0.5, -0.1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 70, 900])
def test_training_step(dtype, T):
    E, K, H, I = 8, 2, 136, 264
    x, logits, wg, wu, wd, K, d_out, d_loss = inputs(T, E, K, H, I, dtype, 0)
    mask = torch.arange(T) % 7 != 5
    r = step(*dev(x, logits, wg, wu, wd), K, *dev(d_out, d_loss), mask=dev(mask))
    r = {k: v.cpu() for k, v in r.items()}
    off, tok, pair = r["off"], r["tok"], r["pair"].long()
    want, wc, bound = bref.balance(logits, r["idx"], mask)
    assert torch.equal(r["counts"], wc)
    within(r["loss"], want, bound)
    want, bound = bref.balance_grad(logits, wc, d_loss, K, mask, r["d_route"])
    within(r["d_logits"], want, bound)
    # forward
    (g, mg), (u, mu) = (gref.mm(x, w, off, tok) for w in (wg, wu))
    eg, eu = gref.sum_bound(mg, H), gref.sum_bound(mu, H)
    c = gref.drelu(g, u)
    within(r["c"], c, gref.rounded(gref.drelu_bound(g, u, eg, eu) + 2.0 ** -23 * c, c, dtype))
    y, mag = gref.mm(r["c"], wd, off, w_kn=True)
    within(r["y"], y, gref.rounded(gref.sum_bound(mag, I), y, dtype))
    # backward, from the codes
    gk, uk = kref.values2(r["codes"], r["exps"])
    assert torch.equal(r["gate"].double(), gk) and torch.equal(r["up"].double(), uk)
    on = ((gk > 0) & (uk > 0)).double()
    d, mag = gref.mm(r["d_y"], wd, off)
    e = gref.sum_bound(mag, H)
    for name, f in (("d_gate", uk * on), ("d_up", gk * on)):
        within(r[name], d * f, gref.rounded(e * f + 2.0 ** -23 * (d * f).abs() + 2.0 ** -23 * e * f, d * f, dtype))
    assert torch.equal(r["c2"], (gk * uk * on).float().to(dtype))
    for name, a, b, src in (("d_wd", r["c2"], r["d_y"], None), ("d_wg", r["d_gate"], x, tok), ("d_wu", r["d_up"], x, tok)):
        want, mag = gref.dw(a, b, off, src)
        within(r[name], want, gref.sum_bound(mag, 2 * T))
    # how far the gradients are from those of the activations themselves: 5
    # significant bits of the other factor (and its block's floor), where gate and up are
    # clear of 0
    clear = (g.abs() > eg) & (u.abs() > eu)
    for name, f, ef in (("d_gate", u, eu), ("d_up", g, eg)):
        want = torch.where((g > 0) & (u > 0), d * f, torch.zeros_like(d))
        top = torch.nn.functional.pad(f.clamp(min=0) + ef, (0, -I % 16)).view(len(f), -1, 16).amax(2)
        floor = top.repeat_interleave(16, 1)[:, :I] * 2.0 ** -15 * 17 / 16
        off_by = (d.abs() + e) * (2.0 ** -5 * (f.abs() + ef) + ef + floor) + e * f.abs()
        bound = gref.rounded(off_by + 2.0 ** -22 * want.abs(), want, dtype)
        assert bool(((r[name].double() - want).abs() <= bound)[clear].all())


def test_gradient_of_activations_that_the_codes_hold_exactly():
    """gate and up of 5 significant bits: the gradient is the layer's own, against
    differences of the 64-bit layer."""
    g = gen(91)
    R, n, k = 40, 48, 24
    grid = lambda *s: (16 + torch.randint(0, 16, s, generator=g)) / 16.0 * torch.exp2(torch.randint(-3, 4, s, generator=g).float())  # noqa: E731
    sign = lambda *s: torch.randint(0, 2, s, generator=g).float() * 2 - 1  # noqa: E731
    gate, up = grid(R, n) * sign(R, n), grid(R, n) * sign(R, n)
    d_y, w = randn(g, R, k), randn(g, 1, n, k)
    codes, exps = kref.pack2(gate, up)
    dg, du, c = ts.grouped_drelu_grad(*dev(d_y, w, codes, exps))
    loss = lambda a, b: (gref.drelu(a, b) @ w[0].double() * d_y.double()).sum()  # noqa: E731
    assert torch.equal(c.cpu().double(), gref.drelu(gate.double(), up.double()))
    h = 2.0 ** -20
    for got, which in ((dg, 0), (du, 1)):
        d = torch.randn(R, n, generator=g, dtype=D)
        pair = [gate.double(), up.double()]
        moved = [[p + s * h * d if i == which else p for i, p in enumerate(pair)] for s in (1, -1)]
        diff = (loss(*moved[0]) - loss(*moved[1])) / (2 * h)
        prod = got.cpu().double() * d
        # (linear in each: no second order; differences to 2^-52 of the loss / h)
        mag = (gref.drelu(gate.double(), up.double()) @ w[0].double().abs() * d_y.double().abs()).sum()
        assert abs(diff - prod.sum()) <= 1e-6 * prod.abs().sum() + 2.0 ** -50 * mag / h


def ffn(x, off, ad, scale, g, u, d, kw={}):
    """The feed-forward layer with adapters at all three projections."""
    c = ts.adapter_drelu(x, g[0], u[0], g[1], g[2], u[1], u[2], off, ad, scale=scale, **kw)
    return c, ts.adapter_mm(c, *d, off, ad, scale=scale, w_kn=True, **kw)


def ffn_inputs(rows, S, H, I, rank, dtype, seed):
    g = gen(92, rows, seed)
    x, (gm, um), off, ad, scale = aref.case(rows, S, 6, rank, I, H, dtype, False, g, products=2)
    _, (dm,), *_ = aref.case(rows, S, 6, rank, H, I, dtype, True, g)
    return x, off, ad, scale, gm, um, dm


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,S", [(1, 1), (32, 32), (700, 11)])
def test_layer_with_adapters(dtype, rows, S):
    H, I, rank = 136, 264, 16
    x, off, ad, scale, gm, um, dm = ffn_inputs(rows, S, H, I, rank, dtype, 0)
    c, y = ffn(*dev(x, off, ad, scale), *[dev(*m) for m in (gm, um, dm)])
    parts = 1 if dtype == BF16 else 0
    (g, eg), (u, eu) = (aref.adapted(x, *m, off, ad, scale, False, parts) for m in (gm, um))
    want, bound = gref.drelu(g, u), gref.drelu_bound(g, u, eg, eu)
    within(c, want, gref.rounded(bound + 2.0 ** -23 * (want + bound), want, dtype))
    want, bound = aref.adapted(c.cpu(), *dm, off, ad, scale, True, parts)
    within(y, want, gref.rounded(bound, want, dtype))


def test_adapters_are_trained_as_groups():
    """Rows sorted by adapter: the groups of grouped_mm and grouped_mm_dw give the
    gradients of what adapter_mm computes, against 64-bit autograd."""
    g = gen(100)
    rows, N, rank, n, k = 150, 4, 8, 136, 72
    off = gref.ragged(rows, N, g)
    x, w = randn(g, rows, k), randn(g, n, k, scale=k ** -0.5)
    a, b, d_y = randn(g, N, rank, k, scale=k ** -0.5), randn(g, N, n, rank), randn(g, rows, n)
    xd, wd, ad, bd, dd, od = dev(x, w, a, b, d_y, off)
    y = ts.adapter_mm(xd, wd, ad, bd, od, torch.arange(N, dtype=torch.int32, device=DEV))
    t = ts.grouped_mm(xd, ad, od)
    d_t = ts.grouped_mm(dd, bd, od, w_kn=True)
    d_a, d_b = ts.grouped_mm_dw(d_t, xd, od), ts.grouped_mm_dw(dd, t, od)
    d_x = ts.grouped_mm(dd, wd[None], w_kn=True) + ts.grouped_mm(d_t, ad, od, w_kn=True)
    leaves = [v.double().requires_grad_() for v in (x, a, b)]
    want = torch.cat([leaves[0][p:q] @ w.double().t() + leaves[0][p:q] @ leaves[1][i].t() @ leaves[2][i].t()
                      for i, p, q in gref.spans(off)])
    want.backward(d_y.double())
    # two products in a row, sums of up to 150 terms each
    for got, ref_ in zip((y, d_x, d_a, d_b), (want.detach(), *(v.grad for v in leaves))):
        assert (got.cpu().double() - ref_).norm() <= 2 * 152 * 2.0 ** -23 * ref_.norm()


# --- streams, graphs, workspaces ------------------------------------------------------

def flat(r):
    return [r[k] for k in sorted(r) if k != "d_route"]


def both(args, fargs, kw={}, mask=None):
    x, off, ad, scale, gm, um, dm = fargs
    x2, logits, wg, wu, wd, K, d_out, d_loss = args
    return [*flat(step(x2, logits, wg, wu, wd, K, d_out, d_loss, mask, kw)), *ffn(x, off, ad, scale, gm, um, dm, kw)]


def calls(T, seed):
    x, logits, wg, wu, wd, K, d_out, d_loss = inputs(T, 8, 2, 128, 272, BF16, seed)
    f = ffn_inputs(T, min(T, 9), 128, 2064, 16, BF16, seed)
    return (*dev(x, logits, wg, wu, wd), K, *dev(d_out, d_loss)), (*dev(*f[:4]), *[dev(*m) for m in f[4:]])


def test_repeats_and_streams_give_the_same_bits():
    sets = [calls(T, s) for s, T in enumerate((1, 90, 3000))]
    serial = [both(*c) for c in sets]
    torch.cuda.synchronize()
    for c, r in zip(sets, serial):
        assert same(both(*c), r)
    streams, got = [torch.cuda.Stream() for _ in sets], []
    for s, c in zip(streams, sets):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(both(*c))
    torch.cuda.synchronize()
    for a, b in zip(got, serial):
        assert same(a, b)


def test_a_given_stream_owns_what_the_call_makes(monkeypatch):
    c = calls(3000, 3)
    want = both(*c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    made, empty = [], torch.empty

    def watched(*args, **kw):
        made.append(torch.cuda.current_stream())
        return empty(*args, **kw)
    monkeypatch.setattr(torch, "empty", watched)
    got = both(*c, kw={"stream": s})
    monkeypatch.undo()
    s.synchronize()
    assert len(made) > 20 and all(m == s for m in made)
    assert same(got, want)


@pytest.mark.parametrize("T", [1, 3000])
def test_graph_replays(T):
    """Captured into one graph: replays with new inputs, eager work between them,
    equal eager calls bit for bit."""
    args, fargs = calls(T, 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(args, fargs)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(args, fargs)
    for i in range(4):
        args[0].copy_(dev(randn(gen(93, i), *args[0].shape, dtype=BF16)))
        args[1].copy_(dev(randn(gen(94, i), *args[1].shape)))
        fargs[0].copy_(dev(randn(gen(95, i), *fargs[0].shape, dtype=BF16)))
        fargs[2].copy_(fargs[2].roll(1))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        assert same(got, both((args[0].clone(), *args[1:]), fargs)), i
        torch.cuda.synchronize()


def test_two_graphs_on_one_workspace():
    """Workspaces hold nothing from one call to the next: graphs that share one,
    replayed in turn, and one of garbage."""
    l = dev(randn(gen(96), 5000, 64))
    idx = l.topk(4).indices.int()
    x, off, ad, scale, gm, um, dm = [dev(*t) if isinstance(t, tuple) else dev(t) for t in ffn_inputs(32, 32, 4096, 264, 16, BF16, 1)]
    ws = torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device=DEV)

    def run(v):
        loss, counts = ts.moe_balance(l * v, idx, ws=ws)
        c = ts.adapter_drelu(x * v, gm[0], um[0], gm[1], gm[2], um[1], um[2], off, ad, scale=scale, ws=ws)
        y = ts.adapter_mm(x * v, gm[0], gm[1], gm[2], off, ad, scale=scale, ws=ws)
        return loss, counts, c, y
    want = [run(v) for v in (1.0, 0.5)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for v in (1.0, 0.5):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(v))
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1):
        ws.fill_(0x7F + i)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert same(outs[i], want[i])


def test_a_short_workspace_is_refused():
    x, off, ad, scale, gm, um, dm = [dev(*t) if isinstance(t, tuple) else dev(t) for t in ffn_inputs(8, 8, 128, 264, 16, BF16, 2)]
    n = ts.adapter_workspace_bytes(8, 16, 1, False, 264, 128, BF16, BF16)
    with pytest.raises(ts.TSError, match="WORKSPACE"):
        ts.adapter_mm(x, *gm, off, ad, ws=torch.empty(n - 1, dtype=torch.uint8, device=DEV))
    with pytest.raises(ts.TSError, match="WORKSPACE"):
        ts.moe_balance(torch.zeros(5000, 64, device=DEV), torch.zeros(5000, 2, dtype=torch.int32, device=DEV),
                       ws=torch.empty(16, dtype=torch.uint8, device=DEV))


# --- the largest sizes -----------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_x_past_4_gb(dtype):
    """Adapters beside a product whose x has more than 4 GB, and gathered rows of such
    an x and d_y: on both sides of that offset."""
    k, n, rank, N = 8192, 144, 8, 3
    S = (1 << 32) // (k * (2 if dtype == BF16 else 4)) + 70
    g = gen(97)
    at = torch.cat([torch.arange(0, 40), torch.arange(S - 90, S)])
    few = randn(g, len(at), k, dtype=dtype)
    x = torch.zeros(S, k, dtype=dtype, device=DEV)
    x[at.to(DEV)] = dev(few)
    w, a = randn(g, n, k, dtype=dtype, scale=k ** -0.5), randn(g, N, rank, k, dtype=dtype, scale=k ** -0.5)
    b = randn(g, N, n, rank, dtype=dtype)
    off = torch.tensor([0, 7, 20, S - 60, S - 33, S], dtype=torch.int32)
    ad = torch.tensor([1, -1, 2, 0, 2], dtype=torch.int32)
    few_off = torch.tensor([0, 7, 20, 70, 97, 130], dtype=torch.int32)
    for w_kn in (False, True):
        m = [t.transpose(-1, -2).contiguous() if w_kn and t is not a else t for t in (w, a, b)]
        got = ts.adapter_mm(x, *dev(*m, off, ad), w_kn=w_kn, out_dtype=F32)[at.to(DEV)]
        want, bound = aref.adapted(few, *m, few_off, ad, None, w_kn, 0 if dtype == F32 else 2)
        within(got, want, bound)
    src, goff = at[torch.randperm(len(at), generator=g)], torch.tensor([0, 50, len(at)], dtype=torch.int32)
    back = torch.searchsorted(at, src).int()
    wg, wu = (randn(g, 2, n, k, dtype=dtype, scale=k ** -0.5) for _ in range(2))
    small = ts.grouped_drelu(*dev(few, wg, wu, goff), row_src=dev(back), keep=True, out_dtype=F32)
    c, codes, exps = ts.grouped_drelu_pack(x, *dev(wg, wu, goff), row_src=dev(src.int()), out_dtype=F32)
    assert (c - small[0]).norm() <= 1e-5 * small[0].norm()  # (another tile: another order of the same sums)
    codes, exps = dev(*kref.pack2(small[1].cpu(), small[2].cpu()))
    p = ts.grouped_drelu_grad(x, dev(wg), codes, exps, dev(goff), row_src=dev(src.int()), out_dtype=F32)
    q = ts.grouped_drelu_grad(dev(few), dev(wg), codes, exps, dev(goff), row_src=dev(back), out_dtype=F32)
    for i, j in zip(p, q):
        assert (i - j).norm() <= 1e-5 * j.norm()


def test_outputs_past_2_31_elements():
    rows, n, k = 140000, 16384, 8
    g = gen(98)
    x, w, w2 = randn(g, rows, k, dtype=BF16), randn(g, 1, n, k, dtype=BF16), randn(g, 1, n, k, dtype=BF16)
    xd, wd, w2d = dev(x, w, w2)
    c, codes, exps = ts.grouped_drelu_pack(xd, wd, w2d)
    gate, up = ts.drelu_unpack(codes, exps)
    dg, du, c2 = ts.grouped_drelu_grad(xd, wd, codes, exps)
    for r in (0, 65535, 131071, 131072, 131073, rows - 1):
        one = ts.grouped_drelu(xd[r:r + 1], wd, w2d, keep=True, out_dtype=F32)
        assert torch.equal(c[r:r + 1], one[0].to(BF16))
        wc, we = kref.pack2(one[1].cpu(), one[2].cpu())
        assert torch.equal(codes[r:r + 1].cpu(), wc) and torch.equal(exps[r:r + 1].cpu(), we)
        gk, uk = kref.values2(wc, we)
        assert torch.equal(gate[r].cpu().double(), gk[0]) and torch.equal(up[r].cpu().double(), uk[0])
        d, mag = gref.mm(x[r:r + 1], w, [0, 1])
        f = uk * (gk > 0)
        within(dg[r:r + 1], d * f, gref.rounded(gref.sum_bound(mag, k + 1) * f, d * f, BF16))
        assert torch.equal(c2[r:r + 1].cpu(), (gk * uk).float().to(BF16))
    del c, codes, exps, gate, up, dg, du, c2
    a, b = randn(g, 2, 8, k, dtype=BF16), randn(g, 2, n, 8, dtype=BF16)
    off, ad = torch.tensor([0, 65536, 131073, rows], dtype=torch.int32), torch.tensor([1, 0, 1], dtype=torch.int32)
    out = ts.adapter_mm(xd, wd[0], *dev(a, b, off, ad))
    for r, i in ((0, 1), (65535, 1), (65536, 0), (131072, 0), (131073, 1), (rows - 1, 1)):
        want, bound = aref.adapted(x[r:r + 1], w[0], a, b, [0, 1], [i], None, False, 1)
        within(out[r:r + 1], want, gref.rounded(bound, want, BF16))


def test_the_most_tokens():
    """2^23 pairs through the balance loss."""
    T, E, K = 1 << 22, 40, 2
    g = torch.Generator(device=DEV).manual_seed(99)
    l = torch.randn(T, E, generator=g, device=DEV)
    idx = torch.randint(0, E, (T, K), generator=g, device=DEV, dtype=torch.int32)
    loss, counts = ts.moe_balance(l, idx)
    wc = torch.bincount(idx.view(-1), minlength=E)
    assert torch.equal(counts[:E].long(), wc) and int(counts[E]) == T
    p, lse = torch.softmax(l.double(), 1), torch.logsumexp(l.double(), 1)
    want = torch.stack([E * (wc.double() / (K * T) * p.sum(0)).sum() / T, (lse * lse).mean()])
    # chains of T / 65536 tokens a lane, 64 lanes, 16 waves; 256 workgroups in 64 bits
    within(loss, want, (T / 65536 + 100 + E) * 2.0 ** -23 * want)
    d = ts.moe_balance_grad(l, counts, torch.ones(2, device=DEV), K)
    f = wc.double() / (K * T)
    at = [0, 1, T // 2, T - 1]
    want = p[at] * (E / T * (f - (p[at] * f).sum(1, keepdim=True)) + 2 / T * lse[at, None])
    mag = p[at] * (E / T * (f + (p[at] * f).sum(1, keepdim=True)) + 2 / T * lse[at, None].abs())
    within(d[at], want, (E + 60) * 2.0 ** -23 * mag)
