"""Measured passes of the operators that train a layer's experts in less memory
and serve what was trained to many requests: the router's balance loss with its
gradient, dReLU's activations kept in 8 bits with the backward product that
reads them, and low-rank adapters beside a shared projection.

Layer shapes are the repository's own (Mixtral: 8 experts of hidden 4096, inter
14336, top 2; the small fp32 layer 512 x 1792) or generic.  Weights are N(0,
1/fan-in), x ~ N(0, 1), logits N(0, 1) with a fixed bias per expert, so groups are
ragged as a trained router's are.

Kept activations: max(0, gate) and max(0, up), 8 bits each, with no sign, 4 bits of
exponent and 4 of mantissa; 0 stands for "not positive".  Blocks of 16 columns
share the exponent byte of their largest.  With t = the value's fp32 bits rounded
to 4 bits of mantissa (to nearest even), shifted right by 19, and the block's
E0 = max(15, largest t >> 4): code = max(1, t - 16 E0 + 240).
"""
import math

import torch

own = False

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = torch.finfo(F32).min


def listed():
    return [
        # the router of one short training sequence: a launch's latency
        {"name": "balance_t64_e8", "op": "balance", "T": 64, "E": 8, "K": 2, "mask": False},
        # a training batch with padded places, a router of many experts
        {"name": "balance_t16384_e64", "op": "balance", "T": 16384, "E": 64, "K": 6, "mask": True},
        # a whole step's tokens of one GPU at once, an odd number: bytes
        {"name": "balance_t200001_e64", "op": "balance", "T": 200001, "E": 64, "K": 8, "mask": False},
        # the small fp32 layer in training
        {"name": "pack_f32_t300", "op": "pack", "type": "f32", "T": 300, "E": 8, "K": 2, "H": 512, "I": 1792},
        # a training step's forward products
        {"name": "pack_bf16_t4096", "op": "pack", "type": "bf16", "T": 4096, "E": 8, "K": 2, "H": 4096, "I": 14336},
        # its backward product, in fp32 and of an odd number of tokens
        {"name": "grad_f32_t301", "op": "grad", "type": "f32", "T": 301, "E": 8, "K": 2, "H": 512, "I": 1792},
        {"name": "grad_bf16_t3001", "op": "grad", "type": "bf16", "T": 3001, "E": 8, "K": 2, "H": 4096, "I": 14336},
        # one decoded token with its adapter, down projection: bound by the shared weights' bytes
        {"name": "adapt_down_t1", "op": "adapt", "type": "bf16", "out": "bf16", "T": 1, "S": 1, "N": 8, "R": 16, "k": 14336, "n": 4096, "kn": True},
        # 32 decoded tokens of as many requests, each with an adapter of its own: down, then gate + up
        {"name": "adapt_down_t32", "op": "adapt", "type": "bf16", "out": "f32", "T": 32, "S": 32, "N": 64, "R": 16, "k": 14336, "n": 4096, "kn": True},
        {"name": "adapt_drelu_t32", "op": "adapt_drelu", "type": "bf16", "out": "bf16", "T": 32, "S": 32, "N": 64, "R": 16, "k": 4096, "n": 14336},
        # prompts of several requests, ragged, and larger adapters
        {"name": "adapt_drelu_t6001", "op": "adapt_drelu", "type": "bf16", "out": "bf16", "T": 6001, "S": 40, "N": 16, "R": 64, "k": 4096, "n": 14336},
        # the small fp32 layer, odd sizes
        {"name": "adapt_up_f32_t77", "op": "adapt", "type": "f32", "out": "f32", "T": 77, "S": 9, "N": 5, "R": 8, "k": 512, "n": 1788, "kn": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: every operator, both types, one token
    to a step's batch, one request to many, odd and ragged sizes."""
    op = rng.choice(["balance", "pack", "pack", "grad", "grad", "adapt", "adapt", "adapt_drelu", "adapt_drelu"])
    if op == "balance":
        E = rng.choice([2, 8, 16, 40, 63, 64])
        return {"op": op, "T": _log(rng, 1, 200001), "E": E, "K": rng.choice([k for k in (1, 2, 6, 8) if k <= E]), "mask": rng.random() < 0.5}
    f32 = rng.random() < 0.25
    q = 4 if f32 else 8
    if op in ("pack", "grad"):
        E = rng.choice([1, 4, 8, 8, 16])
        K = min(E, rng.choice([1, 2, 2, 4]))
        return {"op": op, "type": "f32" if f32 else "bf16", "T": _log(rng, 1, (1024 if f32 else 6002) // K), "E": E, "K": K,
                "H": _log(rng, 512, 2048 if f32 else 4096) // q * q, "I": _log(rng, 1024, 4096 if f32 else 14336 * 8 // max(E, 8)) // q * q}
    T = _log(rng, 1, 600 if f32 else 6001)
    S = min(T, _log(rng, 1, 200))
    c = {"op": op, "type": "f32" if f32 else "bf16", "out": rng.choice(["f32", "bf16"]), "T": T, "S": rng.choice([S, S, min(T, 200)]),
         "N": rng.choice([1, 5, 16, 64]), "R": rng.choice([8, 16, 16, 24, 32, 64]),
         "k": _log(rng, 512, 2048 if f32 else 8192) // q * q, "n": _log(rng, 512, 2048 if f32 else 8192) // q * q}
    if op == "adapt":
        c["kn"] = rng.random() < 0.5
    return c


# ---------------------------------------------------------------------------
# Inputs.

def _type(name):
    return F32 if name == "f32" else BF16


def _randn(g, *shape, dtype=F32, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype).mul_(scale)


def _maps(g, T, E, K):
    """Offsets and the rows' tokens of a random routing, and the largest group's size."""
    logits = _randn(g, T, E) + 0.3 * _randn(g, E)
    idx = logits.topk(K, dim=1).indices.reshape(-1)
    order = torch.sort(idx, stable=True).indices
    count = torch.zeros(E, dtype=torch.int64, device=DEV).index_add_(0, idx, torch.ones_like(idx))
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = count.cumsum(0)
    return {"offsets": offsets, "row_token": (order // K).to(torch.int32), "cap": int(count.max())}


def _segments(g, T, S, N):
    """Requests of ragged lengths that hold all rows (as many rows as requests:
    one each), and their adapters, a tenth of them without one."""
    if T == S:
        offsets = torch.arange(S + 1, device=DEV)
    else:
        # (cuts closer together at the front: short requests beside long ones)
        cuts = (torch.rand(S - 1, generator=g, device=DEV) ** 2 * T).long().sort().values
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), cuts, torch.full((1,), T, dtype=torch.int64, device=DEV)])
    ad = torch.randperm(N, generator=g, device=DEV).repeat(-(-S // N))[:S]
    ad = torch.where(torch.rand(S, generator=g, device=DEV) < 0.1, torch.full_like(ad, -1), ad)
    row = torch.repeat_interleave(ad, offsets[1:] - offsets[:-1])
    used = row[row >= 0]
    cap = int(torch.zeros(N, dtype=torch.int64, device=DEV).index_add_(0, used, torch.ones_like(used)).max())
    return {"offsets": offsets.to(torch.int32), "adapter": ad.to(torch.int32), "row_adapter": row, "cap": cap}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, T = case["op"], case["T"]
    s = {"case": case}
    if op == "balance":
        E, K = case["E"], case["K"]
        s["logits"] = _randn(g, T, E) + 0.3 * _randn(g, E)
        s["idx"] = s["logits"].topk(K, dim=1).indices.to(torch.int32)
        s["mask"] = torch.rand(T, generator=g, device=DEV) < 0.9 if case["mask"] else None
        # the loss is the tokens' mean: the gradient that it is added to is of that size too
        s["d_loss"] = torch.tensor([1e-2, 1e-3], device=DEV) * (0.5 + torch.rand(2, generator=g, device=DEV))
        s["d_route"] = _randn(g, T, E, scale=1e-2 / T)
        return s
    ty = _type(case["type"])
    if op in ("pack", "grad"):
        E, K, H, I = case["E"], case["K"], case["H"], case["I"]
        R = T * K
        s.update(_maps(g, T, E, K))
        if op == "pack":
            s["x"] = _randn(g, T, H, dtype=ty)
            s["wg"] = _randn(g, E, I, H, dtype=ty, scale=H ** -0.5)
            s["wu"] = _randn(g, E, I, H, dtype=ty, scale=H ** -0.5)
            return s
        s["d_y"] = _randn(g, R, H, dtype=ty, scale=1e-3)
        s["w"] = _randn(g, E, I, H, dtype=ty, scale=I ** -0.5)
        kept = [_codes(_randn(g, R, I)) for _ in range(2)]
        s["codes"] = torch.stack([k[0] for k in kept], dim=2)
        s["exps"] = torch.stack([k[1] for k in kept], dim=2)
        return s
    S, N, R, k, n = (case[v] for v in ("S", "N", "R", "k", "n"))
    s.update(_segments(g, T, S, N))
    s["x"] = _randn(g, T, k, dtype=ty)
    s["scale"] = 0.5 + torch.rand(N, generator=g, device=DEV)
    for p in ("g", "u") if op == "adapt_drelu" else ("",):
        kn = case.get("kn", False)
        s["w" + p] = _randn(g, *((k, n) if kn else (n, k)), dtype=ty, scale=k ** -0.5)
        s["a" + p] = _randn(g, N, R, k, dtype=ty, scale=k ** -0.5)
        s["b" + p] = _randn(g, N, *((R, n) if kn else (n, R)), dtype=ty, scale=0.5 * R ** -0.5)
    return s


# ---------------------------------------------------------------------------
# The plain forms.

def _steps(v):
    """16 x exponent + mantissa of max(0, v), rounded to 4 bits of mantissa (a
    finite value to the largest finite one at most), and where v > 0."""
    on = v > 0
    b = torch.where(on, v, 0.0).view(torch.int32)
    b = torch.where(b < 0x7F800000, b.clamp(max=0x7F7BFFFF), b)
    return (b + 0x3FFFF + ((b >> 19) & 1)) >> 19, on


def _blocks(t):
    """t [rows][n] in blocks of 16 columns (zeros behind the last), and each block's E0."""
    R, n = t.shape
    t = torch.nn.functional.pad(t, (0, -n % 16)).view(R, -1, 16)
    return t, (t.amax(2) >> 4).clamp(min=15)


def _codes(v):
    t, on = _steps(v)
    b, e0 = _blocks(t)
    q = (b - 16 * e0[:, :, None] + 240).clamp(min=1).view(v.shape[0], -1)[:, :v.shape[1]]
    return torch.where(on, q, 0).to(torch.uint8), e0.to(torch.uint8)


def _code_values(codes, exps):
    """bf16 values (all of them exact) of codes [rows][n] with exps [rows][blocks]."""
    n = codes.shape[1]
    t = codes.int() - 240 + 16 * exps.int().repeat_interleave(16, 1)[:, :n]
    return torch.where(codes > 0, t << 3, 0).to(torch.int16).view(BF16)


def _expert_of_row(s, R):
    row = torch.arange(R, device=DEV)
    off = s["offsets"].long()
    e = torch.searchsorted(off[1:].contiguous(), row, right=True)
    return e, e * s["cap"] + row - off[e]


def _mm(rows, w, s):
    """y[r] = rows[r] w[e(r)]^T in 32 bits."""
    E, R = w.shape[0], rows.shape[0]
    if R <= E:
        return torch.bmm(w[_expert_of_row(s, R)[0]].float(), rows.float()[:, :, None])[:, :, 0]
    at = _expert_of_row(s, R)[1]
    p = torch.zeros(E * s["cap"], rows.shape[1], dtype=F32, device=DEV)
    p[at] = rows.float()
    return torch.bmm(p.view(E, s["cap"], -1), w.float().transpose(1, 2)).view(E * s["cap"], -1)[at]


def _relu2(g, u):
    return torch.where((g > 0) & (u > 0), g * u, 0.0)


def _adapted(s, p, kn):
    """x W^T + scale (x A^T) B^T of the rows' adapters, in 32 bits."""
    x, w, a, b = s["x"].float(), s["w" + p].float(), s["a" + p].float(), s["b" + p].float()
    b = b if kn else b.transpose(1, 2)  # [N][R][n]
    y = x @ (w if kn else w.t())
    ad = s["row_adapter"]
    T, N = x.shape[0], a.shape[0]
    on, at = ad >= 0, ad.clamp(min=0)
    if T <= N:
        t = torch.bmm(a[at], x[:, :, None]) * s["scale"][at][:, None, None]
        d = torch.bmm(t.transpose(1, 2), b[at])[:, 0]
        return y + torch.where(on[:, None], d, 0.0)
    # rows sorted by adapter, `cap` places for each
    order = torch.argsort(ad, stable=True)
    key = ad[order]
    first = torch.searchsorted(key, torch.arange(N, device=DEV))
    place = torch.where(key >= 0, key * s["cap"] + torch.arange(T, device=DEV) - first[key.clamp(min=0)], N * s["cap"])
    rows = torch.zeros(N * s["cap"] + 1, x.shape[1], device=DEV)
    rows[place] = x[order]
    t = torch.bmm(rows[:-1].view(N, s["cap"], -1), a.transpose(1, 2)) * s["scale"][:, None, None]
    d = torch.nn.functional.pad(torch.bmm(t, b).view(N * s["cap"], -1), (0, 0, 0, 1))
    return y.index_add(0, order, torch.where(key[:, None] >= 0, d[place], 0.0))


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "balance":
        E, K, l = c["E"], c["K"], s["logits"]
        m = l.amax(1, keepdim=True)
        valid = m[:, 0] > LOWEST
        if s["mask"] is not None:
            valid = valid & s["mask"]
        e = torch.exp(l - m)
        total = e.sum(1, keepdim=True)
        p = torch.where(valid[:, None], e / total, 0.0)
        lse = torch.where(valid, m[:, 0] + torch.log(total[:, 0]), 0.0)
        n = valid.sum()
        hit = (s["idx"][:, :, None] == torch.arange(E, device=DEV)) & valid[:, None, None]
        counts = torch.cat([hit.sum((0, 1)), n[None]]).to(torch.int32)
        nf = n.clamp(min=1).double()
        f = (counts[:E].double() / (K * nf))
        loss = torch.stack([E * (f * p.double().sum(0) / nf).sum(), (lse.double() ** 2).sum() / nf])
        d0, d1 = s["d_loss"][0] * E / nf.float(), s["d_loss"][1] * 2 / nf.float()
        f = f.float()
        d = p * (d0 * (f - (p * f).sum(1, keepdim=True)) + d1 * lse[:, None])
        return {"loss": loss.float(), "counts": counts, "d_logits": s["d_route"] + d}
    ty = _type(c["type"])
    if op == "pack":
        rows = s["x"][s["row_token"].long()]
        g, u = _mm(rows, s["wg"], s), _mm(rows, s["wu"], s)
        return {"c": _relu2(g, u).to(ty), "gate": _code_values(*_codes(g)), "up": _code_values(*_codes(u))}
    if op == "grad":
        d = _mm(s["d_y"], s["w"], s)
        g, u = (_code_values(s["codes"][:, :, i], s["exps"][:, :, i]).float() for i in (0, 1))
        on = (g > 0) & (u > 0)
        return {"d_gate": torch.where(on, d * u, 0.0).to(ty), "d_up": torch.where(on, d * g, 0.0).to(ty), "c": (g * u).to(ty)}
    out = _type(c["out"])
    if op == "adapt":
        return _adapted(s, "", c["kn"]).to(out)
    return _relu2(_adapted(s, "g", False), _adapted(s, "u", False)).to(out)


# ---------------------------------------------------------------------------
# The framework's calls.

def _run_own(s):
    from paper_2406_05955_amd import binding as ts
    c = s["case"]
    op = c["op"]
    if op == "balance":
        loss, counts = ts.moe_balance(s["logits"], s["idx"], mask=s["mask"])
        d = ts.moe_balance_grad(s["logits"], counts, s["d_loss"], c["K"], mask=s["mask"], add=s["d_route"])
        return {"loss": loss, "counts": counts, "d_logits": d}
    if op == "pack":
        comb, codes, exps = ts.grouped_drelu_pack(s["x"], s["wg"], s["wu"], s["offsets"], row_src=s["row_token"])
        gate, up = ts.drelu_unpack(codes, exps)
        return {"c": comb, "gate": gate, "up": up}
    if op == "grad":
        dg, du, comb = ts.grouped_drelu_grad(s["d_y"], s["w"], s["codes"], s["exps"], s["offsets"])
        return {"d_gate": dg, "d_up": du, "c": comb}
    out = _type(c["out"])
    if op == "adapt":
        return ts.adapter_mm(s["x"], s["w"], s["a"], s["b"], s["offsets"], s["adapter"], scale=s["scale"], w_kn=c["kn"], out_dtype=out)
    return ts.adapter_drelu(s["x"], s["wg"], s["wu"], s["ag"], s["bg"], s["au"], s["bu"], s["offsets"], s["adapter"], scale=s["scale"], out_dtype=out)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

def _groups(offsets):
    off = offsets.tolist()
    return [(e, a, b) for e, (a, b) in enumerate(zip(off[:-1], off[1:])) if b > a]


def _kept(v):
    """The values that are kept of max(0, v): 5 significant bits, at least 17/16 x
    2^-15 of the power of two of the largest of 16 columns."""
    v = v.clamp(min=0.0)
    out = torch.empty_like(v)
    for a in range(0, v.shape[1], 16):
        m, e = torch.frexp(v[:, a:a + 16])
        q = torch.ldexp(torch.round(m * 32.0), e - 5)
        top = torch.frexp(q.amax(1, keepdim=True))[1].clamp(min=15 - 126) - 1
        least = torch.ldexp(torch.full_like(q[:, :1], 17.0 / 16.0), top - 15)
        out[:, a:a + 16] = torch.where(v[:, a:a + 16] > 0, torch.maximum(q, least), torch.zeros_like(q))
    return out


def _decoded(codes, exps):
    """Values of codes: (1 + low 4 bits / 16) 2^(high bits + exponent byte - 15 - 127)."""
    out = torch.empty(codes.shape, dtype=torch.float64, device=DEV)
    for j in range(exps.shape[1]):
        q = codes[:, 16 * j:16 * j + 16]
        mantissa, e = 1.0 + (q % 16).double() / 16.0, (q // 16).int() + exps[:, j:j + 1].int() - 142
        out[:, 16 * j:16 * j + 16] = torch.ldexp(mantissa, e) * (q != 0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    D = torch.float64
    if op == "balance":
        T, E, K = case["T"], case["E"], case["K"]
        keep = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"]
        l, idx = s["logits"][keep].double(), s["idx"][keep].long()
        n = l.shape[0]
        counts = torch.bincount(idx.reshape(-1), minlength=E)
        lse = torch.logsumexp(l, 1) if n else l.new_zeros(0)
        p = torch.exp(l - lse[:, None])
        f = counts.double() / (K * max(n, 1))
        loss = torch.stack([E * (f * p.sum(0)).sum() / max(n, 1), (lse * lse).sum() / max(n, 1)])
        d0, d1 = s["d_loss"].double()
        d = s["d_route"].double()
        if n:
            d[keep] += p * f * (d0 * E / n) - p * (p @ f)[:, None] * (d0 * E / n) + p * lse[:, None] * (2.0 * d1 / n)
        return {"loss": loss, "counts": torch.cat([counts, torch.tensor([n], device=DEV)]).to(torch.int32), "d_logits": d}
    if op in ("pack", "grad"):
        E, K, H, I = case["E"], case["K"], case["H"], case["I"]
        R = case["T"] * K
        if op == "pack":
            g, u = (torch.empty(R, I, dtype=D, device=DEV) for _ in range(2))
            for e, a, b in _groups(s["offsets"]):
                rows = s["x"][s["row_token"][a:b].long()].double()
                g[a:b], u[a:b] = rows @ s["wg"][e].double().t(), rows @ s["wu"][e].double().t()
            return {"c": g.clamp(min=0) * u.clamp(min=0), "gate": _kept(g), "up": _kept(u)}
        d = torch.empty(R, I, dtype=D, device=DEV)
        for e, a, b in _groups(s["offsets"]):
            d[a:b] = s["d_y"][a:b].double() @ s["w"][e].double().t()
        g, u = (_decoded(s["codes"][:, :, i], s["exps"][:, :, i]) for i in (0, 1))
        return {"d_gate": d * u * (g > 0), "d_up": d * g * (u > 0), "c": g * u}

    def projected(p):
        kn = case.get("kn", False)
        w = s["w" + p].double()
        y = s["x"].double() @ (w if kn else w.t())
        for (_, a, b), i in [(r, int(s["adapter"][r[0]])) for r in _groups(s["offsets"])]:
            if i >= 0:
                up = s["b" + p][i].double()
                t = s["x"][a:b].double() @ s["a" + p][i].double().t()
                y[a:b] += s["scale"][i].double() * (t @ (up if kn else up.t()))
        return y
    if op == "adapt":
        return projected("")
    return projected("g").clamp(min=0) * projected("u").clamp(min=0)


# ---------------------------------------------------------------------------

def work(case):
    op, T = case["op"], case["T"]
    if op == "balance":
        E, K = case["E"], case["K"]
        # logits, the choices and the mask; the gradient that is added to, and the result
        return {"bytes": 12 * T * E + 4 * T * K + (T if case["mask"] else 0) + 4 * (E + 1), "flops": 12 * T * E}
    es = 4 if case["type"] == "f32" else 2
    if op in ("pack", "grad"):
        E, K, H, I = case["E"], case["K"], case["H"], case["I"]
        R = T * K
        w = E * (1 - (1 - K / E) ** T) * I * H  # experts that draw a token (expected)
        kept = 2 * R * I + 2 * R * -(-I // 16)
        if op == "pack":  # the kept codes out, their values (16 bits) out
            return {"bytes": int(es * (2 * w + T * H + R * I) + kept + 4 * R * I) + 4 * R, "flops": 4 * R * H * I}
        return {"bytes": int(es * (w + R * H + 3 * R * I) + kept), "flops": 2 * R * H * I}
    S, N, R, k, n = (case[v] for v in ("S", "N", "R", "k", "n"))
    both = 2 if op == "adapt_drelu" else 1
    used = min(N, 0.9 * S)
    return {"bytes": int(es * (both * (n * k + used * R * (n + k)) + T * k) + (4 if case["out"] == "f32" else 2) * T * n),
            "flops": 2 * both * T * (k * n + R * (k + n))}
