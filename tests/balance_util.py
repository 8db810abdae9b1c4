"""The router's balance loss in 64 bits, and what fp32 results may be off by."""
import torch

D, F32 = torch.float64, torch.float32
LOWEST = torch.finfo(F32).min


def counted(logits, mask=None):
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -float("inf")), logits)
    on = (l > LOWEST).any(1)
    return on if mask is None else on & (mask != 0)


def soft(logits):
    """(p, lse, rel, e_lse): softmax and log-sum in 64 bits, the relative error of p
    and the error of lse in fp32: the argument of exp rounded once (and exp's own
    two units), a sum of E, a reciprocal and a product; lse: one log, one sum."""
    E = logits.shape[1]
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -float("inf")), logits).double()
    m = l.amax(1, keepdim=True)
    e = torch.where(l == m, torch.ones_like(l), torch.exp(l - m))
    s = e.sum(1, keepdim=True)
    lse = (m + torch.log(s))[:, 0]
    far = torch.where(e > 1e-37, (l - m).abs(), torch.zeros_like(l)).nan_to_num(0, 0, 0).amax(1, keepdim=True)
    rel = (far + E + 8) * 2.0 ** -23
    e_lse = ((m.abs() + 2 * torch.log(s) + 4) * 2.0 ** -23 + rel)[:, 0]
    return e / s, lse, rel.expand_as(l), e_lse


def balance(logits, idx, mask=None):
    """(loss, counts, bound of loss)."""
    T, E = logits.shape
    K = idx.shape[1]
    on = counted(logits, mask)
    n = int(on.sum())
    i = idx[on].long().reshape(-1)
    counts = torch.zeros(E + 1, dtype=torch.int32)
    for e in range(E):
        counts[e] = int((i == e).sum())
    counts[E] = n
    if n == 0:
        return torch.zeros(2, dtype=D), counts, torch.zeros(2, dtype=D)
    p, lse, rel, e_lse = soft(logits[on])
    f = counts[:E].double() / (K * n)
    # a lane's chain of tokens, then lanes, waves and workgroups
    chain = (T / 2048 + 64) * 2.0 ** -23
    loss = torch.stack([E * (f * p.sum(0)).sum() / n, (lse * lse).sum() / n])
    bound = torch.stack([E * (f * (p * rel).sum(0)).sum() / n + chain * loss[0],
                         (2 * lse.abs() * e_lse + e_lse ** 2).sum() / n + chain * loss[1]])
    return loss, counts, bound + 2.0 ** -126


def balance_grad(logits, counts, d_loss, K, mask=None, add=None):
    """(d_logits, bound)."""
    T, E = logits.shape
    on = counted(logits, mask)[:, None]
    n = max(int(counts[E]), 1)
    p, lse, rel, e_lse = soft(torch.where(on, logits, torch.zeros_like(logits)))
    d0, d1 = float(d_loss[0]) * E / n, 2 * float(d_loss[1]) / n
    f = counts[:E].double() / (K * n)
    dot = (p * f).sum(1, keepdim=True)
    z = d1 * lse[:, None] if d1 else torch.zeros_like(lse[:, None])
    d = p * (d0 * (f - dot) + z)
    mag = p * (abs(d0) * (f + dot) + z.abs())
    bound = mag * (2 * rel + (E + 16) * 2.0 ** -23) + p * abs(d1) * e_lse[:, None]
    d, bound = torch.where(on, d, torch.zeros_like(d)), torch.where(on, bound, torch.zeros_like(d))
    if add is not None:
        d = d + add.double()
    return d, bound + 2.0 ** -24 * d.abs() + 2.0 ** -126
