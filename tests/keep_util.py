"""dReLU's activations in 8 bits, from their definition in 64 bits (results on
the inputs' device)."""
import torch

D = torch.float64
U8 = torch.uint8
BLOCK = 16


def _blocked(v):
    pad = -v.shape[1] % BLOCK
    return torch.nn.functional.pad(v, (0, pad)).view(v.shape[0], -1, BLOCK)


def steps(v):
    """16 x biased exponent + mantissa of max(0, v) rounded to 5 significant bits
    (finite to finite); fp32's subnormals have the exponent 0 and no hidden bit."""
    v = v.double()
    v = torch.where(v > 0, v, torch.zeros_like(v))
    m, e = torch.frexp(v)
    e = e + 126                                       # biased, v = 2 m 2^(e - 127)
    normal = 16 * e.double() + torch.round(32 * m) - 16
    small = torch.round(torch.ldexp(v, torch.tensor(126 + 4, device=v.device)))   # in units of 2^-130
    t = torch.where(e >= 1, normal, small)
    t = torch.where(torch.isinf(v), torch.full_like(t, 4080), t.clamp(max=4079))
    return torch.where(v > 0, t, torch.zeros_like(t)).long()


def pack(v):
    """(codes [rows][n], exps [rows][ceil(n / 16)]) of max(0, v)."""
    t = steps(v)
    b = _blocked(t)
    e0 = (b.amax(2) // 16).clamp(min=15)
    q = (b - 16 * e0[:, :, None] + 240).clamp(min=1).view(v.shape[0], -1)[:, :v.shape[1]]
    return torch.where(v > 0, q, torch.zeros_like(q)).to(U8), e0.to(U8)


def pack2(gate, up):
    (a, b), (c, d) = pack(gate), pack(up)
    return torch.stack([a, c], 2).contiguous(), torch.stack([b, d], 2).contiguous()


def values(codes, exps):
    """64-bit values of codes [rows][n] with exps [rows][blocks]."""
    q = codes.long()
    t = q - 240 + 16 * exps.long().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    e, m = t // 16, t % 16
    one = torch.ones_like(m, dtype=D)
    v = torch.where(e > 0, torch.ldexp(one + m.double() / 16, e - 127), torch.ldexp(m.double() / 16, torch.full_like(e, -126)))
    v = torch.where(t == 4080, torch.full_like(v, float("inf")), v)
    return torch.where(q > 0, v, torch.zeros_like(v))


def values2(codes, exps):
    return values(codes[:, :, 0], exps[:, :, 0]), values(codes[:, :, 1], exps[:, :, 1])


# values at which the codes can go wrong: both zeros, subnormals, around E0 = 15,
# halfway cases, the largest finite, infinities, NaN
EDGES = [0.0, -0.0, -1.0, 2.0 ** -149, 2.0 ** -131, 3 * 2.0 ** -131, 2.0 ** -126, 2.0 ** -113, 2.0 ** -112, 1.03125, 1.09375, 1.0,
         33.0 / 32, 35.0 / 32, 63.0 / 32, 2.0 - 2.0 ** -23, 2.0 ** -15, 17 * 2.0 ** -19, 2.0 ** -16, 1e-30, 3.4028234663852886e38,
         -3.4e38, float("inf"), -float("inf"), float("nan"), 2.0 ** 127 * 1.96875, 2.0 ** 127 * 1.96874]
