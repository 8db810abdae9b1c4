"""dReLU's activations in 8 bits: the format's bounds on the CPU, and what the
host refuses before anything is enqueued."""
import pytest
import torch

import keep_util as ref
from paper_2406_05955_amd import binding as ts

OK, NULL, SHAPE, DTYPE, ALIGN, WS, HIP, UNSUP = range(8)
A = 0x10000


def test_format_bounds():
    """Half a step of 5 significant bits, the floor at 2^-15 of the block's
    largest, the support exact, all values exact in bf16."""
    g = torch.Generator().manual_seed(1)
    v = torch.randn(300, 72, generator=g) * torch.exp2(torch.randint(-30, 30, (300, 72), generator=g).float())
    codes, exps = ref.pack(v)
    got, want = ref.values(codes, exps), v.clamp(min=0).double()
    top = torch.exp2(exps.double() - 127).repeat_interleave(16, 1)[:, :72]
    # the least code is 17/16 x 2^-15; 1 x 2^-15 has none, and up to 33/32 rounds to that
    low = want <= top * 2.0 ** -15 * 33 / 32
    assert bool(((got - want).abs()[~low] <= 2.0 ** -5 * want[~low]).all())
    assert bool((got[low & (want > 0)] == (top * 2.0 ** -15 * 17 / 16)[low & (want > 0)]).all())
    assert torch.equal(codes > 0, v > 0)
    assert torch.equal(got.to(torch.bfloat16).double(), got)


def test_format_edges():
    v = torch.tensor(ref.EDGES).view(1, -1)
    for one in (v, v.view(-1, 1)):
        codes, exps = ref.pack(one)
        got = ref.values(codes, exps)
        assert torch.equal(codes > 0, one > 0) and not torch.isnan(got).any()
        assert torch.equal(torch.isinf(got), one == float("inf"))
    # alone in its block, a value is within half a step, from 2^-112 up
    codes, exps = ref.pack(v.view(-1, 1))
    got, want = ref.values(codes, exps).view(-1), v.view(-1).double()
    ok = (want >= 2.0 ** -112) & torch.isfinite(want)
    assert bool(((got - want).abs()[ok] <= 2.0 ** -5 * want[ok]).all())


def _pack(x=A, wg=A, wu=A, dt=1, src=None, off=A, rows=10, srows=10, G=4, n=64, k=64, c=A, codes=A, exps=A, odt=1):
    return ts.lib.ts_grouped_drelu_pack(x, wg, wu, dt, src, off, rows, srows, G, n, k, c, codes, exps, odt, None)


def _grad(dy=A, w=A, dt=1, src=None, off=A, rows=10, srows=10, G=4, n=64, k=64, codes=A, exps=A, dg=A, du=A, c=A, odt=1):
    return ts.lib.ts_grouped_drelu_grad(dy, w, dt, src, off, rows, srows, G, n, k, codes, exps, dg, du, c, odt, None)


def _unpack(codes=A, exps=A, rows=10, n=64, g=A, u=A):
    return ts.lib.ts_drelu_unpack(codes, exps, rows, n, g, u, None)


@pytest.mark.parametrize("call", [_pack, _grad])
def test_refusals_of_the_products(call):
    assert call(dt=2) == DTYPE and call(odt=7) == DTYPE
    for bad in (dict(n=60), dict(k=60), dict(n=0), dict(G=0), dict(G=65), dict(rows=-1), dict(srows=9), dict(srows=0),
                dict(rows=(1 << 23) + 1, srows=(1 << 23) + 1), dict(n=1 << 18), dict(dt=0, n=62)):
        assert call(**bad) == SHAPE, bad
    assert call(off=None) == NULL
    for name in ("codes", "exps"):
        assert call(**{name: None}) == NULL
        assert call(**{name: A + 1}) == ALIGN
    assert call(codes=A + 8) == ALIGN
    assert call(off=A + 2) == ALIGN
    assert call(rows=0, srows=0) == OK


def test_refusals_one_by_one():
    for name in ("x", "wg", "wu", "c"):
        assert _pack(**{name: None}) == NULL
        assert _pack(**{name: A + 4}) == ALIGN
    for name in ("dy", "w", "dg", "du"):
        assert _grad(**{name: None}) == NULL
        assert _grad(**{name: A + 4}) == ALIGN
    assert _grad(c=A + 2) == ALIGN
    for name in ("codes", "exps", "g", "u"):
        assert _unpack(**{name: None}) == NULL
        assert _unpack(**{name: A + 1}) == ALIGN
    for bad in (dict(rows=-1), dict(n=0), dict(n=6), dict(n=(1 << 17) + 4)):
        assert _unpack(**bad) == SHAPE, bad
    assert _unpack(rows=0, codes=None) == OK


def test_binding_refuses_tensors():
    f, u8 = torch.zeros(4, 64), lambda *s: torch.zeros(*s, dtype=torch.uint8)
    w = torch.zeros(1, 32, 64)
    with pytest.raises(ValueError, match="contiguous device"):
        ts.grouped_drelu_pack(f, w, w)
    with pytest.raises(TypeError):
        ts.grouped_drelu_pack(f.half(), w, w)
    with pytest.raises(ValueError):
        ts.grouped_drelu_pack(f, w, torch.zeros(1, 16, 64))
    with pytest.raises(ValueError, match="codes"):
        ts.grouped_drelu_grad(f, w, u8(4, 32), u8(4, 2, 2))
    with pytest.raises(ValueError, match="exps"):
        ts.grouped_drelu_grad(f, w, u8(4, 32, 2), u8(4, 3, 2))
    with pytest.raises(TypeError, match="codes"):
        ts.grouped_drelu_grad(f, w, u8(4, 32, 2).int(), u8(4, 2, 2))
    with pytest.raises(ValueError, match="exps"):
        ts.drelu_unpack(u8(4, 33, 2), u8(4, 2, 2))
    with pytest.raises(ValueError, match="offsets"):
        ts.grouped_drelu_grad(f, torch.zeros(2, 32, 64), u8(4, 32, 2), u8(4, 2, 2))
