"""The balance loss: its 64-bit form against autograd, and what the host refuses."""
import pytest
import torch

import balance_util as ref
from paper_2406_05955_amd import binding as ts

OK, NULL, SHAPE, DTYPE, ALIGN, WS, HIP, UNSUP = range(8)
A = 0x10000


def test_gradient_of_the_plain_form():
    g = torch.Generator().manual_seed(3)
    T, E, K = 30, 6, 2
    l = torch.randn(T, E, generator=g, dtype=torch.float64, requires_grad=True)
    mask = torch.rand(T, generator=g) < 0.7
    idx = l.detach().topk(K).indices.int()
    _, counts, _ = ref.balance(l.detach().float(), idx, mask)
    n = int(mask.sum())
    p = torch.softmax(l[mask], 1)
    f = counts[:E].double() / (K * n)
    d = torch.tensor([0.3, -0.7])
    (d[0].double() * E * (f * p.mean(0)).sum() + d[1].double() * (torch.logsumexp(l[mask], 1) ** 2).mean()).backward()
    got, _ = ref.balance_grad(l.detach(), counts, d, K, mask)
    assert torch.allclose(got, l.grad, rtol=1e-6, atol=1e-12)


def _fwd(l=A, idx=A, mask=None, T=100, E=8, K=2, loss=A, counts=A, ws=A, wsb=1 << 30):
    return ts.lib.ts_moe_balance(l, idx, mask, T, E, K, loss, counts, ws, wsb, None)


def _bwd(l=A, counts=A, dl=A, mask=None, add=None, T=100, E=8, K=2, out=A):
    return ts.lib.ts_moe_balance_grad(l, counts, dl, mask, add, T, E, K, out, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_refused_sizes(call):
    for bad in (dict(T=-1), dict(E=0), dict(E=65), dict(K=0), dict(K=9, E=16), dict(K=3, E=2), dict(T=(1 << 23) + 1, K=1)):
        assert call(**bad) == SHAPE, bad


def test_refused_pointers():
    for name in ("l", "idx", "loss", "counts"):
        assert _fwd(**{name: None}) == NULL
        assert _fwd(**{name: A + 2}) == ALIGN
    assert _fwd(T=0, l=None, idx=None, loss=None) == NULL
    for name in ("l", "counts", "dl", "out"):
        assert _bwd(**{name: None}) == NULL
        assert _bwd(**{name: A + 2}) == ALIGN
    assert _bwd(add=A + 1) == ALIGN
    assert _bwd(T=0, l=None) == OK


def test_workspace():
    assert ts.lib.ts_moe_balance_workspace_bytes(64, 8, 2) == 0
    n = ts.lib.ts_moe_balance_workspace_bytes(100000, 64, 2)
    assert n > 0 and ts.lib.ts_moe_balance_workspace_bytes(100000, 65, 2) == 0
    assert _fwd(T=100000, E=64, ws=None) == WS and _fwd(T=100000, E=64, wsb=n - 1) == WS
    assert _fwd(T=100000, E=64, ws=A + 4) == ALIGN


def test_binding_refuses_tensors():
    l, i = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="contiguous device"):
        ts.moe_balance(l, i)
    with pytest.raises(TypeError, match="logits"):
        ts.moe_balance(l.double(), i)
    with pytest.raises(ValueError, match="topk_idx"):
        ts.moe_balance(l, i[:3])
    with pytest.raises(TypeError, match="mask"):
        ts.moe_balance(l, i, mask=torch.zeros(4))
    with pytest.raises(ValueError, match="mask"):
        ts.moe_balance(l, i, mask=torch.zeros(3, dtype=torch.bool))
    c, d = torch.zeros(9, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError, match="counts"):
        ts.moe_balance_grad(l, c[:8], d, 2)
    with pytest.raises(ValueError, match="d_loss"):
        ts.moe_balance_grad(l, c, d[:1], 2)
    with pytest.raises(ValueError, match="top_k"):
        ts.moe_balance_grad(l, c, d, 9)
    with pytest.raises(ValueError, match="add"):
        ts.moe_balance_grad(l, c, d, 2, add=l[:2])
