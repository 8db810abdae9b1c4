"""The router's balance loss, counts and gradient against 64 bits."""
import pytest
import torch

import balance_util as ref
from gpu_util import DEV
from test_gpu_group import dev, gen, randn, within

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2406_05955_amd.binding") if torch.cuda.is_available() else None
F32 = torch.float32

# every number of lanes that hold a token, experts in fours and not, one workgroup and many
CASES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (64, 8, 2), (500, 3, 1), (129, 17, 4), (1030, 33, 8), (2100, 8, 2), (1025, 16, 6),
         (9000, 4, 1), (5000, 64, 8), (4097, 63, 6), (70001, 40, 2), (140000, 2, 1)]


def inputs(T, E, K, masked, seed=0):
    g = gen(70, T, E, K, seed)
    l = randn(g, T, E) + 2 * randn(g, E)
    idx = l.topk(K).indices.to(torch.int32)
    mask = torch.rand(T, generator=g) < 0.8 if masked else None
    return g, l, idx, mask


def check(l, idx, mask, d_loss, add=None):
    T, E = l.shape
    K = idx.shape[1]
    loss, counts = ts.moe_balance(dev(l), dev(idx), mask=dev(mask))
    want, wc, bound = ref.balance(l, idx, mask)
    assert torch.equal(counts.cpu(), wc)
    within(loss, want, bound, "loss")
    got = ts.moe_balance_grad(dev(l), counts, dev(d_loss), K, mask=dev(mask), add=dev(add))
    want, bound = ref.balance_grad(l, wc, d_loss, K, mask, add)
    within(got, want, bound, "grad")
    return loss, counts, got


@pytest.mark.parametrize("T,E,K", CASES)
@pytest.mark.parametrize("masked", [False, True])
def test_balance(T, E, K, masked):
    g, l, idx, mask = inputs(T, E, K, masked)
    d_loss = torch.tensor([0.7, -0.02])
    check(l, idx, mask, d_loss)
    loss, counts, a = check(l, idx, mask, d_loss, randn(g, T, E, scale=1.0 / T))
    if masked:  # bytes as well as bools
        again = ts.moe_balance(dev(l), dev(idx), mask=dev(mask.to(torch.uint8) * 200))
        assert torch.equal(loss, again[0]) and torch.equal(counts, again[1])


@pytest.mark.parametrize("T,E", [(50, 8), (3000, 64)])
def test_logits_not_on_16_bytes(T, E):
    g, l, idx, mask = inputs(T, E, 2, False, 1)
    room = torch.empty(T * E + 1, device=DEV)
    at = room[1:].view(T, E).copy_(l)
    loss, counts = ts.moe_balance(at, dev(idx))
    a, b = ts.moe_balance(dev(l), dev(idx))
    assert torch.equal(loss, a) and torch.equal(counts, b)
    d = dev(torch.tensor([1.0, 0.1]))
    assert torch.equal(ts.moe_balance_grad(at, counts, d, 2), ts.moe_balance_grad(dev(l), counts, d, 2))


def test_gradient_added_in_place():
    g, l, idx, mask = inputs(3000, 64, 6, True, 2)
    d, add = dev(torch.tensor([1.0, 0.1])), dev(randn(g, 3000, 64))
    _, counts = ts.moe_balance(dev(l), dev(idx), mask=dev(mask))
    want = ts.moe_balance_grad(dev(l), counts, d, 6, mask=dev(mask), add=add)
    got = ts.moe_balance_grad(dev(l), counts, d, 6, mask=dev(mask), add=add, out=add)
    assert got is add and torch.equal(got, want)


@pytest.mark.parametrize("T", [40, 5000])
@pytest.mark.parametrize("E", [8, 13])
def test_tokens_that_leave_nothing(T, E):
    """Rows of -inf, NaN, the lowest value: not counted, no gradient; single
    -inf, NaN and lowest logits have no probability."""
    g, l, idx, mask = inputs(T, E, 2, True, 3)
    l[0], l[1], l[2] = -float("inf"), float("nan"), ref.LOWEST
    l[3, 1:], l[4, ::2], l[5, :3] = -float("inf"), float("nan"), ref.LOWEST
    l[6, 0], l[6, 1:] = float("nan"), ref.LOWEST
    mask[:8] = True
    loss, counts, grad = check(l, idx, mask, torch.tensor([0.5, 0.25]))
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all()
    for r in (0, 1, 2, 6):
        assert bool((grad[r] == 0).all())
    add = randn(g, T, E)
    out = ts.moe_balance_grad(dev(l), counts, dev(torch.tensor([0.5, 0.25])), 2, mask=dev(mask), add=dev(add))
    assert torch.equal(out[:3].cpu(), add[:3])


@pytest.mark.parametrize("T,E", [(0, 8), (5, 8), (6000, 64)])
def test_no_token_counts(T, E):
    l, idx = torch.randn(T, E), torch.zeros(T, 2, dtype=torch.int32)
    loss, counts = ts.moe_balance(dev(l), dev(idx), mask=torch.zeros(T, dtype=torch.bool, device=DEV))
    assert loss.tolist() == [0.0, 0.0] and counts.tolist() == [0] * (E + 1)
    grad = ts.moe_balance_grad(dev(l), counts, dev(torch.ones(2)), 2, mask=torch.zeros(T, dtype=torch.bool, device=DEV))
    assert grad.shape == (T, E) and bool((grad == 0).all())


def test_infinite_logits():
    """One +inf takes all of p, two share it; loss[1] and its gradient are lost
    unless its factor is 0."""
    l = torch.zeros(4, 8)
    l[0, 3] = l[1, 2] = l[1, 6] = float("inf")
    idx = torch.tensor([[3, 0], [2, 6], [0, 1], [0, 1]], dtype=torch.int32)
    loss, counts = ts.moe_balance(dev(l), dev(idx))
    assert counts.tolist() == [3, 2, 1, 1, 0, 0, 1, 0, 4] and loss[1].item() == float("inf")
    want = 8 * sum(c / 8 * p / 4 for c, p in zip(counts.tolist(), [.25, .25, .75, 1.25, .25, .25, .75, .25]))
    assert abs(loss[0].item() - want) <= 32 * 2.0 ** -23 * want
    grad = ts.moe_balance_grad(dev(l), counts, dev(torch.tensor([1.0, 0.0])), 2)
    assert torch.isfinite(grad).all() and bool((grad[0] == 0).all())


def test_indices_out_of_range_and_twice():
    l = torch.zeros(3, 4)
    idx = torch.tensor([[-1, 4], [2, 2], [1, 1 << 30]], dtype=torch.int32)
    _, counts = ts.moe_balance(dev(l), dev(idx))
    assert counts.tolist() == [0, 1, 2, 0, 3]


def test_against_differences():
    g, l, idx, mask = inputs(7, 12, 3, True, 4)
    l, d = l.double(), torch.tensor([0.9, 0.3])
    _, counts = ts.moe_balance(dev(l.float()), dev(idx), mask=dev(mask))
    l = l.float().double()
    got = ts.moe_balance_grad(dev(l.float()), counts, dev(d), 3, mask=dev(mask)).cpu().double()
    n, f = int(mask.sum()), counts[:12].cpu().double() / (3 * int(mask.sum()))

    def loss(x):
        x = x[mask]
        return d[0].double() * 12 * (f * torch.softmax(x, 1).mean(0)).sum() + d[1].double() * (torch.logsumexp(x, 1) ** 2).mean()
    h = 1e-6
    for t in range(7):
        for e in range(12):
            s = torch.zeros_like(l)
            s[t, e] = h
            diff = float((loss(l + s) - loss(l - s)) / (2 * h))
            # differences: 2^-53 x the loss (below 10) / h, h^2; the kernel: fp32
            assert abs(float(got[t, e]) - diff) <= 1e-8 + 64 * 2.0 ** -23


def test_repeats_are_the_same_bits():
    g, l, idx, mask = inputs(70001, 40, 6, True, 5)
    args = dev(l, idx)
    first = ts.moe_balance(*args, mask=dev(mask))
    for _ in range(5):
        again = ts.moe_balance(*args, mask=dev(mask))
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
