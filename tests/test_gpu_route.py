"""The router and its gradient against the formulas in 64 bits: order with ties, masked experts, every number of experts.

Tolerances: a weight is a quotient of exponentials, each good to a few 2^-23 of its value (its argument, a difference of two fp32
values, to 2^-24 of the difference, at most 2^-24 * 40 for weights above 1e-17); sums of at most 4000 terms of one sign add as
many roundings of 2^-24 at worst, 2^-12, and in a tree of 32 lanes far fewer: 2^-24 * (E / 32 + 40)."""
import pytest
import torch

from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu

EXPERTS = [1, 2, 7, 31, 32, 33, 64, 65, 128, 160, 256, 288, 512, 513, 1000, 1024, 1025, 4000]


def _rel(E):
    return 2.0 ** -24 * (E / 32 + 40) + 2.0 ** -20


def _logits(T, E, dtype, seed, masked):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    l = (torch.randn((T, E), generator=g, device="cuda") * 2).to(dtype)
    if masked:
        l[torch.rand((T, E), generator=g, device="cuda") < 0.6] = -float("inf")
        l[torch.rand((T, E), generator=g, device="cuda") < 0.1] = float("nan")
        l[0] = -float("inf")
        if T > 1:
            l[1] = float("nan")
        if T > 2:
            l[2] = -float("inf")
            l[2, E // 2] = torch.finfo(dtype).min
        if T > 3:
            l[3] = torch.finfo(dtype).min
        if T > 4:
            l[4] = 0.0
            l[4, ::2] = -0.0
    return l


def _exact(l, k, renorm):
    l = torch.where(l.isnan(), -float("inf"), l.double())
    order = torch.argsort(-l, dim=1, stable=True)[:, :k]
    order = torch.nn.functional.pad(order, (0, k - order.shape[1]), value=-1)
    value = torch.where(order >= 0, l.gather(1, order.clamp(min=0)), -float("inf"))
    used = value > -float("inf")
    # (relative to the largest: of the type's lowest value even 64 bits hold no sum with a logarithm)
    most = torch.where(used[:, :1], value[:, :1], 0.0)
    total = torch.exp((value if renorm else l) - most).sum(1, keepdim=True)
    w = torch.where(used, torch.exp(value - most) / torch.where(total > 0, total, 1.0), 0.0)
    return torch.where(used, order, -1), w


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("E", EXPERTS)
def test_route(E, dtype, masked):
    for T, k in ((1, 1), (5, 2), (131, 8), (16, 32)):
        l = _logits(T, E, dtype, E * 100 + k, masked)
        for renorm in (True, False):
            idx, w = B.route(l, k, renorm)
            want_idx, want_w = _exact(l, k, renorm)
            assert idx.dtype == torch.int32 and w.dtype == torch.float32 and idx.shape == w.shape == (T, k)
            assert torch.equal(idx.long(), want_idx)
            off = (w.double() - want_w).abs()
            assert bool((off <= _rel(E) * want_w + 1e-37).all()), float(off.max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("E", EXPERTS)
def test_route_backward(E, dtype, masked):
    for T, k in ((1, 1), (5, 2), (131, 8), (16, 32)):
        l = _logits(T, E, dtype, E * 100 + k, masked)
        for renorm in (True, False):
            idx, w = _exact(l, k, renorm)
            g = torch.randn((T, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(E + k))
            g[idx < 0] = float("nan")                       # slots without an expert: nobody looks at them
            got = B.route_backward(l, idx.to(torch.int32), g, renorm)
            gz = torch.where(idx < 0, 0.0, g.double())
            mean = (w * gz).sum(1, keepdim=True)
            size = (w * gz.abs()).sum(1, keepdim=True)
            ld = torch.where(l.isnan(), -float("inf"), l.double())
            p = torch.zeros_like(ld)
            if not renorm:
                p = torch.softmax(ld, 1).nan_to_num(0.0)
            want = -p * mean
            tol = p * size
            at = idx.clamp(min=0)
            chosen = torch.where(idx < 0, 0.0, w * (gz - (mean if renorm else 0.0)))
            want = want.scatter_add(1, at, chosen)
            tol = tol.scatter_add(1, at, torch.where(idx < 0, 0.0, w * (gz.abs() + size)))
            half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24
            off = (got.double() - want).abs()
            assert got.dtype == dtype
            assert bool((off <= 4 * _rel(E) * tol + half * want.abs() + 1e-37).all()), float(off.max())


def test_gradient_is_that_of_differences():
    l = _logits(6, 20, torch.float32, 5, False)
    for renorm in (True, False):
        idx, _ = B.route(l, 4, renorm)
        g = torch.randn((6, 4), device="cuda")
        got = B.route_backward(l, idx, g, renorm).double()
        step = 1e-5
        for e in (int(idx[0, 0]), int(idx[2, 3]), 7):
            def value(t):
                m = l.double().clone()
                m[:, e] += t
                v = m.gather(1, idx.long())
                return (torch.exp(v - torch.logsumexp(v if renorm else m, 1, keepdim=True)) * g.double()).sum(1)
            want = (value(step) - value(-step)) / (2 * step)
            assert bool(((got[:, e] - want).abs() <= 1e-6).all())


def test_repeated_and_foreign_ids_count_as_empty_slots():
    l = _logits(4, 16, torch.float32, 9, False)
    idx = torch.tensor([[3, 5, 3], [-1, 2, 16], [7, 7, 7], [-5, 99, -1]], dtype=torch.int32, device="cuda")
    fixed = torch.tensor([[3, 5, -1], [-1, 2, -1], [7, -1, -1], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    g = torch.randn((4, 3), device="cuda")
    for renorm in (True, False):
        got = B.route_backward(l, idx, g, renorm)
        assert torch.equal(got, B.route_backward(l, fixed, g, renorm))
    assert bool((got[3] == 0).all())


def test_no_tokens_and_given_outputs():
    l = _logits(9, 24, torch.bfloat16, 2, False)
    idx, w = torch.empty((9, 3), dtype=torch.int32, device="cuda"), torch.empty((9, 3), device="cuda")
    got = B.route(l, 3, topk_idx=idx, topk_w=w)
    assert got[0] is idx and got[1] is w
    a, b = B.route(l[:0], 3)
    assert a.shape == b.shape == (0, 3)
    assert B.route_backward(l[:0], a, b).shape == (0, 24)


def test_refusals():
    l = _logits(9, 24, torch.float32, 2, False)
    idx, w = B.route(l, 3)
    n0 = B.ubep_launch_count()
    for call in (lambda: B.route(l.half(), 3), lambda: B.route(l[0], 3), lambda: B.route(l.cpu(), 3),
                 lambda: B.route(l, 3, topk_idx=idx.long()), lambda: B.route(l, 3, topk_w=w[:5]),
                 lambda: B.route_backward(l, idx.long(), w), lambda: B.route_backward(l, idx, w[:, :2].contiguous()),
                 lambda: B.route_backward(l, idx, w, grad_logits=l.bfloat16())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AssertionError):
        B.route(l.t(), 3)
    for call in (lambda: B.route(l, 0), lambda: B.route(l, 33), lambda: B.route_backward(l, idx, w, grad_logits=l)):
        with pytest.raises(B.UbepError) as e:
            call()
        assert e.value.code == B.UBEP_ERR_ARG
    assert B.ubep_launch_count() == n0
