"""The activations alone, over every bf16 argument of a range, against 64 bits and relative to the value: the products in front of them are
with the identity, so the argument is exact.

Units are 2^-23.  The exponential is off by 2 + 1.173 |argument| (the CUDA programming guide's bound of __expf), the quotient by 2.
gelu: the polynomial 4, the quotient's 2 twice (the polynomial goes at most with the square of its argument), the rounding of z^2 as 0.5 z^2 / 2,
products and the rest 2: 12 + 1.7 z^2 / 2.  The slope is a sum of Phi and z phi, each as good.
silu: the exponential of -|z|, the quotient and three roundings, 8 + 1.173 |z|.  The slope p (1 + z (1 - p)) takes two such factors: twice that, of
p (1 + |z| (1 - p))."""
import pytest
import torch

from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -23
LOW = 2.0 ** -126        # below it fp32 has fewer bits


def act_exact(z, act):
    """The activation and its slope.  (The lower tail of Phi as erfc: one plus erf cancels there, in 64 bits too.)"""
    if act == "gelu":
        c = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
        return z * c, c + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    if act == "silu":
        p, rest = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
        return z * p, p * (1 + z * rest)
    return (torch.relu(z), (z > 0).double()) if act == "relu" else (z, torch.ones_like(z))


def arguments(most):
    """Every bf16 number up to `most` in magnitude and not below 2^-20 of it, of both signs, and zero: [1, rows, 8]."""
    z = torch.arange(0x8000, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    z = z[(z <= most) & ((z >= most * 2.0 ** -20) | (z == 0))]
    z = torch.cat((z, -z))
    z = torch.nn.functional.pad(z, (0, -len(z) % 8))
    return z.view(1, -1, 8).to(torch.bfloat16).cuda()


def rows_of(x):
    n = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([x.shape[1]], dtype=torch.int32, device="cuda")
    return B.ExpertRows(*n)


def units(z, act):
    return {"gelu": 12 + 0.85 * z * z, "silu": 8 + 1.173 * z.abs()}.get(act, torch.zeros_like(z)) * UNIT


def step(v):
    """Half a step of bf16 at a value."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=LOW))) - 8)


def check(name, got, want, tol):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float((off / tol).max()):.3g} of the tolerance"


@pytest.mark.parametrize("act,most", [("gelu", 13.0), ("silu", 100.0), ("relu", 100.0), ("none", 100.0)])
def test_values_and_slopes(act, most):
    x = arguments(most)
    z, one = x.double(), torch.eye(8, dtype=torch.bfloat16, device="cuda")[None]
    rows = rows_of(x)
    value, slope = act_exact(z, act)
    rel = units(z, act)
    y = B.expert_linear(rows, x, one, act=act)
    check("bf16 value", y, value, rel * value.abs() * (1 + 2.0 ** -8) + step(value) + LOW * (1 + z.abs()))
    # the gated block: gate z, and one in the other matrix's place for a ninth channel that is one
    wide = torch.cat((x, torch.ones_like(x)), -1)
    w = torch.zeros((1, 2, 8, 16), dtype=torch.bfloat16, device="cuda")
    w[0, 0, :, :8] = one[0]
    w[0, 1, :, 8] = 1.0
    h = B.expert_gated(rows, wide, w, act=act)
    check("gated value", h, value, rel * value.abs() * (1 + 2.0 ** -8) + step(value) + LOW * (1 + z.abs()))
    # fp32: the row weight's gradient of a gradient that is one in a single place
    for j in range(8):
        gy = torch.zeros_like(x)
        gy[..., j] = 1.0
        s = torch.ones(x.shape[:2], device="cuda")
        gs = B.expert_linear_backward(rows, x, one, gy, pre=x, row_scale=s, act=act, grad_x=False, grad_w=False, grad_row_scale=True)[3]
        check("fp32 value", gs, value[..., j], rel[..., j] * value[..., j].abs() + LOW * (1 + z[..., j].abs()))
    # the slope, rounded to bf16
    gx = B.expert_linear_backward(rows, x, one, torch.ones_like(x), pre=x, act=act, grad_w=False)[0]
    size = slope.abs()
    if act == "gelu":
        size = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5) + (z * torch.exp(-z * z / 2)).abs() * 0.3989422804014327
    if act == "silu":
        size = 2 * (1 + z.abs() / (1 + torch.exp(z))) / (1 + torch.exp(-z))
    check("slope", gx, slope, rel * size * (1 + 2.0 ** -8) + step(slope) + LOW * (1 + z.abs()))
    gg = B.expert_gated_backward(rows, wide, w, torch.stack((x, torch.ones_like(x)), 2), torch.ones_like(x), act=act, grad_w=False)[0]
    check("gated slope", gg[..., :8], slope, rel * size * (1 + 2.0 ** -8) + step(slope) + LOW * (1 + z.abs()))
