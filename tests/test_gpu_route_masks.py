"""The router's gradient where a slot names an expert that the token's logits mask: the slot is empty, whatever stands in its gradient."""
import pytest
import torch

from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mask", [-float("inf"), float("nan")])
@pytest.mark.parametrize("E", [12, 100, 300, 700])
def test_slots_of_masked_experts_are_empty(E, mask, dtype):
    gen = torch.Generator(device="cuda").manual_seed(E)
    l = torch.randn((9, E), generator=gen, device="cuda").to(dtype)
    idx = torch.stack([torch.randperm(E, generator=gen, device="cuda")[:5] for _ in range(9)]).to(torch.int32)
    g = torch.randn((9, 5), generator=gen, device="cuda")
    masked = torch.rand((9, 5), generator=gen, device="cuda") < 0.4
    masked[0], masked[1] = False, True
    fixed = torch.where(masked, -1, idx)
    for t in range(9):
        for j in range(5):
            if masked[t, j]:
                l[t, idx[t, j]] = mask
    l[2] = mask
    for bad in (float("nan"), float("inf"), 3.0):
        given = torch.where(masked, bad, g)
        for renorm in (True, False):
            got = B.route_backward(l, idx, given, renorm)
            assert bool(torch.isfinite(got).all())
            want = B.route_backward(l, fixed, g, renorm)
            assert torch.equal(got, want)
            assert bool((got[1:3] == 0).all())
