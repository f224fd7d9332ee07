"""The largest numbers of experts and the widest rows the calls take, and calls of several streams at once beside library products.  The checks
and their tolerances are those of test_gpu_experts."""
import pytest
import torch

import test_gpu_experts as X
from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu

MOST = 1 << 20
SEGMENTS = {
    "most_experts": (5, 13200, [((e % 13107), 1 if e % 7 else 0) for e in range(65535)]),
    "few": (1, 20, [(0, 3), (3, 0), (5, 9)]),
    "pairs": (1, 220, [(0, 37), (40, 150)]),
}


@pytest.fixture
def extreme(monkeypatch):
    for name, s in SEGMENTS.items():
        monkeypatch.setitem(X.SEGMENTS, name, s)
    yield
    torch.cuda.empty_cache()


def test_most_experts(extreme):
    # (the formulas of every expert at once: one row each, weights of 8 x 8)
    R = X.Rows("most_experts")
    gen = X._gen(1)
    used = torch.tensor([n for _, n in SEGMENTS["most_experts"][2]], device="cuda") > 0
    x, w = R.randn(gen, 8), X._weights(gen, R.E, 2, 8, 8)
    at = torch.arange(R.E, device="cuda") // R.L * R.cap + R.rows.offset.long()
    rows = lambda t: torch.where(used[(...,) + (None,) * (t.dim() - 2)], t.reshape(R.R * R.cap, *t.shape[2:])[at].double(), 0.0)  # noqa: E731
    xe = rows(x)
    g, u = (torch.einsum("ek,enk->en", xe, w[:, i].double()) for i in range(2))
    out, pre = R.filled(8), R.filled(2, 8)
    B.expert_gated(R.rows, x, w, out=out, pre=pre)
    for i, t in enumerate((g, u)):
        tol = 8 * X.SUM * torch.einsum("ek,enk->en", xe.abs(), w[:, i].double().abs()) + X.HALF * t.abs() * (1 + X.HALF)
        assert bool(((rows(pre)[:, i] - t).abs() <= tol + X.TINY).all())
    v = X.act_exact(g, "silu")[0]
    size = xe.abs().sum(1, keepdim=True) * w.double().abs().amax(dim=(1, 2, 3))[:, None]
    assert bool(((rows(out) - v * u).abs() <= X.HALF * (v * u).abs() * (1 + X.HALF) + 2.0 ** -17 * size * (1 + size)).all())
    grad = R.randn(gen, 8)
    gx, gw = R.filled(8), torch.full_like(w, X.FILL)
    B.expert_gated_backward(R.rows, x, w, pre, grad, grad_x=gx, grad_w=gw)
    p, dh = rows(pre), rows(grad)
    v, s = X.act_exact(p[:, 0], "silu")
    d = torch.stack((dh * p[:, 1] * s, dh * v), 1)
    # (the factors rounded to bf16, the result too; values and slopes are good to 2^-18 of 1 + |z|)
    off = X.HALF * d.abs() + 2.0 ** -18 * torch.stack((dh * p[:, 1], dh), 1).abs() * (1 + p[:, :1].abs())
    want = d[..., None] * xe[:, None, None]
    assert bool(((gw.double() - want).abs() <= (off[..., None] * xe[:, None, None].abs()) * (1 + X.HALF) + X.HALF * want.abs() + X.TINY).all())
    want = torch.einsum("ein,eink->ek", d, w.double())
    tol = torch.einsum("ein,eink->ek", off + 16 * X.SUM * d.abs(), w.double().abs()) * (1 + X.HALF) + X.HALF * want.abs()
    assert bool(((rows(gx) - want).abs() <= tol + X.TINY).all())
    assert torch.equal(gx[~R.mine], torch.full_like(gx[~R.mine], X.FILL)) and torch.equal(out[~R.mine], torch.full_like(out[~R.mine], X.FILL))
    # the linear product with a bias of its own per expert, and the bias's gradient
    w3, bias = w[:, 0].contiguous(), torch.randn((R.E, 8), generator=gen, device="cuda").to(torch.bfloat16)
    y = R.filled(8)
    B.expert_linear(R.rows, x, w3, bias=bias, out=y)
    want = torch.where(used[:, None], g + bias.double(), 0.0)
    tol = 9 * X.SUM * (torch.einsum("ek,enk->en", xe.abs(), w3.double().abs()) + bias.double().abs()) + X.HALF * want.abs() * (1 + X.HALF)
    assert bool(((rows(y) - want).abs() <= tol + X.TINY).all())
    gb = B.expert_linear_backward(R.rows, x, w3, grad, grad_x=False, grad_w=False, grad_bias=True)[2]
    assert torch.equal(gb.double(), dh)      # one row's gradient, or nothing: a bf16 number
    assert int(R.rows.status.item()) == 0


@pytest.mark.parametrize("name", ["few", "pairs"])
def test_widest_rows(extreme, name):
    X.test_linear(name, MOST, 8)
    X.test_linear_backward(name, MOST, 8)
    X.test_gated(name, MOST, 8)
    X.test_gated_backward(name, MOST, 8)
    X.test_gated_takes_fp8_rows(name, MOST, 8)
    X.test_gated_backward_takes_fp8_rows(name, MOST, 8)


def test_widest_results(extreme):
    X.test_linear("few", 8, MOST)
    X.test_gated("few", 8, MOST)
    X.test_gated_backward("few", 8, MOST)
    # (no row weight's gradient of such rows)
    R = X.Rows("few")
    gen = X._gen(2)
    x, w, gy = R.randn(gen, 8), X._weights(gen, R.E, MOST, 8), R.randn(gen, MOST)
    gx, gw, gb = R.filled(8), torch.full_like(w, X.FILL), torch.full((R.E, MOST), X.FILL, dtype=torch.bfloat16, device="cuda")
    B.expert_linear_backward(R.rows, x, w, gy, grad_x=gx, grad_w=gw, grad_bias=gb)
    d = torch.where(R.mine[..., None], gy.double(), 0.0)
    want_x, tx, want_w, tw = X.grads_exact(R, x, w, d, 8)
    R.check("grad_x", gx, want_x, tx)
    X.check_all("grad_w", gw, want_w, tw)
    want = torch.stack([d[r, a:b].sum(0) for _, r, a, b in R.seg])
    tol = torch.stack([(b - a + 4) * X.SUM * d[r, a:b].abs().sum(0) for _, r, a, b in R.seg])
    X.check_all("grad_bias", gb, want, tol * (1 + X.HALF) + X.HALF * want.abs())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_router_of_most_experts(dtype):
    from test_gpu_route import _exact, _logits, _rel
    E = 65535
    l = _logits(6, E, dtype, 3, True)
    l[5] = -float("inf")
    l[5, E - 1] = torch.finfo(dtype).min      # the last one alone
    for renorm in (True, False):
        idx, w = B.route(l, 8, renorm)
        want_idx, want_w = _exact(l, 8, renorm)
        assert torch.equal(idx.long(), want_idx)
        assert bool(((w.double() - want_w).abs() <= _rel(E) * want_w + 1e-37).all())
        g = B.route_backward(l, idx, torch.ones_like(w), renorm)
        assert bool(torch.isfinite(g).all()) and bool((g[l.isnan() | (l == -float("inf"))] == 0).all())


def test_streams_at_once_beside_library_products():
    # pairs, single CTAs, FP8 rows and gradients on streams of their own, large products of the library on another
    gen = X._gen(9)

    def case(E, rows, H, I):
        cap = E * rows
        r = B.ExpertRows(torch.arange(E, dtype=torch.int32, device="cuda") * rows, torch.full((E,), rows - 3, dtype=torch.int32, device="cuda"))
        x, w = torch.randn((1, cap, H), generator=gen, device="cuda").to(torch.bfloat16), X._weights(gen, E, 2, I, H)
        q, scale = x.to(torch.float8_e4m3fn), torch.rand((1, cap, H // 128), generator=gen, device="cuda")
        new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        h, pre, f, gx, gw = new(1, cap, I), new(1, cap, 2, I), new(1, cap, I), new(1, cap, H), new(E, 2, I, H)

        def run():
            B.expert_gated(r, x, w, out=h, pre=pre)
            B.expert_gated(r, q, w, x_scale=scale, out=f)
            B.expert_gated_backward(r, q, w, pre, h, x_scale=scale, grad_x=gx, grad_w=gw)
        return run, (h, pre, f, gx, gw)

    cases = [case(4, 300, 512, 768), case(24, 40, 1024, 512), case(8, 130, 256, 2056)]
    a = torch.randn((4096, 4096), generator=gen, device="cuda").to(torch.bfloat16)
    want = []
    for run, outs in cases:
        run()
        want.append([t.clone() for t in outs])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    other = torch.cuda.Stream()
    for _ in range(30):
        for (run, _), s in zip(cases, streams):
            with torch.cuda.stream(s):
                run()
        with torch.cuda.stream(other):
            torch.mm(a, a)
    torch.cuda.synchronize()
    for (_, outs), w in zip(cases, want):
        for t, v in zip(outs, w):
            assert torch.equal(t, v)
