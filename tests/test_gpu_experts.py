"""The experts' products and their gradients against the formulas in 64 bits, at the segment lengths, widths and contents
where they can go wrong.

Tolerances, elementwise: a bf16 result is off by half a step, 2^-8 of its value; a sum of n products kept in 32 bits by at most
n 2^-23 of the sum of the products' magnitudes (a rounding or a truncation per product); an activation by 2^-18 of its
magnitude (exp and a quotient of a few 2^-23 each, and cancellation where 1 + erf is small: absolute 2^-22, below); gradients of
products take factors rounded to bf16, 2^-8 of every product's magnitude."""
import numpy as np
import pytest
import torch

from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8          # half a step of bf16
SUM = 2.0 ** -23          # per product of a sum
ACT = 2.0 ** -18
TINY = 1e-30
FILL = 7.0

# segments: (regions, rows per region, [(offset, count) of every expert])
SEGMENTS = {
    "one_row": (1, 1, [(0, 1)]),
    "nobody": (1, 8, [(0, 0), (0, 0)]),
    "small": (2, 70, [(0, 1), (1, 0), (1, 15), (0, 16), (16, 17), (33, 33)]),
    "edges": (1, 700, [(0, 63), (63, 64), (127, 65), (192, 0), (192, 128), (320, 129), (449, 250)]),
    "one_long": (1, 1100, [(3, 1000)]),
    "gaps_out_of_order": (2, 300, [(200, 57), (10, 100), (0, 31), (250, 50)]),
    # what passes the region's end is left out, and an offset or a count that makes no sense has no rows
    "over_the_end": (2, 96, [(0, 60), (60, 100), (2 ** 31 - 1, 5), (96, 1), (-7, 20), (40, -3), (90, 2 ** 31 - 1), (50, 9)]),
    "few_rows_in_long_regions": (1, 400, [(0, 1), (1, 0), (1, 16), (17, 31)]),
    "long_over_the_end": (2, 500, [(0, 257), (257, 1000), (2 ** 31 - 1, 5), (-7, 400), (400, 33), (499, 2)]),
    "two_pieces": (1, 3000, [(1, 255), (256, 256), (512, 513), (1025, 1290)]),
    "many_experts": (5, 40, [(i % 8 * 5, (i * 7) % 6) for i in range(40)]),
}


def _clip(cap, offset, count):
    first = min(max(offset, 0), cap)
    return first, min(max(count, 0), cap - first)


class Rows:
    def __init__(self, name):
        self.R, self.cap, seg = SEGMENTS[name]
        self.E = len(seg)
        self.L = self.E // self.R
        assert self.E % self.R == 0
        clipped = [_clip(self.cap, o, c) for o, c in seg]
        self.seg = [(e, e // self.L, a, a + n) for e, (a, n) in enumerate(clipped)]
        self.rows = B.ExpertRows(torch.tensor([o for o, _ in seg], dtype=torch.int64).to(torch.int32).cuda(),
                                 torch.tensor([c for _, c in seg], dtype=torch.int64).to(torch.int32).cuda(),
                                 torch.zeros(1, dtype=torch.int32, device="cuda"))
        self.mine = torch.zeros((self.R, self.cap), dtype=torch.bool, device="cuda")
        for _, r, a, b in self.seg:
            self.mine[r, a:b] = True

    def each(self):
        return [(e, r, a, b) for e, r, a, b in self.seg if b > a]

    def randn(self, gen, *width, scale=1.0, hostile=True):
        """Rows; those of no segment hold NaN and infinities."""
        t = torch.randn((self.R, self.cap, *width), generator=gen, device="cuda").mul_(scale).to(torch.bfloat16)
        if hostile:
            t[~self.mine] = float("nan")
            t[~self.mine, ..., :1] = float("inf")
        return t

    def filled(self, *width, dtype=torch.bfloat16):
        return torch.full((self.R, self.cap, *width), FILL, dtype=dtype, device="cuda")

    def check(self, name, got, want, tol):
        """got at the segments' rows within tol of want, everything else as it was."""
        g = got.double()
        assert torch.equal(got[~self.mine], torch.full_like(got[~self.mine], FILL)), f"{name}: a row of no segment was written"
        off = (g - want).abs()[self.mine]
        bad = ~(off <= tol[self.mine] + TINY)
        assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float((off / (tol[self.mine] + TINY)).max()):.3g} of the tolerance"
        assert int(self.rows.status.item()) == 0


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _weights(gen, *shape):
    return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)


def act_exact(z, name):
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    if name == "gelu":
        c = torch.special.ndtr(z)
        return z * c, c + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
    if name == "relu":
        return torch.relu(z), (z > 0).double()
    return z, torch.ones_like(z)


def act_error(z, dz, name):
    """How far the activation may be off for an argument off by dz (all slopes are below 1.13)."""
    return 1.13 * dz + ACT * z.abs() + (2.0 ** -22 * z.abs() if name == "gelu" else 0.0)


def f64(t, width=None):
    shape = t.shape if width is None else (*t.shape[:2], *width)
    return torch.zeros(shape, dtype=torch.float64, device="cuda")


def gated_exact(R, x, w, act):
    H, I = x.shape[2], w.shape[2]
    pre, pre_tol = f64(x, (2, I)), f64(x, (2, I))
    for e, r, a, b in R.each():
        xe = x[r, a:b].double()
        for i in range(2):
            pre[r, a:b, i] = xe @ w[e, i].double().T
            pre_tol[r, a:b, i] = H * SUM * (xe.abs() @ w[e, i].double().abs().T)
    g, u = pre[:, :, 0], pre[:, :, 1]
    v = act_exact(g, act)[0]
    dv = act_error(g, pre_tol[:, :, 0], act)
    h = v * u
    tol = dv * (u.abs() + pre_tol[:, :, 1]) + v.abs() * pre_tol[:, :, 1]
    return pre, pre_tol + HALF * pre.abs(), h, tol * (1 + HALF) + HALF * h.abs()


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("H,I", [(8, 8), (72, 136), (256, 512)])
def test_gated(segments, H, I):
    R = Rows(segments)
    gen = _gen(H + I)
    x, w = R.randn(gen, H), _weights(gen, R.E, 2, I, H)
    for act in ("silu", "gelu"):
        out, pre = R.filled(I), R.filled(2, I)
        assert B.expert_gated(R.rows, x, w, act=act, out=out, pre=pre) is out
        want_pre, pre_tol, want, tol = gated_exact(R, x, w, act)
        R.check("pre", pre, want_pre, pre_tol)
        R.check("h", out, want, tol)
        again = R.filled(I)
        B.expert_gated(R.rows, x, w, act=act, out=again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("H,I", [(2000, 264), (1024, 1408)])
def test_gated_wide(act, H, I):
    R = Rows("edges")
    gen = _gen(3)
    x, w = R.randn(gen, H), _weights(gen, R.E, 2, I, H)
    out = R.filled(I)
    B.expert_gated(R.rows, x, w, act=act, out=out)
    _, _, want, tol = gated_exact(R, x, w, act)
    R.check("h", out, want, tol)


def _fp8(R, gen, H):
    """e4m3 rows with a scale per 128 channels, and what they stand for; rows of no segment have no number as their scale."""
    x = torch.randn((R.R, R.cap, H), generator=gen, device="cuda")
    scale = torch.rand((R.R, R.cap, H // 128), generator=gen, device="cuda") * 0.02 + 0.001
    q = (x / scale.repeat_interleave(128, dim=2)).clamp(-448, 448).to(torch.float8_e4m3fn)
    scale[~R.mine] = float("nan")
    rows = q.float().double() * scale.double().repeat_interleave(128, dim=2)
    rows[~R.mine] = 0
    return q, scale, rows


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("H,I", [(128, 8), (384, 136), (1024, 264)])
def test_gated_takes_fp8_rows(segments, H, I):
    # (the values are multiplied as they are and the sums scaled in 32 bits: no rounding to bf16 on the way)
    R = Rows(segments)
    gen = _gen(5)
    q, scale, rows = _fp8(R, gen, H)
    w = _weights(gen, R.E, 2, I, H)
    want_pre, pre_tol, want, tol = gated_exact(R, rows, w, "silu")
    for t in (q, q.view(torch.uint8)):
        out, pre = R.filled(I), R.filled(2, I)
        B.expert_gated(R.rows, t, w, x_scale=scale, out=out, pre=pre)
        R.check("pre", pre, want_pre, pre_tol)
        R.check("h", out, want, tol)
        again = R.filled(I)
        B.expert_gated(R.rows, t, w, x_scale=scale, out=again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("H,I", [(128, 72), (640, 264)])
def test_gated_backward_takes_fp8_rows(segments, H, I):
    # (rows as the sum of two bf16 numbers, off by half a step of the second: 2^-17 of the value)
    R = Rows(segments)
    gen = _gen(6)
    q, scale, rows = _fp8(R, gen, H)
    w, pre, grad = _weights(gen, R.E, 2, I, H), R.randn(gen, 2, I), R.randn(gen, I)
    g, u, dh = (torch.where(R.mine[..., None], t.double(), 0.0) for t in (pre[:, :, 0], pre[:, :, 1], grad))
    v, s = act_exact(g, "silu")
    d = torch.cat((dh * u * s, dh * v), -1)
    size = torch.cat((dh * u * (1 + g.abs()), dh * (1 + g.abs())), -1).abs() * 2.0 ** -18
    gx, tx, gw, tw = grads_exact(R, rows, w.view(R.E, 2 * I, H), d, H)
    _, sx, _, sw = grads_exact(R, rows, w.view(R.E, 2 * I, H), size / HALF, H)
    grad_x, grad_w = R.filled(H), torch.full_like(w, FILL)
    B.expert_gated_backward(R.rows, q, w, pre, grad, x_scale=scale, grad_x=grad_x, grad_w=grad_w)
    R.check("grad_x", grad_x, gx, tx + sx)
    # (two products per row: twice the terms of the sum)
    check_all("grad_w", grad_w.view(R.E, 2 * I, H), gw, tw * (1 + 2.0 ** -8) + sw + R.cap * SUM * tw / HALF)
    only = B.expert_gated_backward(R.rows, q, w, pre, grad, x_scale=scale, grad_w=False)[0]
    assert torch.equal(only[R.mine], grad_x[R.mine])


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("K,N", [(8, 8), (136, 264), (512, 256)])
def test_linear(segments, K, N):
    R = Rows(segments)
    gen = _gen(K + N)
    x, w = R.randn(gen, K), _weights(gen, R.E, N, K)
    bias = torch.randn((R.E, N), generator=gen, device="cuda").to(torch.bfloat16)
    scale = torch.randn((R.R, R.cap), generator=gen, device="cuda")
    residual = R.randn(gen, N)
    z, dz = f64(x, (N,)), f64(x, (N,))
    for e, r, a, b in R.each():
        xe, we = x[r, a:b].double(), w[e].double()
        z[r, a:b] = xe @ we.T
        dz[r, a:b] = K * SUM * (xe.abs() @ we.abs().T)
    for act, use_bias, use_scale, use_res in (("none", 0, 0, 0), ("none", 1, 1, 0), ("gelu", 1, 0, 1), ("relu", 0, 1, 1), ("silu", 1, 1, 1)):
        out, pre = R.filled(N), R.filled(N)
        B.expert_linear(R.rows, x, w, bias=bias if use_bias else None, row_scale=scale if use_scale else None,
                        residual=residual if use_res else None, act=act, out=out, pre=pre)
        zb, dzb = z.clone(), dz.clone()
        if use_bias:
            for e, r, a, b in R.each():
                zb[r, a:b] += bias[e].double()
            dzb += 2.0 ** -23 * (zb.abs() + dz)
        R.check("pre", pre, zb, dzb + HALF * (zb.abs() + dzb))
        y, dy = act_exact(zb, act)[0], act_error(zb, dzb, act) if act != "none" else dzb
        if use_scale:
            s = scale.double()[..., None]
            y, dy = y * s, dy * s.abs() + 2.0 ** -23 * (y * s).abs()
        if use_res:
            res = torch.where(R.mine[..., None], residual.double(), 0.0)
            y, dy = y + res, dy + 2.0 ** -23 * (y.abs() + res.abs())
        R.check("y", out, y, dy + HALF * (y.abs() + dy))
        if use_res:   # the residual's memory may be the result's
            own = residual.clone()
            B.expert_linear(R.rows, x, w, bias=bias if use_bias else None, row_scale=scale if use_scale else None, residual=own, act=act,
                            out=own)
            assert torch.equal(own[R.mine], out[R.mine])


def grads_exact(R, x, w, d, width):
    """grad_x, grad_w and their tolerances, of factors d that are rounded to bf16."""
    gx, tx = f64(x, (w.shape[-1],)), f64(x, (w.shape[-1],))
    gw, tw = f64(w), f64(w)
    for e, r, a, b in R.each():
        de, we, xe = d[r, a:b], w[e].double(), x[r, a:b].double()
        n = de.shape[1]
        gx[r, a:b] = de @ we
        tx[r, a:b] = (HALF + n * SUM) * (de.abs() @ we.abs())
        gw[e] = de.T @ xe
        tw[e] = (HALF + (b - a) * SUM) * (de.abs().T @ xe.abs())
    return gx, tx * (1 + HALF) + HALF * gx.abs(), gw, tw * (1 + HALF) + HALF * gw.abs()


def check_all(name, got, want, tol):
    off = (got.double() - want).abs()
    bad = ~(off <= tol + TINY)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float((off / (tol + TINY)).max()):.3g} of the tolerance"


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("H,I", [(8, 8), (136, 72), (512, 264)])
def test_gated_backward(segments, H, I):
    R = Rows(segments)
    gen = _gen(H * I)
    x, w = R.randn(gen, H), _weights(gen, R.E, 2, I, H)
    pre, grad = R.randn(gen, 2, I), R.randn(gen, I)
    for act in ("silu", "gelu", "relu"):
        g, u, dh = (torch.where(R.mine[..., None], t.double(), 0.0) for t in (pre[:, :, 0], pre[:, :, 1], grad))
        v, s = act_exact(g, act)
        d = torch.cat((dh * u * s, dh * v), -1)
        # (the activation's own error, absolute, beside the rounding: values and slopes are good to 2^-18 of 1 + |z|)
        size = torch.cat((dh * u * (1 + g.abs()), dh * (1 + g.abs())), -1).abs() * 2.0 ** -18
        gx, tx, gw, tw = grads_exact(R, x, w.view(R.E, 2 * I, H), d, H)
        _, sx, _, sw = grads_exact(R, x, w.view(R.E, 2 * I, H), size / HALF, H)
        grad_x, grad_w = R.filled(H), torch.full_like(w, FILL)
        got = B.expert_gated_backward(R.rows, x, w, pre, grad, act=act, grad_x=grad_x, grad_w=grad_w)
        assert got[0] is grad_x and got[1] is grad_w
        R.check("grad_x", grad_x, gx, tx + sx)
        check_all("grad_w", grad_w.view(R.E, 2 * I, H), gw, tw + sw)
        # one of the two alone, and the gradients of pre in pre's own memory
        own = pre.clone()
        alone_x = R.filled(H)
        got = B.expert_gated_backward(R.rows, x, w, own, grad, act=act, grad_x=alone_x, grad_w=False, grad_pre=own)
        assert got[1] is None and torch.equal(alone_x, grad_x)
        assert torch.equal(own[~R.mine].view(torch.int16), pre[~R.mine].view(torch.int16))
        got = B.expert_gated_backward(R.rows, x, w, pre, grad, act=act, grad_x=False)
        assert got[0] is None and torch.equal(got[1], grad_w)


@pytest.mark.parametrize("segments", SEGMENTS)
@pytest.mark.parametrize("K,N", [(8, 8), (264, 136), (256, 512)])
def test_linear_backward(segments, K, N):
    R = Rows(segments)
    gen = _gen(K * N)
    x, w = R.randn(gen, K), _weights(gen, R.E, N, K)
    pre, grad = R.randn(gen, N), R.randn(gen, N)
    scale = torch.randn((R.R, R.cap), generator=gen, device="cuda")
    zero = lambda t: torch.where(R.mine[..., None], t.double(), 0.0)  # noqa: E731
    for act, use_scale in (("none", 0), ("none", 1), ("silu", 1), ("gelu", 0), ("relu", 1)):
        dy, z = zero(grad), zero(pre)
        v, s = act_exact(z, act)
        one = scale.double()[..., None] if use_scale else 1.0
        d = dy * s * one
        size = (dy * (1 + z.abs()) * one).abs() * 2.0 ** -18
        gx, tx, gw, tw = grads_exact(R, x, w, d, K)
        _, sx, _, sw = grads_exact(R, x, w, size / HALF, K)
        used = act != "none" or use_scale
        grad_x, grad_w, grad_b = R.filled(K), torch.full_like(w, FILL), torch.full((R.E, N), FILL, dtype=torch.bfloat16, device="cuda")
        grad_s = R.filled(dtype=torch.float32) if use_scale else None
        B.expert_linear_backward(R.rows, x, w, grad, pre=pre if used else None, row_scale=scale if use_scale else None, act=act,
                                 grad_x=grad_x, grad_w=grad_w, grad_bias=grad_b, grad_row_scale=grad_s)
        R.check("grad_x", grad_x, gx, tx + sx)
        check_all("grad_w", grad_w, gw, tw + sw)
        gb, tb = torch.zeros((R.E, N), dtype=torch.float64, device="cuda"), torch.zeros((R.E, N), dtype=torch.float64, device="cuda")
        for e, r, a, b in R.each():
            gb[e] = d[r, a:b].sum(0)
            tb[e] = ((b - a + 4) * SUM * d[r, a:b].abs() + size[r, a:b]).sum(0)
        check_all("grad_bias", grad_b, gb, tb * (1 + HALF) + HALF * gb.abs())
        if used:   # the gradients of pre in pre's own memory, and what no product needs by itself
            own, alone = pre.clone(), R.filled(K)
            got = B.expert_linear_backward(R.rows, x, w, grad, pre=own, row_scale=scale if use_scale else None, act=act, grad_x=alone,
                                           grad_w=False, grad_pre=own, grad_bias=True)
            assert torch.equal(alone, grad_x) and torch.equal(got[2], grad_b)
            assert torch.equal(own[~R.mine].view(torch.int16), pre[~R.mine].view(torch.int16))
        got = B.expert_linear_backward(R.rows, x, w, grad, pre=pre if used else None, row_scale=scale if use_scale else None, act=act,
                                       grad_x=False, grad_w=False, grad_bias=True)
        assert got[0] is None and got[1] is None and torch.equal(got[2], grad_b)
        if use_scale:
            gs = (dy * v).sum(-1)
            ts = ((N + 4) * SUM * (dy * v).abs() + (dy * (1 + z.abs())).abs() * 2.0 ** -18).sum(-1)
            R.check("grad_row_scale", grad_s, gs, ts)


def test_gated_gradients_are_those_of_differences():
    # d/dv of sum(h * grad) along a random direction of x and of w, by central differences of the formula in 64 bits
    R = Rows("small")
    gen = _gen(11)
    H, I = 64, 48
    x, w = R.randn(gen, H), _weights(gen, R.E, 2, I, H)
    grad = R.randn(gen, I)
    pre = R.filled(2, I)
    B.expert_gated(R.rows, x, w, pre=pre)
    grad_x, grad_w = B.expert_gated_backward(R.rows, x, w, pre, grad)
    dx, dw = torch.randn(x.shape, generator=gen, device="cuda").double(), torch.randn(w.shape, generator=gen, device="cuda").double()
    dx[~R.mine] = 0

    def value(t):
        total = 0.0
        for e, r, a, b in R.each():
            xe, we = x[r, a:b].double() + t * dx[r, a:b], w[e].double() + t * dw[e]
            total += float((act_exact(xe @ we[0].T, "silu")[0] * (xe @ we[1].T) * grad[r, a:b].double()).sum())
        return total

    step = 1e-4
    want = (value(step) - value(-step)) / (2 * step)
    used = torch.zeros(R.E, dtype=torch.bool, device="cuda")
    for e, _, _, _ in R.each():
        used[e] = True
    tx, tw = torch.where(R.mine[..., None], grad_x.double() * dx, 0.0), grad_w.double() * dw * used[:, None, None, None]
    # the products of the roundings (three of them: pre, its gradient, the result) average out over the sum
    size = float(tx.square().sum() + tw.square().sum()) ** 0.5
    assert abs(float(tx.sum() + tw.sum()) - want) <= 3 * HALF * 6 * size + 1e-3


def test_refusals():
    R = Rows("small")
    gen = _gen(1)
    x, w, w3 = R.randn(gen, 64), _weights(gen, R.E, 2, 32, 64), _weights(gen, R.E, 32, 64)
    n0 = B.ubep_launch_count()
    for call in (lambda: B.expert_gated(R.rows, x, w[:-1].contiguous()),
                 lambda: B.expert_gated(R.rows, x, w.float()),
                 lambda: B.expert_gated(R.rows, x.float(), w),
                 lambda: B.expert_gated(R.rows, x[0], w),
                 lambda: B.expert_gated(R.rows, x, w, act="tanh"),
                 lambda: B.expert_gated(R.rows, x, w, out=R.filled(33)),
                 lambda: B.expert_gated(R.rows, x, w, pre=R.filled(32)),
                 lambda: B.expert_gated(R.rows, x.view(torch.uint8), w, x_scale=torch.ones((R.R, R.cap, 1), device="cuda")),
                 lambda: B.expert_gated(B.ExpertRows(R.rows.offset, R.rows.count[:-1]), x, w),
                 lambda: B.expert_gated(B.ExpertRows(R.rows.offset.long(), R.rows.count), x, w),
                 lambda: B.expert_gated(B.ExpertRows(R.rows.offset.cpu(), R.rows.count), x, w),
                 lambda: B.expert_linear(R.rows, x, w),
                 lambda: B.expert_linear(R.rows, x, w3, bias=torch.zeros((R.E, 31), dtype=torch.bfloat16, device="cuda")),
                 lambda: B.expert_linear(R.rows, x, w3, row_scale=torch.zeros((R.R, R.cap), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AssertionError):
        B.expert_gated(R.rows, x.transpose(0, 1), w)
    with pytest.raises(TypeError):
        B.expert_gated(R.rows, None, w)
    grad = R.randn(gen, 32)
    for call in (lambda: B.expert_gated(R.rows, R.randn(gen, 12), _weights(gen, R.E, 2, 32, 12)),     # no multiple of 8
                 lambda: B.expert_linear(R.rows, R.randn(gen, 64), _weights(gen, R.E, 20, 64)),
                 lambda: B.expert_linear(B.ExpertRows(R.rows.offset[:5], R.rows.count[:5]), x, w3[:5].contiguous()),   # 5 experts, 2 regions
                 lambda: B.expert_linear_backward(R.rows, x, w3, grad, act="silu"),                     # no pre
                 lambda: B.expert_linear_backward(R.rows, x, w3, grad, grad_row_scale=True),            # no row_scale
                 lambda: B.expert_linear_backward(R.rows, x, w3, grad, grad_x=False, grad_w=False)):    # nothing asked for
        with pytest.raises(B.UbepError) as e:
            call()
        assert e.value.code == B.UBEP_ERR_ARG
    # an address that is not on a 16-byte boundary
    odd = torch.empty(R.R * R.cap * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(R.R, R.cap, 64)
    with pytest.raises(B.UbepError):
        B.expert_linear(R.rows, odd, w3)
    assert B.ubep_launch_count() == n0
