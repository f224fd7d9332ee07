"""A whole mixture-of-experts layer out of the library's calls -- router, dispatch, experts, combine -- and its backward pass, against
the layer's formula in 64 bits; captured in a graph, on several streams, with FP8 rows, and with ranks that own an arena each.

Tolerance: every array the layer rounds to bf16 on the way (rows, h, y, out; their gradients) is off by at most half a step, 2^-8 of
each value, and the products after it take the errors on with the values, so the norm of the result is off by at most 2^-8 for each of
the roundings in front of it: six of them, forward and backward, at the most used here."""
import pytest
import torch

from paper_2607_06202_b200 import binding as B
from test_gpu_experts import act_exact

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def near(name, got, want, roundings):
    got, want = got.double(), want.double()
    off, size = float((got - want).norm()), float(want.norm())
    assert off <= roundings * HALF * size + 1e-12, f"{name}: off by {off / size:.3g} of the norm"


class Layer:
    def __init__(self, T, H, I, E, R, k, payload=0, seed=0, cap=None, act="silu"):
        self.T, self.H, self.I, self.E, self.R, self.k, self.payload, self.act = T, H, I, E, R, k, payload, act
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(torch.bfloat16)  # noqa: E731
        self.x, self.logits = bf(T, H), torch.randn((T, E), generator=g, device="cuda")
        self.w1, self.w2, self.grad = bf(E, 2, I, H, scale=H ** -0.5), bf(E, H, I, scale=I ** -0.5), bf(T, H)
        self.bias = bf(E, H, scale=0.1)
        cap = cap or T * min(k, E // R)
        mk = lambda p: B.Buffer(num_ranks=R, num_experts=E, hidden=H, topk=k, max_tokens=T, rows_per_rank_cap=cap,  # noqa: E731
                                payload=p, fill=0xA5)
        self.buf, self.gbuf = mk(payload), mk(0)
        self.cap = cap
        self.ones = torch.ones((T, k), device="cuda")
        self.h, self.pre = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((R, cap, I), (R, cap, 2, I)))
        self.y, self.z = (torch.empty((R, cap, H), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.idx, self.w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
        self.out = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")

    def serve(self):
        B.route(self.logits, self.k, topk_idx=self.idx, topk_w=self.w)
        self.buf.dispatch(self.x, self.idx, self.w)
        rows = self.buf.expert_segments()
        B.expert_gated(rows, self.buf.recv_x, self.w1, act=self.act, x_scale=self.buf.recv_scale, out=self.h)
        B.expert_linear(rows, self.h, self.w2, bias=self.bias, out=self.y)
        return self.buf.combine(self.y, self.w, self.out)

    def train_forward(self):
        B.route(self.logits, self.k, topk_idx=self.idx, topk_w=self.w)
        self.buf.dispatch(self.x, self.idx, self.w)
        rows = self.buf.expert_segments()
        B.expert_gated(rows, self.buf.recv_x, self.w1, act=self.act, x_scale=self.buf.recv_scale, out=self.h, pre=self.pre)
        B.expert_linear(rows, self.h, self.w2, bias=self.bias, row_scale=self.buf.recv_weight, out=self.y, pre=self.z)
        return self.buf.combine(self.y, self.ones, self.out)

    def train_backward(self):
        rows = self.buf.expert_segments()
        self.gbuf.dispatch(self.grad, self.idx, self.w)          # the same table: the same rows
        gy = self.gbuf.recv_x.view(torch.bfloat16)
        gh, gw2, gb, gs = B.expert_linear_backward(rows, self.h, self.w2, gy, pre=self.z, row_scale=self.buf.recv_weight, grad_bias=True,
                                                   grad_row_scale=True)
        gx_rows, gw1 = B.expert_gated_backward(rows, self.buf.recv_x, self.w1, self.pre, gh, act=self.act, x_scale=self.buf.recv_scale)
        gx = self.buf.combine(gx_rows, self.ones)
        e = self.idx.long().clamp(min=0)
        rank = e // (self.E // self.R)
        at = rank * self.cap + self.buf.slot_row[:self.T].long().clamp(min=0)
        gw = torch.where(self.idx >= 0, gs.view(-1)[at], 0.0)
        return gx, gw1, gw2, gb, B.route_backward(self.logits, self.idx, gw)

    def check_logits(self, got, want):
        """dl_j = w_j (s_j - sum_i w_i s_i) with s_j = <grad, z_j>: the differences may be much smaller than the s_j, which are off by what
        the roundings of h and z (two, and the sums') make of their products, at most 3 * 2^-8 |grad| |z_j|; twice that, at most,
        for a difference with an average of them."""
        e = self.idx.long().clamp(min=0)
        at = e // (self.E // self.R) * self.cap + self.buf.slot_row[:self.T].long().clamp(min=0)
        size = self.z.view(-1, self.H)[at].double().norm(dim=-1).amax(1) * self.grad.double().norm(dim=-1)
        off = (got.double() - want).abs().amax(1)
        assert bool((off <= 2 * 3 * HALF * size + 1e-12).all()), float((off / size).max())

    def exact(self, grad=False):
        x, logits, w1, w2, bias = (t.double().requires_grad_(grad) for t in (self.x, self.logits, self.w1, self.w2, self.bias))
        top = self.idx.long()
        v = torch.where(self.idx >= 0, logits.gather(1, top.clamp(min=0)), -float("inf"))
        w = torch.softmax(v, 1)
        out = torch.zeros((self.T, self.H), dtype=torch.float64, device="cuda")
        for e in range(self.E):
            t, j = (self.idx == e).nonzero(as_tuple=True)
            if t.numel() == 0:
                continue
            xe = x[t]
            g, u = xe @ w1[e, 0].T, xe @ w1[e, 1].T
            y = (act_exact(g, self.act)[0] * u) @ w2[e].T + bias[e]
            out = out.index_add(0, t, w[t, j][:, None] * y)
        if not grad:
            return out
        (out * self.grad.double()).sum().backward()
        return out.detach(), x.grad, w1.grad, w2.grad, bias.grad, logits.grad


SHAPES = [(1, 64, 32, 4, 2, 2), (77, 256, 136, 16, 4, 4), (500, 512, 264, 8, 2, 3)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_serving(shape, act):
    l = Layer(*shape, act=act)
    out = l.serve()
    assert l.buf.status() == 0
    near("out", out, l.exact(), 3)     # h, y, out


def test_serving_with_fp8_rows():
    l = Layer(300, 512, 264, 8, 2, 3, payload=1)
    out = l.serve()
    # the rows as the dispatch quantised them: the oracle of what the experts see
    want = torch.zeros((l.T, l.H), dtype=torch.float64, device="cuda")
    q = l.buf.recv_x.view(torch.float8_e4m3fn).float().double() * l.buf.recv_scale.double().repeat_interleave(128, dim=2)
    off, cnt, src = l.buf.expert_offset.tolist(), l.buf.num_tokens_per_expert.tolist(), l.buf.recv_src_idx
    for e in range(l.E):
        r = e // (l.E // l.R)
        rows = slice(off[e], off[e] + cnt[e])
        xe, t = q[r, rows], src[r, rows].long()
        y = (act_exact(xe @ l.w1[e, 0].double().T, "silu")[0] * (xe @ l.w1[e, 1].double().T)) @ l.w2[e].double().T + l.bias[e].double()
        want.index_add_(0, t, l.buf.recv_weight[r, rows].double()[:, None] * y)
    near("out", out, want, 3)
    assert l.buf.status() == 0


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_training(shape, act):
    l = Layer(*shape, seed=3, act=act)
    out = l.train_forward()
    gx, gw1, gw2, gb, gl = l.train_backward()
    assert l.buf.status() == 0 and l.gbuf.status() == 0
    want, wx, ww1, ww2, wb, wl = l.exact(grad=True)
    near("out", out, want, 3)
    for name, got, ref in (("x", gx, wx), ("w1", gw1, ww1), ("w2", gw2, ww2), ("bias", gb, wb)):
        near(name, got, ref, 6)
    l.check_logits(gl, wl)


def test_captured_layer_follows_its_inputs():
    l = Layer(200, 256, 136, 16, 4, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        l.train_forward()
        l.train_backward()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l.train_forward()
        grads = l.train_backward()
    for seed in (1, 2, 3):
        new = Layer(200, 256, 136, 16, 4, 4, seed=seed)
        for n in ("x", "logits", "w1", "w2", "grad", "bias"):
            getattr(l, n).copy_(getattr(new, n))
        graph.replay()
        out = new.train_forward()
        want = new.train_backward()
        assert torch.equal(l.out, out)
        for a, b in zip(grads, want):
            assert torch.equal(a, b)


def test_layers_on_their_own_streams():
    layers = [Layer(150 + 40 * i, 256, 136, 16, 4, 4, seed=i) for i in range(3)]
    want = [l.serve().clone() for l in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for l in layers:
        l.out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for l, s in zip(layers, streams):
            with torch.cuda.stream(s):
                l.serve()
    torch.cuda.synchronize()
    for l, w in zip(layers, want):
        assert torch.equal(l.out, w)


def test_a_stream_by_argument_keeps_its_scratch():
    # (the scratch of a call belongs to the stream it runs on, not to torch's current one)
    from test_gpu_experts import Rows, _fp8, _gen, _weights
    R = Rows("edges")
    gen = _gen(4)
    q, scale, _ = _fp8(R, gen, 512)
    w, pre, grad = _weights(gen, R.E, 2, 264, 512), R.randn(gen, 2, 264), R.randn(gen, 264)
    want = B.expert_gated_backward(R.rows, q, w, pre, grad, x_scale=scale)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(8):
        outs.append(B.expert_gated_backward(R.rows, q, w, pre, grad, x_scale=scale, stream=side))
        torch.full((R.R, R.cap, 2, 512), float("nan"), dtype=torch.bfloat16, device="cuda")   # would take freed scratch over
    side.synchronize()
    for gx, gw in outs:
        assert torch.equal(gx[R.mine], want[0][R.mine]) and torch.equal(gw, want[1])


def test_rows_dropped_at_capacity_are_left_out():
    l = Layer(300, 256, 136, 8, 2, 3, cap=200)
    l.y.zero_()
    l.serve()
    assert l.buf.status() == B.UBEP_ERR_CAPACITY
    assert bool(torch.isfinite(l.y.float()).all())
    # the segments that fit are whole
    off, cnt = l.buf.expert_offset.tolist(), l.buf.num_tokens_per_expert.tolist()
    r, e = 0, 0
    rows = slice(off[e], min(off[e] + cnt[e], 200))
    xe = l.buf.recv_x.view(torch.bfloat16)[r, rows].double()
    y = (act_exact(xe @ l.w1[e, 0].double().T, "silu")[0] * (xe @ l.w1[e, 1].double().T)) @ l.w2[e].double().T + l.bias[e].double()
    near("y", l.y[r, rows], y, 2)


def test_rows_per_token_and_rank_are_refused():
    buf = B.Buffer(num_ranks=2, num_experts=8, hidden=256, topk=2, max_tokens=16, rows_per_rank_cap=32, dedup=1)
    with pytest.raises(B.UbepError) as e:
        buf.expert_segments()
    assert e.value.code == B.UBEP_ERR_ARG


def test_no_tokens():
    l = Layer(8, 64, 32, 4, 2, 2)
    l.buf.dispatch(l.x[:0], l.idx[:0], l.w[:0])
    l.h.fill_(7.0)
    B.expert_gated(l.buf.expert_segments(), l.buf.recv_x, l.w1, out=l.h)
    assert bool((l.h == 7.0).all())
    gw = torch.full_like(l.w1, 7.0)
    B.expert_gated_backward(l.buf.expert_segments(), l.buf.recv_x, l.w1, l.pre, l.h, grad_x=False, grad_w=gw)
    assert bool((gw == 0).all()) and l.buf.status() == 0


def test_ranks_with_an_arena_each():
    # every rank's experts on its own region; the rows arrive as in the sharded dispatch
    T, H, I, E, R, k = 96, 256, 72, 8, 4, 2
    whole = Layer(T, H, I, E, R, k, seed=5)
    want = whole.serve().clone()
    L = E // R
    ranks = [B.Buffer(num_ranks=R, num_experts=E, hidden=H, topk=k, max_tokens=T, rows_per_rank_cap=whole.cap) for _ in range(R)]
    ptrs = [b.arena.data_ptr() for b in ranks]
    for r, b in enumerate(ranks):
        B.ubep_set_peers(b.handle, r, ptrs)
    for s, b in enumerate(ranks):
        B.ubep_dispatch_sharded(b.handle, whole.x[s * T // R:(s + 1) * T // R].contiguous(), whole.idx, whole.w, T)
    for r, b in enumerate(ranks):
        B.ubep_wait_arrivals(b.handle)
        rows = b.expert_segments()
        assert rows.offset.shape == (L,)
        w1, w2, bias = (t[r * L:(r + 1) * L] for t in (whole.w1, whole.w2, whole.bias))
        h = B.expert_gated(rows, b.recv_x[r:r + 1], w1)
        y = B.expert_linear(rows, h, w2, bias=bias)
        n = int(b.num_rows_per_rank[r])
        assert torch.equal(y[0, :n], whole.y[r, :n]) and b.status() == 0
    assert torch.equal(whole.out, want)


def test_offsets_beyond_32_bits():
    # rows whose elements lie past 2^31: read, written, and summed over
    H, cap = 8192, 270000
    x = torch.zeros((1, cap, H), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 70
    x[0, -n:] = torch.randn((n, H), generator=g, device="cuda").to(torch.bfloat16)
    rows = B.ExpertRows(torch.tensor([0, cap - n], dtype=torch.int32, device="cuda"), torch.tensor([3, n], dtype=torch.int32, device="cuda"))
    w = (torch.randn((2, 16, H), generator=g, device="cuda") * H ** -0.5).to(torch.bfloat16)
    y = B.expert_linear(rows, x, w)
    want = x[0, -n:].double() @ w[1].double().T
    near("y", y[0, -n:], want, 2)
    assert bool((y[0, :3] == 0).all())
    gy = torch.zeros((1, cap, 16), dtype=torch.bfloat16, device="cuda")
    gy[0, -n:] = torch.randn((n, 16), generator=g, device="cuda").to(torch.bfloat16)
    gx, gw, _, _ = B.expert_linear_backward(rows, x, w, gy, grad_x=torch.zeros_like(x))
    near("grad_x", gx[0, -n:], gy[0, -n:].double() @ w[1].double(), 2)
    near("grad_w", gw[1], gy[0, -n:].double().T @ x[0, -n:].double(), 2)
    assert bool((gx[0, 3:-n] == 0).all())
