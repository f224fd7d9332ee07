"""The operators of a mixture-of-experts layer around dispatch and combine, as cases to time: the router
(top-k of the gate's logits, with its gradient), the experts' gated feed-forward block and the experts' matrix
product with bias, activation, row weight and residual in its epilogue, both with their backward passes.

Rows are laid out like receive regions, [R, cap, .]: expert e of rank e // L owns the rows offset[e] .. offset[e] +
count[e] - 1 of its rank's region.  Inputs are synthetic and made on the GPU from a seed: Gaussian activations and
gradients, weights scaled by the root of their length, routing as a top-k over Gaussian logits with a popularity
that belongs to the model.
"""
from __future__ import annotations

import torch

own = False

# ------------------------------------------------------------------------------------- cases

# hidden size, inner size, experts, ranks, top-k.  Hidden sizes, experts per rank and top-k of the benchmark's shapes (some of their
# ranks), inner sizes generic; the last is the toy shape.
FAMILIES = (
    (7168, 2048, 32, 4, 8),
    (4096, 2048, 16, 2, 8),
    (5120, 1536, 20, 2, 8),
    (2048, 1408, 32, 2, 4),
    (1024, 712, 16, 4, 4),
    (256, 512, 16, 4, 2),
)
ACTS = ("none", "silu", "gelu", "relu")


def _route(T, E, k, **kw):
    return dict(dict(op="route", T=T, E=E, k=k, renorm=True, dtype="float32", masked=0.0), **kw)


def _gated(T, family, **kw):
    H, I, E, R, k = family
    return dict(dict(op="gated", T=T, H=H, I=I, E=E, R=R, k=k, act="silu", fp8=False, save=False, tilt=0.0), **kw)


def _linear(T, family, **kw):
    H, I, E, R, k = family
    return dict(dict(op="linear", T=T, K=I, N=H, E=E, R=R, k=k, act="none", bias=False, scale=True, residual=False,
                     save=False, tilt=0.0), **kw)


def listed():
    f = FAMILIES
    return [
        # The toy layer's router: latency and launches alone.
        dict(_route(128, 16, 2), name="route_tiny"),
        # Router of the largest batch the benchmark dispatches, as the gate's product leaves its logits in bf16 (many ties).
        dict(_route(16384, 256, 8, dtype="bfloat16"), name="route_prefill"),
        # Training step of a router whose weights are probabilities over all experts, some of them switched off.
        dict(_route(8192, 128, 8, op="route_backward", renorm=False, masked=0.05), name="route_backward"),
        # The toy layer's experts.
        dict(_gated(128, f[5]), name="gated_tiny"),
        # Decode: sixteen rows per expert, every weight read once.
        dict(_gated(64, f[0]), name="gated_decode"),
        # Prefill: a thousand rows per expert, as an FP8 dispatch delivers them.
        dict(_gated(4096, f[0], fp8=True), name="gated_prefill_fp8"),
        # Forward pass of training at ragged sizes: popular and empty experts, an inner size that is no multiple of a tile.
        dict(_gated(1537, f[3], act="gelu", save=True, tilt=1.5), name="gated_train"),
        # Backward pass of the gated block on a training batch.
        dict(_gated(3000, f[1], op="gated_backward"), name="gated_backward"),
        # The toy layer's second product with everything its epilogue can do.
        dict(_linear(128, f[5], act="relu", bias=True, residual=True), name="linear_tiny"),
        # Decode: the down projection with the router's weight of every row.
        dict(_linear(64, f[0]), name="linear_decode"),
        # A prefill chunk through a product with bias, activation and residual.
        dict(_linear(3000, f[2], act="gelu", bias=True, scale=False, residual=True), name="linear_prefill"),
        # Backward pass of the down projection, the gradient of the rows' weights and of the bias among it.
        dict(_linear(3000, f[1], op="linear_backward", act="silu", bias=True), name="linear_backward"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("route", "route_backward", "gated", "gated", "gated_backward", "linear", "linear", "linear_backward"))
    if op.startswith("route"):
        E = rng.choice((8, 16, 60, 128, 160, 256, 288, 1000))
        return _route(_log_int(rng, 1, 16384), E, rng.choice((1, 2, 4, 6, 8)), op=op, renorm=rng.random() < 0.5,
                      dtype=rng.choice(("float32", "bfloat16")), masked=rng.choice((0.0, 0.0, 0.3)))
    family = rng.choice(FAMILIES)
    T = _log_int(rng, 1, 4096)
    tilt = rng.choice((0.0, 0.0, 1.0))
    if op.startswith("gated"):
        c = _gated(T, family, op=op, act=rng.choice(("silu", "gelu", "relu")), tilt=tilt)
        if op == "gated":
            c["save"] = rng.random() < 0.5
        c["fp8"] = family[0] % 128 == 0 and rng.random() < 0.4
    else:
        c = _linear(T, family, op=op, act=rng.choice(ACTS), bias=rng.random() < 0.5, scale=rng.random() < 0.6, tilt=tilt)
        if op == "linear":
            c["residual"], c["save"] = rng.random() < 0.4, rng.random() < 0.4
    # never more than the largest listed case
    most = work(_gated(4096, FAMILIES[0], fp8=True))["flops"]
    while work(c)["flops"] > most:
        c["T"] = c["T"] * 3 // 4
    return c


# ------------------------------------------------------------------------------------- inputs

class _State:
    pass


def _popularity(E, tilt, dev):
    """What the model's experts are chosen by beside the token; the last of them is switched off where they differ."""
    p = tilt * torch.sin(2.4 * torch.arange(E, device=dev, dtype=torch.float32))
    if tilt:
        p[-1] = -float("inf")
    return p


def _segments(case, gen, dev):
    T, E, R, k = (case[n] for n in ("T", "E", "R", "k"))
    L = E // R
    scores = torch.randn((T, E), generator=gen, device=dev) + _popularity(E, case["tilt"], dev)
    count = torch.bincount(scores.topk(k, dim=1).indices.reshape(-1), minlength=E)
    per_rank = count.view(R, L)
    offset = per_rank.cumsum(1) - per_rank
    return count.to(torch.int32), offset.reshape(E).to(torch.int32), per_rank


def _capacity(case, dev):
    """Rows a region holds and the most rows an expert's segment has, sized once from a batch of the same kind with room for the
    spread between batches (eight standard deviations)."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(23)
    count, _, per_rank = _segments(case, gen, dev)
    room = lambda n, most: int(min(most, n + 8 * n ** 0.5 + 16))  # noqa: E731
    cap = (room(int(per_rank.sum(1).max()), case["T"] * case["k"]) + 127) // 128 * 128
    return cap, min(cap, room(int(count.max()), case["T"]))


def _randn(gen, dev, *shape, scale=1.0):
    return torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16).mul_(scale)


def prepare(case, seed):
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    s = _State()
    s.case = dict(case)
    op = case["op"]
    if op.startswith("route"):
        T, E, k = case["T"], case["E"], case["k"]
        dtype = getattr(torch, case["dtype"])
        s.logits = torch.randn((T, E), generator=gen, device=dev).to(dtype)
        if case["masked"]:
            s.logits[torch.rand((T, E), generator=gen, device=dev) < case["masked"]] = -float("inf")
        if op == "route_backward":
            s.idx, s.w = _route_plain(s.logits, k, case["renorm"])
            s.grad_w = torch.randn((T, k), generator=gen, device=dev)
            s.grad_logits = torch.empty_like(s.logits)
        else:
            s.idx = torch.empty((T, k), dtype=torch.int32, device=dev)
            s.w = torch.empty((T, k), dtype=torch.float32, device=dev)
        torch.cuda.synchronize()
        return s
    E, R = case["E"], case["R"]
    s.cap, s.most = _capacity(case, dev)
    s.count, s.offset, per_rank = _segments(case, gen, dev)
    assert int(per_rank.sum(1).max()) <= s.cap and int(s.count.max()) <= s.most
    s.x_scale = s.pre = s.bias = s.scale = s.residual = None
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=dev)  # noqa: E731
    if op.startswith("gated"):
        H, I = case["H"], case["I"]
        s.x = _randn(gen, dev, R, s.cap, H)
        if case["fp8"]:   # as dispatch delivers them: e4m3 with one scale per 128 channels
            groups = s.x.view(R, s.cap, H // 128, 128).float()
            s.x_scale = groups.abs().amax(-1).clamp_(min=1e-4) / 448.0
            s.x = (groups / s.x_scale[..., None]).view(R, s.cap, H).to(torch.float8_e4m3fn)
        s.w = _randn(gen, dev, E, 2, I, H, scale=H ** -0.5)
        if op == "gated":
            s.out = zeros(R, s.cap, I)
            s.pre = zeros(R, s.cap, 2, I) if case["save"] else None
        else:
            s.pre = _randn(gen, dev, R, s.cap, 2, I)
            s.grad = _randn(gen, dev, R, s.cap, I)
            s.grad_x, s.grad_w = zeros(R, s.cap, H), torch.empty_like(s.w)
    else:
        K, N = case["K"], case["N"]
        s.x = _randn(gen, dev, R, s.cap, K)
        s.w = _randn(gen, dev, E, N, K, scale=K ** -0.5)
        if case["bias"]:
            s.bias = _randn(gen, dev, E, N, scale=0.1)
        if case["scale"]:
            s.scale = torch.rand((R, s.cap), generator=gen, device=dev)
        if op == "linear":
            if case["residual"]:
                s.residual = _randn(gen, dev, R, s.cap, N)
            s.out = zeros(R, s.cap, N)
            s.pre = zeros(R, s.cap, N) if case["save"] else None
        else:
            if case["act"] != "none" or case["scale"]:
                s.pre = _randn(gen, dev, R, s.cap, N)
            s.grad = _randn(gen, dev, R, s.cap, N)
            s.grad_x, s.grad_w = zeros(R, s.cap, K), torch.empty_like(s.w)
            s.grad_bias = torch.empty_like(s.bias) if case["bias"] else None
            s.grad_scale = torch.zeros((R, s.cap), device=dev) if case["scale"] else None
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------- plain forms

def _route_plain(logits, k, renorm):
    l = logits.float()
    l = torch.where(l.isnan(), -float("inf"), l)
    top, order = torch.sort(l, dim=1, descending=True, stable=True)
    top, idx = top[:, :k], order[:, :k]
    if top.shape[1] < k:
        top = torch.nn.functional.pad(top, (0, k - top.shape[1]), value=-float("inf"))
        idx = torch.nn.functional.pad(idx, (0, k - idx.shape[1]))
    used = top > -float("inf")
    most = torch.where(used[:, :1], top[:, :1], 0.0)
    e = torch.exp(top - most)
    total = e.sum(1, keepdim=True) if renorm else torch.exp(l - most).sum(1, keepdim=True)
    w = torch.where(used, e / torch.where(used[:, :1], total, 1.0), 0.0)
    return torch.where(used, idx, -1).to(torch.int32), w


def _route_backward_plain(logits, idx, grad_w, renorm):
    l = logits.float()
    l = torch.where(l.isnan(), -float("inf"), l)
    used = idx >= 0
    at = idx.clamp(min=0).long()
    g = torch.zeros_like(l).scatter_add_(1, at, torch.where(used, grad_w, 0.0))
    chosen = torch.zeros_like(l).scatter_add_(1, at, used.float()) > 0
    if renorm:
        l = torch.where(chosen, l, -float("inf"))
    most = l.amax(1, keepdim=True)
    e = torch.exp(l - torch.where(most > -float("inf"), most, 0.0))
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    return (p * (g - (p * g).sum(1, keepdim=True))).to(logits.dtype)


def _act(z, name):
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    return z.clamp(min=0.0) if name == "relu" else z


def _act_grad(z, name):
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    return (z > 0).to(z.dtype) if name == "relu" else torch.ones_like(z)


def _places(s):
    """For every expert the rows of its segment in [R * cap] and which of them exist; experts padded to the same length."""
    E, R = s.case["E"], s.case["R"]
    i = torch.arange(s.most, device=s.count.device)
    first = s.offset.long() + torch.arange(E, device=s.count.device) // (E // R) * s.cap
    exists = i[None, :] < s.count[:, None]
    return torch.where(exists, first[:, None] + i[None, :], 0), exists


def _taken(t, at, exists):
    """The experts' rows in 32 bits, zero where there are none: [E, most, width]."""
    rows = t.reshape(t.shape[0] * t.shape[1], -1)[at].float()
    return torch.where(exists[..., None], rows, 0.0)


def _rows_of(s, at, exists):
    rows = _taken(s.x, at, exists)
    if s.x_scale is None:
        return rows
    scale = _taken(s.x_scale, at, exists)
    return (rows.view(*scale.shape, 128) * scale[..., None]).view(rows.shape)


def _put(out, values, at, exists):
    """The experts' rows back to their places in an array like `out`; the other rows are zero."""
    n = out.shape[0] * out.shape[1]
    flat = torch.zeros((n + 1, values.shape[-1]), dtype=out.dtype, device=out.device)
    flat[torch.where(exists, at, n)] = values.to(out.dtype)   # (what does not exist goes to a row of its own)
    return flat[:n].view(out.shape)


def _gated_plain(s):
    at, exists = _places(s)
    x = _rows_of(s, at, exists)
    g = torch.bmm(x, s.w[:, 0].float().transpose(1, 2))
    u = torch.bmm(x, s.w[:, 1].float().transpose(1, 2))
    out = _put(s.out, _act(g, s.case["act"]) * u, at, exists)
    if s.pre is None:
        return {"out": out}
    return {"out": out, "pre": _put(s.pre, torch.cat((g, u), -1), at, exists)}


def _gated_backward_plain(s):
    at, exists = _places(s)
    x = _rows_of(s, at, exists)
    I = s.case["I"]
    pre = _taken(s.pre, at, exists)
    g, u, grad = pre[..., :I], pre[..., I:], _taken(s.grad, at, exists)
    d = torch.cat((grad * u * _act_grad(g, s.case["act"]), grad * _act(g, s.case["act"])), -1)
    w = s.w.float().view(s.w.shape[0], -1, s.w.shape[-1])
    grad_w = torch.bmm(d.transpose(1, 2), x).to(s.w.dtype).view(s.w.shape)
    return {"grad_x": _put(s.grad_x, torch.bmm(d, w), at, exists), "grad_w": grad_w}


def _linear_plain(s):
    at, exists = _places(s)
    z = torch.bmm(_rows_of(s, at, exists), s.w.float().transpose(1, 2))
    if s.bias is not None:
        z = z + s.bias.float()[:, None]
    y = _act(z, s.case["act"])
    if s.scale is not None:
        y = y * _taken(s.scale, at, exists)
    if s.residual is not None:
        y = y + _taken(s.residual, at, exists)
    out = _put(s.out, y, at, exists)
    return {"out": out} if s.pre is None else {"out": out, "pre": _put(s.pre, z, at, exists)}


def _linear_backward_plain(s):
    at, exists = _places(s)
    act = s.case["act"]
    d = grad = _taken(s.grad, at, exists)
    z = None if s.pre is None else _taken(s.pre, at, exists)
    if act != "none":
        d = d * _act_grad(z, act)
    if s.scale is not None:
        d = d * _taken(s.scale, at, exists)
    got = {"grad_x": _put(s.grad_x, torch.bmm(d, s.w.float()), at, exists),
           "grad_w": torch.bmm(d.transpose(1, 2), _rows_of(s, at, exists)).to(s.w.dtype)}
    if s.bias is not None:
        got["grad_bias"] = d.sum(1).to(s.bias.dtype)
    if s.scale is not None:
        got["grad_scale"] = _put(s.grad_scale, (grad * _act(z, act)).sum(-1, keepdim=True), at, exists)
    return got


# ------------------------------------------------------------------------------------- one pass

def _run_own(s):
    from paper_2607_06202_b200 import binding as B
    c = s.case
    op = c["op"]
    if op == "route":
        idx, w = B.route(s.logits, c["k"], renormalize=c["renorm"], topk_idx=s.idx, topk_w=s.w)
        return {"idx": idx, "w": w}
    if op == "route_backward":
        return {"grad_logits": B.route_backward(s.logits, s.idx, s.grad_w, renormalize=c["renorm"], grad_logits=s.grad_logits)}
    rows = B.ExpertRows(s.offset, s.count)
    if op == "gated":
        out = B.expert_gated(rows, s.x, s.w, act=c["act"], x_scale=s.x_scale, out=s.out, pre=s.pre)
        return {"out": out} if s.pre is None else {"out": out, "pre": s.pre}
    if op == "gated_backward":
        grad_x, grad_w = B.expert_gated_backward(rows, s.x, s.w, s.pre, s.grad, act=c["act"], x_scale=s.x_scale,
                                                 grad_x=s.grad_x, grad_w=s.grad_w)
        return {"grad_x": grad_x, "grad_w": grad_w}
    if op == "linear":
        out = B.expert_linear(rows, s.x, s.w, bias=s.bias, row_scale=s.scale, residual=s.residual, act=c["act"],
                              out=s.out, pre=s.pre)
        return {"out": out} if s.pre is None else {"out": out, "pre": s.pre}
    grad_x, grad_w, grad_bias, grad_scale = B.expert_linear_backward(
        rows, s.x, s.w, s.grad, pre=s.pre, row_scale=s.scale, act=c["act"], grad_x=s.grad_x, grad_w=s.grad_w,
        grad_bias=s.grad_bias, grad_row_scale=s.grad_scale)
    got = {"grad_x": grad_x, "grad_w": grad_w}
    if s.bias is not None:
        got["grad_bias"] = grad_bias
    if s.scale is not None:
        got["grad_scale"] = grad_scale
    return got


def run(s):
    if own:
        return _run_own(s)
    c = s.case
    op = c["op"]
    if op == "route":
        idx, w = _route_plain(s.logits, c["k"], c["renorm"])
        return {"idx": idx, "w": w}
    if op == "route_backward":
        return {"grad_logits": _route_backward_plain(s.logits, s.idx, s.grad_w, c["renorm"])}
    if op == "gated":
        return _gated_plain(s)
    if op == "gated_backward":
        return _gated_backward_plain(s)
    return _linear_plain(s) if op == "linear" else _linear_backward_plain(s)


# ------------------------------------------------------------------------------------- bounds

def work(case):
    op = case["op"]
    T, k, E = case["T"], case["k"], case["E"]
    if op.startswith("route"):
        logits = T * E * (4.0 if case["dtype"] == "float32" else 2.0)
        if op == "route":
            return {"bytes": logits + 8.0 * T * k, "flops": 3.0 * T * E}
        return {"bytes": 2 * logits + 8.0 * T * k, "flops": 6.0 * T * E}
    rows = float(T * k)
    used = E * (1.0 - (1.0 - 1.0 / E) ** rows)   # experts that have rows: only their weights are read
    if op.startswith("gated"):
        H, I = case["H"], case["I"]
        x = rows * (H + 4.0 * (H // 128) if case["fp8"] else 2.0 * H)
        w = 4.0 * I * H
        if op == "gated":
            return {"bytes": x + used * w + rows * I * (6.0 if case["save"] else 2.0), "flops": 4.0 * rows * H * I}
        return {"bytes": x + used * w + rows * 6.0 * I + rows * 2.0 * H + E * w, "flops": 8.0 * rows * H * I}
    K, N = case["K"], case["N"]
    x, y, w = rows * 2.0 * K, rows * 2.0 * N, 2.0 * N * K
    extra = (2.0 * E * N if case["bias"] else 0.0) + (4.0 * rows if case["scale"] else 0.0)
    if op == "linear":
        return {"bytes": x + used * w + y * (1 + case["save"] + case["residual"]) + extra, "flops": 2.0 * rows * K * N}
    saved = y if case["act"] != "none" or case["scale"] else 0.0
    return {"bytes": 2 * x + used * w + y + saved + E * w + 2 * extra, "flops": 4.0 * rows * K * N}


# ------------------------------------------------------------------------------------- in 64 bits

def _exact_act(z, name):
    """The activation and its derivative."""
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    if name == "gelu":
        c = torch.special.ndtr(z)
        return z * c, c + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    if name == "relu":
        return torch.relu(z), (z > 0).double()
    return z, torch.ones_like(z)


def _exact_route(s):
    c = s.case
    l = s.logits.double()
    if c["op"] == "route":
        # the order of the kept values decides: pairs (-logit, id) sorted one after the other
        l32 = s.logits.float()
        by_id = torch.argsort(-l32, dim=1, stable=True)[:, :c["k"]]
        if by_id.shape[1] < c["k"]:
            return None
        idx = torch.where(torch.gather(l32, 1, by_id) == -float("inf"), -1, by_id)
    else:
        idx = s.idx.long()
    used = idx >= 0
    got = torch.where(used, torch.gather(l, 1, idx.clamp(min=0)), -float("inf"))
    base = torch.logsumexp(got if c["renorm"] else l, 1, keepdim=True)
    w = torch.where(used, torch.exp(got - torch.where(base.isinf(), 0.0, base)), 0.0)
    if c["op"] == "route":
        return {"idx": idx.to(torch.int32), "w": w}
    mean = torch.where(used, w * s.grad_w.double(), 0.0).sum(1, keepdim=True)
    if c["renorm"]:
        grad = torch.zeros_like(l)
    else:
        grad = -torch.exp(l - torch.where(base.isinf(), 0.0, base)) * mean
    chosen = torch.where(used, w * (s.grad_w.double() - (mean if c["renorm"] else 0.0)), 0.0)
    return {"grad_logits": grad.scatter_add_(1, idx.clamp(min=0), chosen)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("route"):
        return _exact_route(s)
    E, R, act = case["E"], case["R"], case["act"]
    L = E // R
    counts, offsets = s.count.tolist(), s.offset.tolist()
    f64 = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    if op in ("gated", "linear"):
        got = {"out": f64(s.out)}
        if s.pre is not None:
            got["pre"] = f64(s.pre)
    else:
        got = {"grad_x": f64(s.grad_x), "grad_w": f64(s.grad_w)}
        if op == "linear_backward" and s.bias is not None:
            got["grad_bias"] = f64(s.bias)
        if op == "linear_backward" and s.scale is not None:
            got["grad_scale"] = f64(s.scale)
    for e in range(E):
        r, a, b = e // L, offsets[e], offsets[e] + counts[e]
        if a == b:
            continue
        x = s.x[r, a:b].double()
        if s.x_scale is not None:
            x = x * s.x_scale[r, a:b].double().repeat_interleave(128, dim=1)
        w = s.w[e].double()
        if op == "gated":
            g, u = x @ w[0].T, x @ w[1].T
            got["out"][r, a:b] = _exact_act(g, act)[0] * u
            if s.pre is not None:
                got["pre"][r, a:b, 0], got["pre"][r, a:b, 1] = g, u
        elif op == "gated_backward":
            g, u, grad = s.pre[r, a:b, 0].double(), s.pre[r, a:b, 1].double(), s.grad[r, a:b].double()
            value, slope = _exact_act(g, act)
            dg, du = grad * u * slope, grad * value
            got["grad_x"][r, a:b] = dg @ w[0] + du @ w[1]
            got["grad_w"][e, 0], got["grad_w"][e, 1] = dg.T @ x, du.T @ x
        elif op == "linear":
            z = x @ w.T
            if s.bias is not None:
                z = z + s.bias[e].double()
            y = _exact_act(z, act)[0]
            if s.scale is not None:
                y = y * s.scale[r, a:b, None].double()
            if s.residual is not None:
                y = y + s.residual[r, a:b].double()
            got["out"][r, a:b] = y
            if s.pre is not None:
                got["pre"][r, a:b] = z
        else:
            grad = s.grad[r, a:b].double()
            d = grad
            if s.pre is not None:
                value, slope = _exact_act(s.pre[r, a:b].double(), act)
                d = grad * slope
            if s.scale is not None:
                d = d * s.scale[r, a:b, None].double()
                got["grad_scale"][r, a:b] = (grad * value).sum(1)
            got["grad_x"][r, a:b], got["grad_w"][e] = d @ w, d.T @ x
            if s.bias is not None:
                got["grad_bias"][e] = d.sum(0)
    return got
