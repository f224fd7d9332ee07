"""Calls on a stream given by argument: what they allocate belongs to that stream, not to torch's current one.

The allocator hands a block out again as soon as it is given back; what the stream it was given back on still does with it is not over
by then.  Here the current stream has a queue of products in front of a fill of the block, which is given back at once."""
import pytest
import torch

from paper_2607_06202_b200 import binding as B
from test_gpu_experts import Rows, _fp8, _gen, _weights

pytestmark = pytest.mark.gpu


def behind_a_queue(shape, dtype, fill):
    """Leaves the current stream with some tens of milliseconds of products and a fill of a block behind them, given back already."""
    a = torch.ones((8192, 8192), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(a)
    for _ in range(60):
        torch.mm(a, a, out=out)
    block = torch.full(shape, fill, dtype=dtype, device="cuda")
    done = torch.cuda.Event()
    done.record()
    del block
    return done


def pool_of(stream):
    """Bytes the allocator holds for a stream."""
    return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)


def a_side_stream():
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    assert side.cuda_stream != torch.cuda.current_stream().cuda_stream and pool_of(side) == 0
    return side


def test_outputs_belong_to_the_call_s_stream():
    R = Rows("edges")
    gen = _gen(4)
    x, w = R.randn(gen, 512), _weights(gen, R.E, 1024, 512)
    want = B.expert_linear(R.rows, x, w)
    side = a_side_stream()
    done = behind_a_queue(want.shape, torch.bfloat16, float("nan"))
    got = B.expert_linear(R.rows, x, w, stream=side)
    side.synchronize()
    assert not done.query()                  # the fill comes after the call's kernels
    torch.cuda.synchronize()
    assert torch.equal(got[R.mine], want[R.mine])


def test_scratch_belongs_to_the_call_s_stream():
    R = Rows("edges")
    gen = _gen(5)
    H, I, N = 512, 264, 1024
    q, scale, _ = _fp8(R, gen, H)
    w, w3 = _weights(gen, R.E, 2, I, H), _weights(gen, R.E, N, H)
    x, pre, gh, z, gy = R.randn(gen, H), R.randn(gen, 2, I), R.randn(gen, I), R.randn(gen, N), R.randn(gen, N)
    h, gx, gw = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((R.R, R.cap, I), (R.R, R.cap, H), w.shape))
    gw3, gb = torch.empty_like(w3), torch.empty((R.E, N), dtype=torch.bfloat16, device="cuda")
    rows = R.R * R.cap
    for name, scratch, call in (
            ("gated of FP8 rows", rows * H * 2, lambda s: B.expert_gated(R.rows, q, w, x_scale=scale, out=h, stream=s)),
            ("gated backward of FP8 rows", 2 * rows * H * 2 + rows * 2 * I * 2,
             lambda s: B.expert_gated_backward(R.rows, q, w, pre, gh, x_scale=scale, grad_x=gx, grad_w=gw, stream=s)),
            ("linear backward", rows * N * 2 + 1024 * N * 4,
             lambda s: B.expert_linear_backward(R.rows, x, w3, gy, pre=z, act="silu", grad_x=gx, grad_w=gw3, grad_bias=gb, stream=s))):
        call(None)
        want = [t.clone() for t in (h, gx, gw, gw3, gb)]
        side = a_side_stream()
        behind_a_queue((scratch // 2,), torch.bfloat16, float("nan"))
        call(side)
        assert pool_of(side) >= scratch, name
        torch.cuda.synchronize()
        for t, v in zip((h, gx, gw, gw3, gb), want):
            bits = lambda u: u.view(torch.int16)  # noqa: E731
            assert torch.equal(bits(t), bits(v)), name


def test_the_default_stream_by_its_handles():
    R = Rows("small")
    gen = _gen(6)
    q, scale, _ = _fp8(R, gen, 128)
    w = _weights(gen, R.E, 2, 72, 128)
    want = B.expert_gated(R.rows, q, w, x_scale=scale)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for handle in (0, 1):                    # the legacy default stream and its other name
        with torch.cuda.stream(side):
            got = B.expert_gated(R.rows, q, w, x_scale=scale, stream=handle)
        torch.cuda.synchronize()
        assert torch.equal(got[R.mine], want[R.mine])


def test_captured_with_a_stream_by_argument():
    # a side stream that joined the capture: its memory belongs to the graph
    R = Rows("edges")
    gen = _gen(7)
    q, scale, _ = _fp8(R, gen, 256)
    w = _weights(gen, R.E, 2, 72, 256)
    want = B.expert_gated(R.rows, q, w, x_scale=scale)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = B.expert_gated(R.rows, q, w, x_scale=scale, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for _ in range(2):
        got.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[R.mine], want[R.mine])


def test_combine_and_layout_allocate_on_the_call_s_stream():
    T, H, E, R, k = 2048, 2048, 64, 8, 4
    gen = _gen(8)
    x = torch.randn((T, H), generator=gen, device="cuda").to(torch.bfloat16)
    idx, w = B.route(torch.randn((T, E), generator=gen, device="cuda"), k)
    buf = B.Buffer(num_ranks=R, num_experts=E, hidden=H, topk=k, max_tokens=T, rows_per_rank_cap=T * k)
    buf.dispatch(x, idx, w)
    y = buf.recv_x.view(torch.bfloat16)
    layout, out = buf.get_dispatch_layout(idx), buf.combine(y, w)
    side = a_side_stream()
    done = behind_a_queue(out.shape, torch.bfloat16, float("nan"))
    got = buf.combine(y, w, stream=side)
    side.synchronize()
    assert not done.query()                  # the fill comes after the call's kernels
    torch.cuda.synchronize()
    assert torch.equal(got, out)
    side = a_side_stream()
    behind_a_queue((T, R), torch.uint8, 9)
    parts = buf.get_dispatch_layout(idx, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(parts, layout):
        assert torch.equal(a, b)
