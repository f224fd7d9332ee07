"""The experts' calls where each CTA, or pair of CTAs, works on several tiles, with experts without rows in between; where their passes over
the rows take several turns or are split by columns; and the wide tiles of single CTAs.  The checks and their tolerances are those of
test_gpu_experts.py, on other segments and widths."""
import pytest
import torch

import test_gpu_experts as X
from paper_2607_06202_b200 import binding as B

pytestmark = pytest.mark.gpu


def _in_regions(counts, R, gap):
    """One expert after the other in its region, `gap` rows apart."""
    L, seg = len(counts) // R, []
    for r in range(R):
        at = r
        for n in counts[r * L:(r + 1) * L]:
            seg.append((at, n))
            at += n + gap
    return seg


PAIRS = [0 if i % 6 == 5 else (i * 53) % 271 for i in range(36)]
SINGLE = [0 if i % 6 == 5 else 100 if i == 22 else (i * 7) % 41 for i in range(40)]
SEGMENTS = {
    "pairs": (2, 2500, _in_regions(PAIRS, 2, 3)),      # 138 rows of capacity per expert, and more than 32 experts
    "single": (2, 600, _in_regions(SINGLE, 2, 1)),     # 30
    "narrow": (2, 570, _in_regions([0 if i == 7 else 90 if i % 2 else 10 for i in range(18)], 2, 0)),   # 63
}


@pytest.fixture
def many(monkeypatch):
    for name, s in SEGMENTS.items():
        assert all(0 <= o and o + n <= s[1] for o, n in s[2])
        monkeypatch.setitem(X.SEGMENTS, name, s)


def units(name):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return sms // 2 if name == "pairs" else sms


def row_tiles(name):
    most = 256 if name == "pairs" else 64
    return sum(-(-n // most) for _, n in SEGMENTS[name][2])


def tiles(name, features, span):
    return row_tiles(name) * -(-features // span)


def wide(name, features):
    """Features per tile of a product with one matrix per expert."""
    return 256 if name == "pairs" or len(SEGMENTS[name][2]) * -(-features // 128) > units(name) else 128


@pytest.mark.parametrize("name,H,I", [("pairs", 136, 1032), ("single", 136, 2056)])
def test_gated(many, name, H, I):
    assert tiles(name, I, 128) >= 3 * units(name)
    X.test_gated(name, H, I)


@pytest.mark.parametrize("name,H,I", [("pairs", 256, 1032), ("single", 256, 2056)])
def test_gated_takes_fp8_rows(many, name, H, I):
    assert tiles(name, I, 128) >= 3 * units(name)
    X.test_gated_takes_fp8_rows(name, H, I)


@pytest.mark.parametrize("name,K,N,span", [("pairs", 136, 2056, 256), ("single", 136, 3848, 256), ("narrow", 72, 1016, 128)])
def test_linear(many, name, K, N, span):
    assert wide(name, N) == span and tiles(name, N, span) >= (1.3 if name == "narrow" else 3) * units(name)
    X.test_linear(name, K, N)


# (the rows' gradient has the width of the rows as its features; the weights' gradient tiles of 256 x 256 of every expert)
@pytest.mark.parametrize("name,H,I", [("pairs", 2056, 72), ("pairs", 72, 1032), ("single", 72, 2056), ("single", 3848, 72)])
def test_gated_backward(many, name, H, I):
    E = len(SEGMENTS[name][2])
    assert E * -(-H // 256) * -(-2 * I // 256) >= 3 * units(name) or tiles(name, H, wide(name, H)) >= 3 * units(name)
    X.test_gated_backward(name, H, I)


@pytest.mark.parametrize("name,H,I", [("pairs", 2176, 72), ("pairs", 128, 1032), ("single", 128, 2056)])
def test_gated_backward_takes_fp8_rows(many, name, H, I):
    X.test_gated_backward_takes_fp8_rows(name, H, I)


@pytest.mark.parametrize("name,K,N,span", [("pairs", 2056, 136, 256), ("pairs", 136, 2056, 256), ("single", 3848, 72, 256),
                                           ("single", 72, 3848, 128)])
def test_linear_backward(many, name, K, N, span):
    E = len(SEGMENTS[name][2])
    assert wide(name, K) == span
    assert E * -(-K // 256) * -(-N // 256) >= 3 * units(name) and (K < N or tiles(name, K, span) >= 3 * units(name))
    X.test_linear_backward(name, K, N)


# (narrow tiles are taken where there is an SM for each: a second one comes from experts with more than 64 rows)
@pytest.mark.parametrize("K,N", [(1016, 72), (72, 1016)])
def test_linear_backward_in_narrow_tiles(many, K, N):
    assert wide("narrow", K) == 128 and (K < N or tiles("narrow", K, 128) >= 1.3 * units("narrow"))
    X.test_linear_backward("narrow", K, N)


# columns of a thread: 8 up to N = 2048, then 16, 32 and 64; without a row weight's gradient more than 8192 columns are split
@pytest.mark.parametrize("segments", ["small", "gaps_out_of_order", "nobody"])
@pytest.mark.parametrize("N", [2048, 2056, 4096, 4104, 8192, 8200, 16384])
def test_linear_backward_of_wide_rows(segments, N):
    X.test_linear_backward(segments, 8, N)


@pytest.mark.parametrize("N", [16392, 20000])
def test_bias_gradient_of_wider_rows(N):
    R = X.Rows("gaps_out_of_order")
    gen = X._gen(N)
    x, w = R.randn(gen, 8), X._weights(gen, R.E, N, 8)
    z, gy = R.randn(gen, N), R.randn(gen, N)
    out = torch.full((R.E, N), X.FILL, dtype=torch.bfloat16, device="cuda")
    B.expert_linear_backward(R.rows, x, w, gy, pre=z, act="relu", grad_x=False, grad_w=False, grad_bias=out)
    want, tol = torch.zeros((R.E, N), dtype=torch.float64, device="cuda"), torch.zeros((R.E, N), dtype=torch.float64, device="cuda")
    for e, r, a, b in R.each():
        d = gy[r, a:b].double() * (z[r, a:b] > 0)
        want[e], tol[e] = d.sum(0), (b - a + 4) * X.SUM * d.abs().sum(0)
    X.check_all("grad_bias", out, want, tol * (1 + X.HALF) + X.HALF * want.abs())


# widening: 1536 channels per turn of a warp; the gated gradient's pass: 2048 inner features per turn of a block
@pytest.mark.parametrize("segments", ["small", "edges"])
def test_passes_over_rows_in_several_turns(segments):
    X.test_gated_takes_fp8_rows(segments, 1664, 8)
    X.test_gated_takes_fp8_rows(segments, 4352, 8)
    X.test_gated_backward_takes_fp8_rows(segments, 1664, 8)
    X.test_gated_backward_takes_fp8_rows(segments, 3200, 8)
    X.test_gated_backward(segments, 8, 2056)
    X.test_gated_backward(segments, 8, 4104)
