"""Host-side checks of the router's and the experts' entry points: nothing here needs a GPU, every call is refused before it
would ask for one."""
import ctypes

import pytest

from paper_2607_06202_b200 import binding as B
from paper_2607_06202_b200 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return B.load()


P = 1 << 20      # an address that is never followed
ODD = P + 8


def _rows(**kw):
    r = B.ubep_expert_rows_t(P, P, 8, 2, 64, 0, None)
    for k, v in kw.items():
        setattr(r, k, v)
    return ctypes.byref(r)


def _gated(lib, rows=None, x=P, scale=None, w=P, H=128, I=64, act=1, h=P, pre=None, scratch=None):
    return lib.ubep_expert_gated(rows if rows is not None else _rows(), x, scale, w, H, I, act, h, pre, scratch, None)


BAD_ROWS = [dict(offset=None), dict(count=None), dict(num_experts=0), dict(num_ranks=0), dict(num_experts=7), dict(rows_per_rank_cap=0),
            dict(rows_per_rank_cap=2 ** 31 - 1), dict(num_experts=65536), dict(device=-1)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_rows_that_make_no_sense(lib, bad):
    assert _gated(lib, _rows(**bad)) == B.UBEP_ERR_ARG
    assert lib.ubep_expert_linear(_rows(**bad), P, P, None, None, None, 64, 64, 0, P, None, None) == B.UBEP_ERR_ARG


def test_gated_arguments(lib):
    for bad in (dict(x=None), dict(w=None), dict(h=None), dict(x=ODD), dict(pre=ODD), dict(H=4), dict(H=0), dict(I=12), dict(I=-8),
                dict(act=-1), dict(act=4), dict(H=136, scale=P, scratch=P), dict(scale=P), dict(scale=ODD, scratch=P),
                dict(H=1 << 21)):
        assert _gated(lib, **bad) == B.UBEP_ERR_ARG, bad
    assert lib.ubep_expert_gated(None, P, None, P, 128, 64, 1, P, None, None, None) == B.UBEP_ERR_ARG


def test_gated_backward_arguments(lib):
    def call(x=P, scale=None, w=P, pre=P, gh=P, H=128, I=64, act=1, gp=P, gx=P, gw=P, scratch=None):
        return lib.ubep_expert_gated_backward(_rows(), x, scale, w, pre, gh, H, I, act, gp, gx, gw, scratch, None)
    for bad in (dict(pre=None), dict(gh=None), dict(gp=None), dict(gx=None, gw=None), dict(w=None), dict(x=None), dict(scale=P),
                dict(gp=ODD), dict(act=9), dict(H=20)):
        assert call(**bad) == B.UBEP_ERR_ARG, bad


def test_linear_arguments(lib):
    def call(x=P, w=P, bias=None, scale=None, res=None, K=64, N=64, act=0, y=P, pre=None):
        return lib.ubep_expert_linear(_rows(), x, w, bias, scale, res, K, N, act, y, pre, None)
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(bias=ODD), dict(scale=ODD), dict(res=ODD), dict(K=12), dict(N=0),
                dict(act=7)):
        assert call(**bad) == B.UBEP_ERR_ARG, bad


def test_linear_backward_arguments(lib):
    def call(x=P, w=P, pre=P, scale=None, gy=P, K=64, N=64, act=1, gp=2 * P, gx=P, gw=P, gb=None, gs=None, scratch=None):
        return lib.ubep_expert_linear_backward(_rows(), x, w, pre, scale, gy, K, N, act, gp, gx, gw, gb, gs, scratch, None)
    for bad in (dict(gy=None), dict(pre=None), dict(gp=None), dict(gs=P), dict(w=None), dict(x=None), dict(gb=P),
                dict(gb=P, scratch=ODD), dict(scale=P, gs=P, N=16392),
                dict(gx=None, gw=None), dict(gx=ODD), dict(scale=P, act=0, pre=None)):
        assert call(**bad) == B.UBEP_ERR_ARG, bad


def test_route_arguments(lib):
    def call(l=P, t=0, T=4, E=16, k=2, idx=P, w=P):
        return lib.ubep_route(l, t, T, E, k, 1, idx, w, 0, None)
    for bad in (dict(l=None), dict(t=2), dict(T=-1), dict(E=0), dict(E=65536), dict(k=0), dict(k=33), dict(idx=None), dict(w=ODD)):
        assert call(**bad) == B.UBEP_ERR_ARG, bad
    assert call(T=0) == B.UBEP_OK
    assert lib.ubep_route_backward(P, 0, P, P, 4, 16, 2, 1, None, 0, None) == B.UBEP_ERR_ARG
    assert lib.ubep_route_backward(P, 0, P, P, 4, 16, 2, 1, P, 0, None) == B.UBEP_ERR_ARG      # the logits' own memory
    assert lib.ubep_route_backward(P, 0, P, P, 0, 16, 2, 1, None, 0, None) == B.UBEP_OK


def test_rows_of_no_buffer(lib):
    assert lib.ubep_expert_segments(None, _rows()) == B.UBEP_ERR_ARG


def test_tensors_on_the_host_are_refused(lib):
    import torch
    with pytest.raises(ValueError, match="not on a GPU"):
        B.route(torch.zeros((4, 8)), 2)
    with pytest.raises(ValueError, match="act"):
        B.expert_gated(B.ExpertRows(None, None), None, None, act="tanh")
    with pytest.raises(TypeError):
        B.expert_gated(B.ExpertRows(None, None), None, None)
