"""Outputs in their inputs' place: where a dimension is one, its stride is no matter (one token
of [B, T, H, d] rows and of [B, H, T, d] ones is the same memory).  On the CPU the launch says
what it was given."""
import pytest
import torch

from paper_2608_23253_amd import _serve as V
from paper_2608_23253_amd import _step as S


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        for module in (S, V):
            monkeypatch.setattr(module, "_check", lambda *a, **k: None)
            monkeypatch.setattr(module, "_launch", lambda *a, **k: None)
    return request.param


CALLS = [S.norm_rotate, V.rotate_positions]


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_one_token_of_either_order(device, call):
    B, H, d = 3, 4, 64
    x = torch.randn(B, 1, H, d, generator=torch.Generator().manual_seed(0)).to(device)
    pos, plan = torch.full((1,), 5, dtype=torch.int32, device=device), V.rotary_plan(d)
    q = x.transpose(1, 2)
    want = call(q, None, pos, plan)[0]
    there = x.view(B, H, 1, d)
    assert there.stride() != q.stride()
    got = call(q, None, pos, plan, q_out=there)[0]
    assert got is there
    assert device == "cpu" or torch.equal(x.transpose(1, 2), want)


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_rows_that_lie_otherwise_are_refused(device, call):
    x = torch.randn(2, 3, 3, 64, device=device)
    pos, plan = torch.arange(3, dtype=torch.int32, device=device), V.rotary_plan(64)
    with pytest.raises(ValueError, match="strides"):
        call(x, None, pos, plan, q_out=x.transpose(1, 2))
    with pytest.raises(ValueError, match="strides"):
        call(None, x, pos, plan, k_out=x.transpose(1, 2))
