"""Tangents of forward-mode differentiation: the operators have no rule for them and say so,
where the launch would drop them.  On the CPU the launch does nothing."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2608_23253_amd import _serve as V
from paper_2608_23253_amd import _step as S


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        for module in (S, V):
            monkeypatch.setattr(module, "_check", lambda *a, **k: None)
            monkeypatch.setattr(module, "_launch", lambda *a, **k: None)
    return request.param


def norm_inputs(device):
    q, k = torch.randn(1, 2, 3, 64, device=device), torch.randn(1, 1, 3, 64, device=device)
    w = [torch.ones(64, device=device) for _ in range(2)]
    return [q, k, *w], torch.arange(3, dtype=torch.int32, device=device), V.rotary_plan(64)


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("leaf", [None, 0, 3])
def test_norm_rotate(device, which, leaf):
    x, pos, plan = norm_inputs(device)
    if leaf is not None:
        x[leaf].requires_grad_(True)
    with fwd.dual_level():
        x[which] = fwd.make_dual(x[which], torch.ones_like(x[which]))
        with pytest.raises(RuntimeError, match="forward-mode"):
            S.norm_rotate(x[0], x[1], pos, plan, x[2], x[3])


@pytest.mark.parametrize("which", range(6))
def test_norm_rotate_backward(device, which):
    x, pos, plan = norm_inputs(device)
    x += [torch.ones_like(t) for t in x[:2]]
    with fwd.dual_level():
        x[which] = fwd.make_dual(x[which], torch.ones_like(x[which]))
        with pytest.raises(RuntimeError, match="forward-mode"):
            S.norm_rotate_backward(x[4], x[5], x[0], x[1], pos, plan, x[2], x[3])


@pytest.mark.parametrize("which", range(2))
def test_rotate_positions(device, which):
    x, pos, plan = norm_inputs(device)
    with fwd.dual_level():
        x[which] = fwd.make_dual(x[which], torch.ones_like(x[which]))
        with pytest.raises(RuntimeError, match="forward-mode"):
            V.rotate_positions(x[0], x[1], pos, plan)


def test_what_has_no_tangent_goes_through(device):
    """Within a dual level, too; and a tangent that the call does not take is no matter."""
    x, pos, plan = norm_inputs(device)
    with fwd.dual_level():
        fwd.make_dual(x[0], torch.ones_like(x[0]))
        for call in (S.norm_rotate, V.rotate_positions):
            y = call(x[0], x[1], pos, plan)
            assert y[0].shape == x[0].shape and y[1].shape == x[1].shape


@pytest.mark.gpu
@pytest.mark.parametrize("make,attend", [(S.PagedCache4, S.cache4_attend),
                                         (V.PagedCache, V.cache_attend)])
def test_attention(make, attend):
    cache = make(2, 1, 64)
    pages, lengths = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([[0]], [3]))
    q = torch.randn(1, 2, 1, 64, device="cuda").bfloat16()
    attend(q, cache, pages, lengths)
    with fwd.dual_level():
        attend(q, cache, pages, lengths)
        with pytest.raises(RuntimeError, match="forward-mode"):
            attend(fwd.make_dual(q, torch.ones_like(q)), cache, pages, lengths)
