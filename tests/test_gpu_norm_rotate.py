"""norm_rotate and its backward pass against the formula in float64, and against
differences."""
import numpy as np
import pytest
import torch

import _serve_helpers as R
import _step_helpers as H
import paper_2608_23253_amd as E

pytestmark = pytest.mark.gpu


def rows(g, shape, dtype, order, scale=1.0):
    B, heads, T, d = shape
    x = torch.randn(B, heads, T, d, generator=g, dtype=torch.float64) * scale
    x = x.to(dtype)
    if order == "token":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    if order == "wide":                               # rows of a wider buffer, at an odd offset
        big = torch.zeros(B, heads, T, d + 3, dtype=dtype, device="cuda")
        big[..., 1:d + 1] = x.cuda()
        return big[..., 1:d + 1]
    return x.cuda()


CASES = [
    # d, rot, layout, axes, dtype, weight, order, B, H, Hkv, T
    (128, 128, "half", 1, "bf16", "own", "token", 2, 4, 2, 5),
    (128, 128, "half", 3, "f16", "f32", "head", 1, 28, 4, 1),
    (128, 64, "interleaved", 1, "f32", "own", "head", 3, 12, 2, 37),
    (64, 64, "half", 1, "bf16", "none", "token", 2, 3, 1, 33),
    (256, 64, "half", 1, "bf16", "f32", "token", 1, 2, 2, 9),
    (80, 80, "half", 1, "f16", "own", "head", 2, 3, 1, 7),
    (96, 24, "interleaved", 3, "f32", "f32", "token", 1, 5, 5, 13),
    (72, 36, "half", 1, "bf16", "own", "token", 1, 3, 2, 4),
    (256, 256, "interleaved", 1, "f32", "own", "wide", 1, 2, 1, 3),
    (255, 254, "half", 1, "bf16", "f32", "wide", 1, 2, 1, 5),
    (2, 2, "half", 1, "f32", "own", "head", 2, 1, 1, 3),
    (34, 2, "interleaved", 1, "f16", "none", "wide", 1, 3, 2, 6),
    (128, 128, "half", 1, "bf16", "f32", "token", 1, 1, 1, 2100),
    (64, 32, "half", 1, "f32", "own", "head", 40, 2, 1, 130),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward_and_backward(case):
    d, rot, layout, axes, kind, weight, order, B, Hq, Hk, T = case
    dtype = H.DTYPES[kind]
    g = torch.Generator().manual_seed(d * 7 + rot + T)
    q, k = rows(g, (B, Hq, T, d), dtype, order), rows(g, (B, Hk, T, d), dtype, order, 3.0)
    gq, gk = rows(g, (B, Hq, T, d), dtype, order), rows(g, (B, Hk, T, d), dtype, "head", 0.2)
    wt = {"own": dtype, "f32": torch.float32}.get(weight)
    qw, kw = (None if wt is None else
              (1 + 0.3 * torch.randn(d, generator=g)).to(wt).cuda() for _ in range(2))
    half = rot // 2
    sections = (half - 2 * (half // 3), half // 3, half // 3) if axes == 3 else None
    plan = E.rotary_plan(d, rot, base=1e4, layout=layout, sections=sections, amplitude=1.25)
    pos = torch.randint(-5, 70000, ((3,) if axes == 3 else ()) + (B, T), generator=g,
                        dtype=torch.int32)
    f = R.frequencies(rot, 1e4)
    axis = list(plan.axis[:half]) if axes == 3 else None
    leaves = [t.detach().requires_grad_(True) for t in (q, k, qw, kw) if t is not None]
    ql, kl = leaves[:2]
    ws = leaves[2:] if wt is not None else (None, None)
    y = E.norm_rotate(ql, kl, pos.cuda(), plan, *ws, eps=1e-5)
    grads = torch.autograd.grad(y, leaves, (gq, gk))
    for i, (x, w, gr) in enumerate(((q, qw, gq), (k, kw, gk))):
        x64, g64 = x.double().cpu(), gr.double().cpu()
        w64 = None if w is None else w.double().cpu()
        ref, pre = H.norm_rotate(x64, w64, pos, f, 1e-5, axis, layout, 1.25)
        tol = H.norm_tolerance(ref, pre, rot, layout, dtype, 1.25)
        err = (y[i].detach().double().cpu() - ref).abs()
        assert bool((err <= tol).all()), (i, float((err / tol).max()))
        dx, dw, z = H.norm_back(g64, x64, w64, pos, f, 1e-5, axis, layout, 1.25)
        tx, tw = H.back_tolerances(dx, dw, g64, z, rot, layout, dtype, wt or dtype, 1.25)
        err = (grads[i].double().cpu() - dx).abs()
        assert bool((err <= tx).all()), (i, float((err / tx).max()))
        if w is not None:
            assert grads[2 + i].dtype == wt
            err = (grads[2 + i].double().cpu() - dw).abs()
            assert bool((err <= tw).all()), (i, float((err / tw).max()))


def test_backward_is_the_forward_passes_derivative():
    """The gradients against differences of the float32 call itself: central differences of
    step h are off by h^2 times a third derivative, below 40 here, and by the outputs'
    rounding, 32 U of a sum of 3 * 2 * 5 * 16 products of size 4, over h."""
    g = torch.Generator().manual_seed(3)
    q = torch.randn(1, 2, 5, 16, generator=g).cuda()
    k = torch.randn(1, 1, 5, 16, generator=g).cuda()
    w = [(1 + 0.2 * torch.randn(16, generator=g)).cuda() for _ in range(2)]
    up = [torch.randn(t.shape, generator=g).cuda() for t in (q, k)]
    pos = torch.arange(5, dtype=torch.int32).cuda()
    plan = E.rotary_plan(16, 8)

    def loss(q, k, qw, kw):
        y = E.norm_rotate(q, k, pos, plan, qw, kw)
        return sum((a.double() * b.double()).sum() for a, b in zip(y, up))
    leaves = [t.clone().requires_grad_(True) for t in (q, k, *w)]
    grads = torch.autograd.grad(loss(*leaves), leaves)
    h = 2.0 ** -7
    tol = 40 * h * h + 32 * H.U * 480 * 4 / h
    for i, leaf in enumerate((q, k, *w)):
        for j in torch.randperm(leaf.numel(), generator=g)[:12].tolist():
            ends = []
            for s in (h, -h):
                moved = [t.clone() for t in (q, k, *w)]
                moved[i].view(-1)[j] += s
                with torch.no_grad():
                    ends.append(float(loss(*moved)))
            slope = (ends[0] - ends[1]) / (2 * h)
            assert abs(slope - float(grads[i].view(-1)[j])) <= tol, (i, j)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_no_weight_at_identity_is_the_rotation_of_unit_rows(kind):
    """Rows of +-1, whose mean square is 1 (an eps of 2^-40 is lost beside it), keep their values."""
    dtype = H.DTYPES[kind]
    g = torch.Generator().manual_seed(5)
    x = torch.randint(0, 2, (2, 3, 9, 64), generator=g).mul(2).sub(1).to(dtype).cuda()
    pos = torch.zeros(9, dtype=torch.int32).cuda()
    y, none = E.norm_rotate(x, None, pos, E.rotary_plan(64), eps=2.0 ** -40)
    assert none is None and torch.equal(y, x)


def test_zero_rows_and_values_that_are_not_finite():
    x = torch.randn(1, 4, 3, 64, device="cuda")
    x[0, 0] = 0
    x[0, 1, 1, 7] = float("nan")
    x[0, 2, 2, 9] = float("inf")
    pos = torch.arange(3, dtype=torch.int32).cuda()
    y, _ = E.norm_rotate(x, None, pos, E.rotary_plan(64))
    assert torch.equal(y[0, 0], torch.zeros_like(y[0, 0]))
    bad = torch.isnan(y).any(-1)[0].cpu()
    assert bad[1].tolist() == [False, True, False] and bad[2].tolist() == [False, False, True]
    assert not bad[0].any() and not bad[3].any()


def test_in_place_and_given_outputs():
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn(2, 4, 6, 128, generator=g).bfloat16().cuda(), \
        torch.randn(2, 2, 6, 128, generator=g).bfloat16().cuda()
    w = torch.randn(128, generator=g).bfloat16().cuda()
    pos, plan = torch.arange(6, dtype=torch.int32).cuda(), E.rotary_plan(128)
    ref = E.norm_rotate(q, k, pos, plan, w, w)
    wide = torch.full((2, 6, 4, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[..., 16:144].transpose(1, 2)
    E.norm_rotate(q, None, pos, plan, w, q_out=out)
    assert torch.equal(out, ref[0])
    assert bool((wide[..., :16] == 7).all()) and bool((wide[..., 144:] == 7).all())
    a, b = q.clone(), k.clone()
    E.norm_rotate(a, b, pos, plan, w, w, q_out=a, k_out=b)
    assert torch.equal(a, ref[0]) and torch.equal(b, ref[1])


def test_broadcast_inputs_and_gradients():
    """One row seen by every head, and a gradient that is one number seen by all."""
    x = torch.randn(1, 1, 5, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    pos, plan = torch.arange(5, dtype=torch.int32).cuda(), E.rotary_plan(64)
    y, _ = E.norm_rotate(x.expand(2, 4, 5, 64), None, pos, plan, w)
    dx, dw = torch.autograd.grad(y.sum(), (x, w))
    y1, _ = E.norm_rotate(x, None, pos, plan, w)
    dx1, dw1 = torch.autograd.grad(y1, (x, w), torch.ones_like(y1))
    # (8 equal rows: sums of equal terms, exact but for the last rounding of each)
    assert torch.allclose(dx, 8 * dx1, rtol=8 * H.U, atol=64 * H.U)
    assert torch.allclose(dw, 8 * dw1, rtol=64 * H.U, atol=2000 * H.U)


def test_gradients_asked_for_in_part():
    q = torch.randn(1, 2, 3, 64, device="cuda")
    k = torch.randn(1, 1, 3, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    pos, plan = torch.arange(3, dtype=torch.int32).cuda(), E.rotary_plan(64)
    yq, yk = E.norm_rotate(q, k, pos, plan, w, w.detach())
    (dk,) = torch.autograd.grad(yk.sum(), (k,), retain_graph=True)
    (dw,) = torch.autograd.grad(yq.sum(), (w,), retain_graph=True)
    full = E.norm_rotate_backward(torch.ones_like(yq), torch.ones_like(yk), q, k.detach(), pos,
                                  plan, w.detach(), w.detach())
    assert torch.equal(dk, full[1]) and torch.equal(dw, full[2])
    none = E.norm_rotate_backward(torch.ones_like(yq), None, q, None, pos, plan, w.detach(),
                                  want_q_weight=False)
    assert torch.equal(none[0], full[0]) and none[1:] == (None, None, None)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(yk.sum(), (k,), create_graph=True)


def test_empty_calls():
    plan = E.rotary_plan(64)
    pos = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    q = torch.randn(2, 3, 0, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    y, _ = E.norm_rotate(q, None, pos, plan, w)
    dq, dw = torch.autograd.grad(y.sum(), (q, w))
    assert y.shape == q.shape == dq.shape and torch.equal(dw, torch.zeros_like(dw))


def test_streams_and_graphs():
    """The same bits on a stream of its own and from a captured graph, replayed with the
    program's own work between, as eagerly."""
    g = torch.Generator().manual_seed(9)
    q = torch.randn(3, 4, 700, 128, generator=g).bfloat16().cuda()
    k = torch.randn(3, 2, 700, 128, generator=g).bfloat16().cuda()
    w = torch.randn(128, generator=g).bfloat16().cuda()
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    pos, plan = torch.arange(700, dtype=torch.int32).cuda(), E.rotary_plan(128)
    ref = [*E.norm_rotate(q, k, pos, plan, w, w),
           *E.norm_rotate_backward(gq, gk, q, k, pos, plan, w, w)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [*E.norm_rotate(q, k, pos, plan, w, w),
               *E.norm_rotate_backward(gq, gk, q, k, pos, plan, w, w)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    got = [*E.norm_rotate(q, k, pos, plan, w, w, stream=side.cuda_stream),
           *E.norm_rotate_backward(gq, gk, q, k, pos, plan, w, w, stream=side.cuda_stream)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [*E.norm_rotate(q, k, pos, plan, w, w),
               *E.norm_rotate_backward(gq, gk, q, k, pos, plan, w, w)]
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        ref = [*E.norm_rotate(q, k, pos, plan, w, w),
               *E.norm_rotate_backward(gq, gk, q, k, pos, plan, w, w)]
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
