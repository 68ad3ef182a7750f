"""norm_rotate and its backward pass at the sizes that choose other kernels and cuts than small
calls do: what passes the caches by, runs of many tokens, buffers that 32 bits do not number;
and the derivative held to differences closely enough that a missing term shows.  References
are float64, on the GPU where they are large."""
import numpy as np
import pytest
import torch

import _serve_helpers as R
import _step_helpers as H
import paper_2608_23253_amd as E
from test_gpu_norm_rotate import rows

pytestmark = pytest.mark.gpu

EPS = 1e-5


def plan_of(d, rot, layout):
    return E.rotary_plan(d, rot, base=1e4, layout=layout), R.frequencies(rot, 1e4)


def weights(g, d, dtype):
    return [(1 + 0.3 * torch.randn(d, generator=g, device=g.device)).to(dtype).cuda()
            for _ in range(2)]


def hold(y, grads, x, g, w, pos, f, rot, layout):
    """One tensor's output, and its and its weight's gradient, within their tolerances."""
    x64, g64, w64 = x.double(), g.double(), w.double()
    ref, pre = H.norm_rotate(x64, w64, pos, f, EPS, None, layout)
    tol = H.norm_tolerance(ref, pre, rot, layout, x.dtype)
    assert bool(((y.double() - ref).abs() <= tol).all())
    del ref, pre, tol
    dx, dw, z = H.norm_back(g64, x64, w64, pos, f, EPS, None, layout)
    tx, tw = H.back_tolerances(dx, dw, g64, z, rot, layout, x.dtype, w.dtype)
    assert bool(((grads[0].double() - dx).abs() <= tx).all())
    assert bool(((grads[1].double() - dw).abs() <= tw).all())


# heads of q and of k so that the forward pass moves 274 to 285 MB, past the 256 MB above which
# loads and stores are non-temporal (the backward pass moves half as much again)
LARGE = [
    # dtype, weight, layout, rot, heads of q, of k
    ("bf16", "f32", "half", 128, 40, 12),
    ("bf16", "own", "interleaved", 64, 40, 12),
    ("f16", "own", "half", 64, 52, 0),
    ("f16", "f32", "interleaved", 128, 12, 40),
    ("f32", "own", "half", 128, 20, 7),
    ("f32", "own", "interleaved", 96, 20, 7),
]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: "-".join(map(str, c)))
def test_what_passes_the_caches_by(case):
    """10300 tokens, in runs of five with threads that have none: against float64, and row by row
    the same bits as in four calls that the caches hold (how a row is computed does not depend on
    where tokens are cut)."""
    kind, weight, layout, rot, Hq, G = case
    dtype, d, T = H.DTYPES[kind], 128, 10300
    g = torch.Generator(device="cuda").manual_seed(31)
    x = [torch.randn((1, T, h, d), generator=g, device="cuda").to(dtype).transpose(1, 2)
         for h in (Hq, G)]
    up = [torch.randn((1, T, h, d), generator=g, device="cuda").to(dtype).transpose(1, 2)
          for h in (Hq, G)]
    w = weights(g, d, torch.float32 if weight == "f32" else dtype)
    pos = torch.randint(0, 100000, (1, T), generator=g, device="cuda").to(torch.int32)
    plan, f = plan_of(d, rot, layout)
    assert 2 * T * (Hq + G) * d * dtype.itemsize > 1 << 28

    def call(a, b):
        q, k = (t[:, :, a:b] if t.shape[1] else None for t in x)
        gq, gk = (t[:, :, a:b] if t.shape[1] else None for t in up)
        return (E.norm_rotate(q, k, pos[:, a:b], plan, *w, eps=EPS),
                E.norm_rotate_backward(gq, gk, q, k, pos[:, a:b], plan, *w, eps=EPS))
    y, grads = call(0, T)
    for a in range(0, T, T // 4):
        b = a + T // 4
        part, part_grads = call(a, b)
        for i in range(2):
            if x[i].shape[1]:
                assert torch.equal(part[i], y[i][:, :, a:b])
                assert torch.equal(part_grads[i], grads[i][:, :, a:b])
    for i in range(2):
        if x[i].shape[1]:
            hold(y[i], (grads[i], grads[2 + i]), x[i], up[i], w[i], pos, f, rot, layout)


RUNS = [
    # d, rot, layout, dtype, order, B, heads of q, of k, T: tokens of a run
    (128, 128, "half", "bf16", "token", 1, 3, 2, 10300),            # 5
    (128, 64, "interleaved", "f32", "head", 3, 2, 1, 2100),         # 3, a run to a sequence's end
    (64, 64, "half", "f16", "token", 2, 4, 4, 7001),                # 6
    (255, 254, "half", "bf16", "wide", 1, 2, 1, 6200),              # 3 of 64 lanes each, one idle
    (256, 64, "half", "f32", "head", 1, 2, 2, 20000),               # 8: all threads, one lane
    (96, 24, "interleaved", "bf16", "token", 1, 1, 1, 40000),       # 16, fewer heads than lanes
    (2, 2, "half", "f32", "head", 1, 3, 1, 130000),                 # 63 of 64
    (80, 80, "half", "f16", "head", 5, 2, 3, 2999),                 # 7
]


@pytest.mark.parametrize("case", RUNS, ids=lambda c: "-".join(map(str, c)))
def test_runs_of_many_tokens(case):
    d, rot, layout, kind, order, B, Hq, G, T = case
    dtype = H.DTYPES[kind]
    g = torch.Generator().manual_seed(32)
    x = [rows(g, (B, h, T, d), dtype, order) for h in (Hq, G)]
    up = [rows(g, (B, h, T, d), dtype, order) for h in (Hq, G)]
    w = weights(g, d, dtype)
    pos = torch.randint(0, 100000, (B, T), generator=g, dtype=torch.int32).cuda()
    plan, f = plan_of(d, rot, layout)
    y = E.norm_rotate(*x, pos, plan, *w, eps=EPS)
    grads = E.norm_rotate_backward(*up, *x, pos, plan, *w, eps=EPS)
    for i in range(2):
        hold(y[i], (grads[i], grads[2 + i]), x[i], up[i], w[i], pos, f, rot, layout)


def test_buffers_that_32_bits_do_not_number():
    """Tokens 2^30 elements apart, in and out: as rows side by side."""
    B, h, T, d, gap = 2, 3, 5, 64, 1 << 30
    big = torch.empty(T * gap, dtype=torch.bfloat16, device="cuda")
    strides = (2 * h * d, d, gap, 1)
    x, out = (big[at:].as_strided((B, h, T, d), strides) for at in (0, h * d))
    g = torch.Generator().manual_seed(33)
    near, up = rows(g, (B, h, T, d), torch.bfloat16, "head"), rows(g, (B, h, T, d), torch.bfloat16,
                                                                     "head")
    x.copy_(near)
    w, _ = weights(g, d, torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32).cuda()
    plan, _ = plan_of(d, d, "half")
    want = E.norm_rotate(near, None, pos, plan, w)[0]
    back = E.norm_rotate_backward(up, None, near, None, pos, plan, w)
    E.norm_rotate(x, None, pos, plan, w, q_out=out)
    assert torch.equal(out, want) and torch.equal(x, near)
    got = E.norm_rotate_backward(up, None, x, None, pos, plan, w)
    assert torch.equal(got[0], back[0]) and torch.equal(got[2], back[2])
    out.copy_(up)
    got = E.norm_rotate_backward(out, None, x, None, pos, plan, w)
    assert torch.equal(got[0], back[0]) and torch.equal(got[2], back[2])


def differences(loss, x, i, j, h):
    """The central difference of fourth order in element j of x[i]."""
    ends = {}
    for s in (2, 1, -1, -2):
        moved = [t.clone() for t in x]
        moved[i].view(-1)[j] += s * h
        ends[s] = loss(*moved)
    return float((8 * (ends[1] - ends[-1]) - (ends[2] - ends[-2])) / (12 * h))


def test_differences_that_a_missing_term_would_show():
    """Gradients against differences of the float32 call, of step h.  The quotient is off its own
    value in float64 by the outputs that move with the element (others give the same bits): each
    end's rounding, weighed 8, 8, 1 and 1 in 12 h, so 18/12 h of the outputs' tolerance times the
    upstream gradient.  The same formula in float64 gives what the difference misses by its order,
    and the gradient has its own tolerance.  Without the term mean(g w x r), or without the
    weight, a gradient is refused at most elements."""
    g = torch.Generator().manual_seed(34)
    B, Hq, G, T, d, rot = 1, 2, 1, 5, 16, 8
    x = [torch.randn(B, h, T, d, generator=g) for h in (Hq, G)]
    x += [1 + 0.2 * torch.randn(d, generator=g) for _ in range(2)]
    up = [torch.randn(t.shape, generator=g) for t in x[:2]]
    pos = torch.arange(T, dtype=torch.int32)
    plan, f = plan_of(d, rot, "half")
    up64, pos64 = [u.double() for u in up], pos[None]

    def own(*v):
        y = E.norm_rotate(v[0], v[1], pos.cuda(), plan, v[2], v[3], eps=EPS)
        return sum((a.double().cpu() * b).sum() for a, b in zip(y, up64))

    def plain(*v):
        return sum((H.norm_rotate(v[i], v[2 + i], pos64, f, EPS)[0] * up64[i]).sum()
                   for i in range(2))
    leaves = [t.cuda().requires_grad_(True) for t in x]
    grads = torch.autograd.grad(E.norm_rotate(*leaves[:2], pos.cuda(), plan, *leaves[2:], eps=EPS),
                                leaves, [u.cuda() for u in up])
    x64 = [t.double() for t in x]
    h = 2.0 ** -6
    refused = {"mean": 0, "weight": 0}
    tried = 0
    for i in range(2):
        ref, pre = H.norm_rotate(x64[i], x64[2 + i], pos64, f, EPS)
        # (the ends' outputs are within h of these, relative to rows of size 4: half as much again)
        end = 1.5 * H.norm_tolerance(ref, pre, rot, "half", torch.float32) * up64[i].abs()
        dx, dw, z = H.norm_back(up64[i], x64[i], x64[2 + i], pos64, f, EPS)
        tx, tw = H.back_tolerances(dx, dw, up64[i], z, rot, "half", torch.float32, torch.float32)
        without = {"mean": z["r"] * z["u"],
                   "weight": z["r"] * (z["gb"] - z["unit"] * (z["gb"] * z["unit"]).mean(-1, True))}
        pair = [(j + rot // 2) % rot if j < rot else j for j in range(d)]
        for which, ref_grad, tol in ((i, dx, tx), (2 + i, dw, tw)):
            got = grads[which].double().cpu().reshape(-1)
            for j in torch.randperm(ref_grad.numel(), generator=g)[:12].tolist():
                if which < 2:
                    moving = end.reshape(-1, d)[j // d].sum()
                else:
                    moving = end[..., sorted({j, pair[j]})].sum()
                miss = abs(differences(plain, x64, which, j, h) - float(ref_grad.reshape(-1)[j]))
                most = miss + 18 / (12 * h) * float(moving) + float(tol.reshape(-1)[j])
                slope = differences(own, [t.detach() for t in leaves], which, j, h)
                assert abs(slope - float(got[j])) <= most, (which, j, most)
                if which < 2:
                    tried += 1
                    for n, bad in without.items():
                        refused[n] += abs(slope - float(bad.reshape(-1)[j])) > most
    assert all(n > tried // 2 for n in refused.values()), (refused, tried)
