"""GPU checks of rotary positions (e2s_rotate_positions) against the formula in float64:
layouts, parts of a head, scalings, three axes, strides and alignments, both directions
as each other's gradient, in place, and no tokens."""
import numpy as np
import pytest

import _serve_helpers as S

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E = pytest.importorskip("paper_2608_23253_amd")

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def _x(seed, shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


def _check(got, x, pos, plan_kw, dtype, inverse=False, axis=None, amplitude=1.0):
    R = plan_kw["rot_dim"]
    layout = plan_kw.get("layout", "half")
    fk = {k: v for k, v in plan_kw.items() if k in ("scaling", "factor", "original_len")}
    f = S.frequencies(R, plan_kw["base"], **fk)
    ref = S.rotate(x.double(), pos, f, axis, layout, amplitude, inverse)
    tol = S.rotate_tolerance(x.double(), ref, R, layout, dtype, amplitude)
    bad = (got.cpu().double() - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} beyond the rounding"


CASES = [  # B, Hq, Hk, T, d, dtype, plan
    (1, 28, 4, 1, 128, BF, dict(rot_dim=128, base=1e6)),
    (2, 4, 2, 37, 128, HF, dict(rot_dim=64, base=1e4, layout="interleaved")),
    (3, 3, 1, 129, 64, FL, dict(rot_dim=16, base=1e4)),
    (1, 2, 2, 300, 80, BF, dict(rot_dim=20, base=1e4)),                  # 10 pairs: W = 2
    (2, 1, 1, 7, 10, FL, dict(rot_dim=6, base=500.0, layout="interleaved")),   # 3 pairs: W = 1
    (1, 2, 1, 5, 3, BF, dict(rot_dim=2, base=10.0)),                     # odd row
    (1, 1, 1, 3, 256, HF, dict(rot_dim=256, base=1e4)),
    (1, 1, 1, 3, 256, HF, dict(rot_dim=2, base=1e4)),
    (2, 8, 8, 1500, 128, BF, dict(rot_dim=128, base=1e4, scaling="linear", factor=4.0)),
    (2, 2, 2, 33, 128, FL, dict(rot_dim=128, base=1e4, scaling="base", factor=8.0)),
    (1, 2, 2, 65, 128, FL, dict(rot_dim=2, base=1e4, scaling="base", factor=8.0)),
]


@pytest.mark.parametrize("B,Hq,Hk,T,d,dtype,kw", CASES)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate_against_float64(B, Hq, Hk, T, d, dtype, kw, inverse):
    q, k = _x(1, (B, Hq, T, d), dtype), _x(2, (B, Hk, T, d), dtype)
    pos = torch.randint(0, 5000, (B, T), generator=torch.Generator().manual_seed(3),
                        dtype=torch.int32)
    plan = E.rotary_plan(d, **kw)
    qo, ko = E.rotate_positions(q.cuda(), k.cuda(), pos.cuda(), plan, inverse=inverse)
    for got, x in ((qo, q), (ko, k)):
        _check(got, x, pos, kw, dtype, inverse)
        R = kw["rot_dim"]
        assert torch.equal(got.cpu()[..., R:], x[..., R:])


def test_ramp_and_its_amplitude():
    kw = dict(rot_dim=128, base=1e4, scaling="ramp", factor=16.0, original_len=4096.0)
    amp = 0.1 * np.log(16.0) + 1.0
    x = _x(4, (2, 3, 50, 128), FL)
    pos = (torch.arange(50, dtype=torch.int32) * 1300).expand(2, 50)
    for a in (0.0, 0.75):
        plan = E.rotary_plan(128, amplitude=a, **kw)
        got, none = E.rotate_positions(x.cuda(), None, pos.cuda(), plan)
        assert none is None
        _check(got, x, pos, kw, FL, amplitude=a or amp)


def test_far_and_negative_positions():
    """Angles of far positions: turns are reduced in float64 (2^31 * 2^-53 of a turn)."""
    kw = dict(rot_dim=128, base=1e4)
    x = _x(5, (1, 2, 6, 128), FL)
    pos = torch.tensor([[0, -1, 1 << 20, -(1 << 20), (1 << 31) - 1, -(1 << 31)]],
                       dtype=torch.int64)
    plan = E.rotary_plan(128, **kw)
    got, _ = E.rotate_positions(x.cuda(), None, pos.to(torch.int32).cuda(), plan)
    # The frequencies have a relative error of a few 2^-53, and so has the reference's own
    # product: 8 * 2^-53 of p f radians beside the float32 terms.
    R, f = 128, S.frequencies(128, 1e4)
    ref = S.rotate(x.double(), pos, f)
    tol = S.rotate_tolerance(x.double(), ref, R, "half", FL)
    far = pos.abs().double()[0][:, None] * torch.from_numpy(np.concatenate([f, f])) * 2.0 ** -50
    tol = tol + far * (x.abs() + x.roll(64, -1).abs())
    assert ((got.cpu().double() - ref).abs() <= tol).all()


def test_three_axes():
    kw = dict(rot_dim=128, base=1e6)
    x = _x(6, (2, 4, 40, 128), BF)
    pos = torch.randint(0, 300, (3, 2, 40), generator=torch.Generator().manual_seed(7),
                        dtype=torch.int32)
    plan = E.rotary_plan(128, sections=(16, 24, 24), **kw)
    axis = [0] * 16 + [1] * 24 + [2] * 24
    got, _ = E.rotate_positions(x.cuda(), None, pos.cuda(), plan)
    _check(got, x, pos, kw, BF, axis=axis)
    # three equal positions are one
    one = E.rotary_plan(128, **kw)
    same = pos[:1].expand(3, -1, -1)
    a, _ = E.rotate_positions(x.cuda(), None, same.cuda(), plan)
    b, _ = E.rotate_positions(x.cuda(), None, pos[0].cuda(), one)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_strides_alignment_and_broadcast(dtype, offset):
    """Token-major rows inside a wider projection, starting at an odd element; positions
    shared by the batch."""
    B, H, T, d = 2, 3, 21, 64
    wide = _x(8, (B, T, H * d + 2 * offset + 8), dtype).cuda()
    q = wide[..., offset:offset + H * d].unflatten(2, (H, d)).transpose(1, 2)
    pos = torch.arange(100, 100 + T, dtype=torch.int32)
    kw = dict(rot_dim=64, base=1e4)
    plan = E.rotary_plan(d, **kw)
    got, _ = E.rotate_positions(q, None, pos.cuda(), plan)
    _check(got, q.cpu(), pos.expand(B, T), kw, dtype)
    # the same into a strided output
    out = torch.full((B, T, H, d + 3), 9.0, dtype=dtype, device="cuda")
    view = out[..., 1:1 + d].transpose(1, 2)
    E.rotate_positions(q, None, pos.cuda(), plan, q_out=view)
    assert torch.equal(view, got)
    assert (out[..., 0] == 9).all() and (out[..., d + 1:] == 9).all()
    # a query that all heads share
    shared = q[:, :1].expand(B, 5, T, d)
    wide_out, _ = E.rotate_positions(shared, None, pos.cuda(), plan)
    assert torch.equal(wide_out[:, 3], got[:, 0])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place_and_strided_positions(layout):
    q, k = _x(9, (2, 4, 17, 128), BF).cuda(), _x(10, (2, 2, 17, 128), BF).cuda()
    pos = torch.randint(0, 900, (17, 2), dtype=torch.int32).cuda().t()      # [2, 17] strided
    plan = E.rotary_plan(128, rot_dim=96, layout=layout)
    want = E.rotate_positions(q, k, pos, plan)
    E.rotate_positions(q, k, pos.contiguous(), plan, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_gradient_is_the_way_back():
    """d<w, rotate(x)>/dx = rotate back(w), by differences in float64 of the formula (which
    the forward direction is held to above) and by <w, R x> = <R' w, x>."""
    kw = dict(rot_dim=32, base=1e4, scaling="ramp", factor=4.0, original_len=512.0)
    amp = 0.1 * np.log(4.0) + 1.0
    x, w = _x(11, (1, 2, 9, 64), FL), _x(12, (1, 2, 9, 64), FL)
    pos = torch.arange(0, 900, 100, dtype=torch.int32)[None]
    plan = E.rotary_plan(64, **kw)
    back, _ = E.rotate_positions(w.cuda(), None, pos.cuda(), plan, inverse=True)
    f = S.frequencies(32, 1e4, scaling="ramp", factor=4.0, original_len=512.0)
    loss = lambda y: float((w.double() * S.rotate(y, pos, f, amplitude=amp)).sum())   # noqa: E731
    y = x.double()
    for at in [(0, 0, 3, 5), (0, 1, 8, 20), (0, 1, 2, 40), (0, 0, 0, 0)]:
        step = torch.zeros_like(y)
        step[at] = 1e-3
        slope = (loss(y + step) - loss(y - step)) / 2e-3       # exact: the map is linear
        partner = (at[0], at[1], at[2], (at[3] + 16) % 32) if at[3] < 32 else at
        tol = 9 * 2.0 ** -24 * amp * float(w[at].abs() + w[partner].abs()) + 1e-9
        assert abs(float(back[at]) - slope) <= tol
    # there and back is the amplitude squared: two passes' rounding
    there, _ = E.rotate_positions(x.cuda(), None, pos.cuda(), plan)
    again, _ = E.rotate_positions(there, None, pos.cuda(), plan, inverse=True)
    both = x[..., :32].abs()
    both = both[..., :16] + both[..., 16:]
    both = torch.cat([both, both], -1).double()
    err = (again[..., :32].cpu().double() - amp * amp * x[..., :32].double()).abs()
    assert (err <= 40 * 2.0 ** -24 * amp * amp * both).all()


def test_no_tokens():
    plan = E.rotary_plan(64)
    q = torch.empty((2, 3, 0, 64), dtype=BF, device="cuda")
    out, _ = E.rotate_positions(q, None, torch.empty((2, 0), dtype=torch.int32, device="cuda"),
                                plan)
    assert out.shape == q.shape
