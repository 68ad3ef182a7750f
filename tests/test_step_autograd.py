"""norm_rotate's backward pass on saved tensors that are not where they were, or do not lie as
they did: copies that a saved-tensor hook gives back, weights that a checkpoint makes again.
On the CPU the launch is replaced by the formula, behind a look at what the record says of the
tensors that it is handed; on a GPU gradients are those of the direct call, bit for bit."""
import ctypes

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import _serve_helpers as R
import _step_helpers as H
from paper_2608_23253_amd import _serve as V
from paper_2608_23253_amd import _step as S

BASE, EPS = 1e4, 1e-5


def plain_launch(where, tensors, fn, record, plan_ref, positions_at, q_at, k_at, qw_at, kw_at,
                 *rest, stream=None):
    """The launch in float64, of tensors on the CPU, whose record has to be theirs."""
    sh = S.NormRotateShape.from_buffer_copy(record)
    back = where.endswith("backward")
    q, k, positions, qw, kw = tensors[:5]
    grads, outs = (tensors[5:7], tensors[7:9]) if back else ((None, None), tensors[5:7])
    for t, at in ((q, q_at), (k, k_at), (qw, qw_at), (kw, kw_at), (positions, positions_at)):
        assert at == (None if t is None else t.data_ptr())
    weight = qw if qw is not None else kw
    if weight is not None:
        assert sh.weight_dtype == (0 if weight.dtype is torch.float32 else sh.dtype)
    plan = plan_ref._obj
    f = R.frequencies(plan.rot_dim, BASE)
    p = positions.expand(sh.batch, sh.num_tokens)
    if sh.pos_stride[1] != 0 or positions.dim() == 2:
        assert tuple(sh.pos_stride)[1:] == positions.stride()
    dws = tensors[9:11] if back else ()
    for i, (t, w, g, o) in enumerate(zip((q, k), (qw, kw), grads, outs)):
        heads = (sh.q_heads, sh.k_heads)[i]
        if t is None:
            assert heads == 0
            continue
        assert t.shape == (sh.batch, heads, sh.num_tokens, plan.head_dim) and t.stride(3) == 1
        assert tuple((sh.q_stride, sh.k_stride)[i]) == t.stride()[:3]
        assert tuple((sh.q_out_stride, sh.k_out_stride)[i]) == o.stride()[:3]
        w64 = None if w is None else w.double()
        if not back:
            o.copy_(H.norm_rotate(t.double(), w64, p, f, sh.eps)[0])
            continue
        assert tuple((sh.q_grad_stride, sh.k_grad_stride)[i]) == g.stride()[:3]
        dx, dw, _ = H.norm_back(g.double(), t.double(), w64, p, f, sh.eps)
        o.copy_(dx)
        if dws[i] is not None:
            dws[i].copy_(dw)


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        monkeypatch.setattr(S, "_launch", plain_launch)
        for module in (S, V):
            monkeypatch.setattr(module, "_check", lambda *a, **k: None)
    return request.param


def contiguous_copy(t):
    return t.detach().clone(memory_format=torch.contiguous_format)


def wide_copy(t):
    """The same values as part of a larger buffer."""
    big = t.new_zeros((*t.shape[:-1], 2 * t.shape[-1] + 3))
    big[..., :t.shape[-1]] = t
    return big[..., :t.shape[-1]]


def reversed_copy(t):
    """The same values, the last dimension's elements furthest apart."""
    order = list(range(t.dim()))[::-1]
    return t.detach().permute(order).contiguous().permute(order)


class Layer:
    """Queries and keys as parts of one buffer of rows of a token, and the gradients that the
    direct calls give."""

    def __init__(self, device, kind, parts=("q", "k"), weight="own"):
        g = torch.Generator().manual_seed(11)
        B, T, Hq, G, d = 2, 7, 4, 2, 64
        dtype = H.DTYPES[kind]
        self.plan = V.rotary_plan(d, base=BASE)
        self.fused = torch.randn(B, T, (Hq + 2 * G) * d, generator=g).to(dtype).to(device)
        self.sizes = (B, T, Hq, G, d)
        self.positions = torch.randint(0, 3000, (B, T), generator=g, dtype=torch.int32).to(device)
        kind_w = torch.float32 if weight == "f32" else dtype
        self.w = [(0.2 * torch.randn(d, generator=g)).to(kind_w).to(device) for _ in range(2)]
        self.up = [torch.randn(B, T, h, d, generator=g).to(dtype).to(device).transpose(1, 2)
                   for h in (Hq, G)]
        self.parts = parts

    def split(self, fused):
        B, T, Hq, G, d = self.sizes
        q = fused[..., :Hq * d].view(B, T, Hq, d).transpose(1, 2)
        k = fused[..., Hq * d:(Hq + G) * d].view(B, T, G, d).transpose(1, 2)
        return q if "q" in self.parts else None, k if "k" in self.parts else None

    def call(self, fused, wq, wk):
        q, k = self.split(fused)
        y = S.norm_rotate(q, k, self.positions, self.plan, wq, wk, eps=EPS)
        return tuple(t for t in y if t is not None)

    def ups(self):
        return [u for u, n in zip(self.up, "qk") if n in self.parts]

    def direct(self, wq, wk):
        """Gradients of the buffer and of the weights as they are given."""
        q, k = self.split(self.fused)
        up = [u if n in self.parts else None for u, n in zip(self.up, "qk")]
        dq, dk, dwq, dwk = S.norm_rotate_backward(*up, q, k, self.positions, self.plan, wq, wk,
                                                  eps=EPS)
        B, T, Hq, G, d = self.sizes
        whole = torch.zeros_like(self.fused)
        gq, gk = self.split(whole)
        for at, grad in ((gq, dq), (gk, dk)):
            if at is not None:
                at.copy_(grad)
        return whole, dwq, dwk


    def check(self, got):
        """Gradients within what their arithmetic allows of the formula's in float64."""
        d = self.sizes[4]
        rotary = (R.frequencies(d, BASE), EPS)
        of_fused, position = got[0].double().cpu(), self.positions.cpu()
        for i, (t, dx, g, n) in enumerate(zip(self.split(self.fused), self.split(of_fused), self.up,
                                              "qk")):
            if n not in self.parts:
                assert got[1 + i] is None
                continue
            x, w, g = (a.double().cpu() for a in (t, self.w[i], g))
            ref, dw, z = H.norm_back(g, x, w, position, *rotary)
            tx, tw = H.back_tolerances(ref, dw, g, z, d, "half", t.dtype, self.w[i].dtype)
            assert bool(((dx - ref).abs() <= tx).all())
            assert bool(((got[1 + i].double().cpu() - dw).abs() <= tw).all())


def same(got, want):
    for a, b in zip(got, want):
        assert (a is None) == (b is None)
        assert a is None or (a.dtype == b.dtype and torch.equal(a, b))


COPIES = [contiguous_copy, wide_copy, reversed_copy]


@pytest.mark.parametrize("copy", COPIES, ids=lambda f: f.__name__)
@pytest.mark.parametrize("kind,parts,weight", [("bf16", ("q", "k"), "own"), ("f32", ("q", "k"), "own"),
                                               ("f16", ("q", "k"), "f32"), ("f32", ("k",), "own"),
                                               ("bf16", ("q",), "f32")])
def test_a_hook_that_gives_copies(device, kind, parts, weight, copy):
    L = Layer(device, kind, parts, weight)
    want = L.direct(*L.w)
    leaves = [t.clone().requires_grad_(True) for t in (L.fused, *L.w)]

    def unpack(t):
        return copy(t) if t.dim() != 1 or copy is not wide_copy else copy(t[None])[0]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach().clone(), unpack):
        y = L.call(*leaves)
    got = torch.autograd.grad(y, leaves, L.ups(), allow_unused=True)
    L.check(got)
    # Rows of an odd stride are read by narrower loads, so a lane holds other elements of a row
    # and its sums are added in another order: those are held to the formula alone.
    if copy is not wide_copy:
        same(got, want)


def test_a_hook_and_one_output_alone(device):
    """Of the outputs one has a gradient: the other tensor takes no part."""
    L = Layer(device, "f32")
    leaves = [t.clone().requires_grad_(True) for t in (L.fused, *L.w)]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, contiguous_copy):
        y = L.call(*leaves)
    got = torch.autograd.grad(y[1], leaves, L.up[1], allow_unused=True)
    only = Layer(device, "f32", ("k",))
    want = only.direct(*L.w)
    same(got[:1] + got[2:], (want[0], want[2]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_a_checkpoint_that_makes_its_weights_again(device, kind):
    """Weights of 1 + w that only the region holds: the first forward pass's are gone, and
    their memory is another's, when the backward pass comes."""
    L = Layer(device, kind)
    direct = L.direct(*(1 + w for w in L.w))
    leaves = [t.clone().requires_grad_(True) for t in (L.fused, *L.w)]
    y = checkpoint(lambda f, a, b: L.call(f, 1 + a, 1 + b), *leaves, use_reentrant=False)
    others = [torch.full_like(L.w[0], 1e4) for _ in range(64)]
    got = torch.autograd.grad(y, leaves, L.ups())
    same(got, direct)
    assert all(bool((t == 1e4).all()) for t in others)


@pytest.mark.gpu
def test_saved_tensors_kept_on_the_host():
    L = Layer("cuda", "bf16")
    want = L.direct(*L.w)
    leaves = [t.clone().requires_grad_(True) for t in (L.fused, *L.w)]
    with torch.autograd.graph.save_on_cpu(pin_memory=True):
        y = L.call(*leaves)
    same(torch.autograd.grad(y, leaves, L.ups()), want)


def test_what_a_hook_gives_is_checked(device):
    """Fewer tokens than were saved: refused, not read past."""
    L = Layer(device, "f32")
    fused = L.fused.clone().requires_grad_(True)
    with torch.autograd.graph.saved_tensors_hooks(
            lambda t: t, lambda t: t[:, :, :3] if t.dim() == 4 else t):
        y = L.call(fused, None, None)
    with pytest.raises(ValueError):
        torch.autograd.grad(y, fused, L.ups())


def test_the_record_is_read_as_the_library_reads_it():
    assert ctypes.sizeof(S.NormRotateShape) == S._NORM.size
