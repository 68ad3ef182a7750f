"""The step's operators as a program runs them: norms and positions, the kept tokens into the
4-bit cache, attention over it, step after step; the same eagerly, on another stream and from
captured graphs; and what the binding refuses."""
import ctypes

import numpy as np
import pytest
import torch

import _serve_helpers as R
import _step_helpers as H
import paper_2608_23253_amd as E
from paper_2608_23253_amd import _step as S

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Layer:
    """A layer's state: 3 sequences, 8 heads of 2 key heads, d = 64."""

    def __init__(self, kind="bf16", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.H, self.G, self.d, self.P = H.DTYPES[kind], 3, 8, 2, 64, 32
        self.plan = E.rotary_plan(self.d, base=1e4)
        self.cache = E.PagedCache4(12, self.G, self.d, self.P)
        self.pages = ints(np.random.default_rng(seed).permutation(12).reshape(3, 4))
        self.w = [(1 + 0.2 * torch.randn(self.d, generator=g)).to(self.dtype).cuda()
                  for _ in range(2)]
        self.lengths = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.g = g

    def rows(self, heads, T):
        x = torch.randn(self.B, T, heads, self.d, generator=self.g)
        return x.to(self.dtype).cuda().transpose(1, 2)

    def step(self, q, k, v, positions, kept=None, stream=None):
        q, k = E.norm_rotate(q, k, positions, self.plan, *self.w, stream=stream)
        E.cache4_append(self.cache, self.pages, self.lengths, k, v, src_idx=kept, stream=stream)
        n = k.shape[2] if kept is None else kept.shape[1]
        with torch.cuda.stream(torch.cuda.ExternalStream(stream) if stream else
                               torch.cuda.current_stream()):
            self.lengths.add_(n)
        return E.cache4_attend(q, self.cache, self.pages, self.lengths, causal=kept is None,
                               stream=stream)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_a_prompt_its_kept_tokens_and_answers(kind):
    """Against float64 on the values that each call was given: the rotated rows that torch
    holds, the tables that the cache holds."""
    L = Layer(kind)
    kept = ints(np.stack([np.sort(np.random.default_rng(b).permutation(60)[:40])
                          for b in range(3)]))
    at = 0
    for T, keep in ((60, kept), (5, None), (1, None), (1, None)):
        q, k, v = L.rows(L.H, T), L.rows(L.G, T), L.rows(L.G, T)
        pos = torch.arange(at, at + T, dtype=torch.int32, device="cuda")
        out = L.step(q, k, v, pos, keep)
        at += T
        ref_q, ref_k = E.norm_rotate(q, k, pos, L.plan, *L.w)
        p64 = pos[None].expand(3, T).cpu()
        want, pre = H.norm_rotate(k.double().cpu(), L.w[1].double().cpu(), p64,
                                  R.frequencies(64, 1e4), 1e-6)
        tol = H.norm_tolerance(want, pre, 64, "half", L.dtype)
        assert bool(((ref_k.double().cpu() - want).abs() <= tol).all())
        pool = H.Pool4(12, 2, 32, 64)
        pool.k, pool.ks, pool.v = (t.cpu().numpy().copy() for t in
                                   (L.cache.k, L.cache.k_scale, L.cache.v))
        pool.vs = L.cache.v_scale.float().cpu().numpy()
        n = L.lengths.tolist()
        held = E.cache4_read(L.cache, L.pages, ints([0, 0, 0]), max(n), dtype=torch.float32)
        for b in range(3):
            for h in range(2):
                for which, x in zip("kv", held):
                    assert np.array_equal(x[b, h, :n[b]].double().cpu().numpy(),
                                          pool.rows(which, L.pages[b].tolist(), n[b], h))
        ref, tol = H.attend(pool, L.pages.cpu().numpy(), n, ref_q.double().cpu(), kind,
                            causal=keep is None)
        err = np.abs(out.double().cpu().numpy() - ref)
        assert (err <= tol).all(), float((err / tol).max())


def test_streams_and_graphs_give_the_same_bits():
    """A decoding step eagerly, on a stream of its own, on a stream that is given, and from a
    graph, replayed with eager work between."""
    def start():
        L = Layer(seed=3)
        L.step(L.rows(8, 40), L.rows(2, 40), L.rows(2, 40),
               torch.arange(40, dtype=torch.int32, device="cuda"))
        return L, (L.rows(8, 1), L.rows(2, 1), L.rows(2, 1), ints([40]))
    ref = []
    L, x = start()
    for i in range(4):
        ref.append(L.step(*x[:3], x[3] + i).clone())
    tables = [t.clone() for t in (L.cache.k, L.cache.k_scale, L.cache.v, L.cache.v_scale)]

    side = torch.cuda.Stream()
    for mode in ("side", "given", "graph"):
        L, x = start()
        torch.cuda.synchronize()
        got = []
        if mode == "graph":
            pos = x[3].clone()
            graph = torch.cuda.CUDAGraph()
            lengths = L.lengths.clone()
            with torch.cuda.graph(graph):
                out = L.step(*x[:3], pos)
            L.lengths.copy_(lengths)                  # (nothing ran while it was captured)
            for i in range(4):
                graph.replay()
                torch.cuda.synchronize()
                got.append(out.clone())
                torch.randn(1000, device="cuda").sum()
                pos.add_(1)
        else:
            for i in range(4):
                p = x[3] + i
                torch.cuda.synchronize()
                if mode == "side":
                    with torch.cuda.stream(side):
                        got.append(L.step(*x[:3], p))
                else:
                    got.append(L.step(*x[:3], p, stream=side.cuda_stream))
                torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), mode
        now = (L.cache.k, L.cache.k_scale, L.cache.v, L.cache.v_scale)
        assert all(torch.equal(a, b) for a, b in zip(now, tables)), mode


def test_one_attention_object_many_calls_and_two_at_once():
    """Split sequences: an object's calls one after the other, and two objects of the same
    sizes on two streams at once."""
    rng = np.random.default_rng(5)
    pool, table = H.filled(rng, 1, 2, 128, 128, [640])
    cache = E.PagedCache4.of(*pool.tensors())
    pages = ints(np.tile(table[:, :5], (2, 4)))       # 2560 tokens, of the same pages
    lengths = ints([2560, 2300])
    qs = [torch.from_numpy(rng.standard_normal((2, 8, 1, 128))).bfloat16().cuda()
          for _ in range(4)]
    one, two = (E.Cache4Attention(cache, 2, 8, 1, 2560) for _ in range(2))
    assert one.workspace.numel() > 0
    ref = [E.cache4_attend(q, cache, pages, lengths, max_tokens=2560) for q in qs]
    assert all(torch.equal(one(q, pages, lengths), r) for q, r in zip(qs, ref))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for q in qs:
        with torch.cuda.stream(a):
            got.append(one(q, pages, lengths))
        with torch.cuda.stream(b):
            got.append(two(q, pages, lengths))
    torch.cuda.synchronize()
    for i, r in enumerate(ref):
        assert torch.equal(got[2 * i], r) and torch.equal(got[2 * i + 1], r)


def test_the_backward_pass_of_no_tokens_zeroes_the_weights_gradients():
    plan = E.rotary_plan(64)
    sh = S.NormRotateShape(2, 0, 3, 0, 1, 0, 1e-6, 0)
    for n in ("q_stride", "q_grad_stride", "q_out_stride"):
        getattr(sh, n)[:] = (192, 64, 64)
    dw = torch.full((66,), 7.0, device="cuda")
    st = S._LIB.e2s_norm_rotate_backward(ctypes.byref(sh), ctypes.byref(plan), None, None, None,
                                         None, None, None, None, None, None, dw.data_ptr(), None,
                                         None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and not dw[:64].any() and bool((dw[64:] == 7).all())


def test_the_binding_refuses():
    cache = E.PagedCache4(4, 2, 64)
    pages, n = ints([[0, 1]]), ints([3])
    q = torch.randn(1, 4, 1, 64, device="cuda").bfloat16()
    k = torch.randn(1, 2, 3, 64, device="cuda").bfloat16()
    plan, pos = E.rotary_plan(64), torch.arange(3, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    with pytest.raises(ValueError):
        E.norm_rotate(None, None, pos, plan)
    with pytest.raises(ValueError):
        E.norm_rotate(k, k[:, :, :2], pos, plan)                    # two numbers of tokens
    with pytest.raises(ValueError):
        E.norm_rotate(k, None, pos[:2], plan)
    with pytest.raises(ValueError):
        E.norm_rotate(k, None, pos, plan, w[:32])
    with pytest.raises(TypeError):
        E.norm_rotate(k, None, pos, plan, w.half())
    with pytest.raises(TypeError):
        E.norm_rotate(k, k.clone(), pos, plan, w, w.bfloat16())
    with pytest.raises(E.E2SError):
        E.norm_rotate(k, None, pos, plan, w, eps=0.0)
    with pytest.raises(ValueError):
        E.norm_rotate(k.requires_grad_(True), None, pos, plan, k_out=None, q_out=k.detach())
    k = k.detach()
    with pytest.raises(ValueError):
        E.norm_rotate_backward(k, None, None, k, pos, plan)
    with pytest.raises(ValueError):
        E.PagedCache4(4, 2, 64, page_tokens=16)
    with pytest.raises(ValueError):
        E.PagedCache4.of(cache.k, cache.k_scale, cache.v[..., :8], cache.v_scale)
    with pytest.raises(TypeError):
        E.PagedCache4.of(cache.k, cache.k_scale, cache.v, cache.v_scale.float())
    with pytest.raises(ValueError):
        E.cache4_append(cache, pages, n, k[:, :1], k[:, :1])
    with pytest.raises(ValueError):
        E.cache4_read(cache, pages, n, 3, k_out=k[:, :, :2])
    with pytest.raises(E.E2SError):
        E.Cache4Attention(cache, 1, 3, 1, 128)                      # 3 heads of 2 key heads
    with pytest.raises(ValueError):
        E.cache4_attend(q.requires_grad_(True), cache, pages, n, out=torch.empty_like(q))
    out = E.cache4_attend(q, cache, pages, n)
    with pytest.raises(RuntimeError):
        out.sum().backward()
    with pytest.raises(E.E2SError):
        with torch.no_grad():
            E.cache4_attend(q, cache, pages, n, out=q)
