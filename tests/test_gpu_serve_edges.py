"""GPU checks of the operators of e2s_serve.h at the edges of what their header allows: NaN
beside missing pages, the largest values, overlapping rows, gradients, and memory that
another stream still uses."""
import numpy as np
import pytest

import _serve_helpers as S
from test_gpu_cache import _check_attend, _cuda, _filled, _ints, _match

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E = pytest.importorskip("paper_2608_23253_amd")

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("T,max_tokens", [(1, 128), (1, 3000), (4, 2000), (20, 128), (20, 3000)])
def test_nan_key_beside_a_missing_page(T, max_tokens):
    """A token whose page is not there is seen by no query: its weight stays what it was,
    also where a NaN key makes every weight of the tokens that are there NaN."""
    rng = np.random.default_rng(51)
    n, P = 100, 16
    pool, table = _filled(rng, [n, n], 1, P, 64)
    pool.k[table[0, 1], 0, 3, 9] = 0x7F
    table[:, 4] = -1
    there = np.ones(n, bool)
    there[4 * P:5 * P] = False
    q = torch.from_numpy(rng.standard_normal((2, 7, T, 64))).to(BF).cuda()
    was = torch.full((2, 1, max_tokens), 0.25, device="cuda")
    call = E.CacheAttention(E.PagedCache.of(*pool.tensors()), 2, 7, T, max_tokens, BF,
                            causal=False, weights=True)
    out, w = call(q, _cuda(table), _ints([n, n]), weights_in=was, weights_out=was.clone())
    w = w.cpu().numpy()
    assert out[0].isnan().all() and not out[1].isnan().any()
    assert np.isnan(w[0, 0, :n][there]).all()
    assert (w[0, 0, :n][~there] == 0.25).all(), "a weight for tokens that no query sees"
    assert not np.isnan(w[1]).any() and (w[1, 0, :n][~there] == 0.25).all()


def test_evict_moves_the_largest_values():
    """Elements from 248 * 2^120 on are held as 2^128, which float32 does not have: moved to
    another block they, and what shares the block, stay what they are."""
    rng = np.random.default_rng(52)
    D, P, G, n, K = 64, 16, 2, 40, 20
    both, pages = S.tables(rng, [n, K], P, 1)
    pool = S.Pool(pages, G, P, D)
    rows = rng.standard_normal((G, n, D)) * 1e37
    rows[0, 5], rows[1, 30, 3] = 3.35e38, -3.4e38
    rows = rows.astype(np.float32).astype(np.float64)
    for which in ("k", "v"):
        pool.append(which, list(both[0]), 0, rows)
    assert pool.ks[both[0][0], 0] == 2.0 ** 120 and pool.ks[both[0][1], 1] == 2.0 ** 120
    cache = E.PagedCache.of(*pool.tensors())
    w = np.zeros((1, G, n), np.float32)
    w[0, :, 2:2 * K:2] = 1.0                          # tokens 2, 4 .. 38, and the first
    w[0, 0, 5], w[0, 0, 4] = 1.0, 0.0
    keep, _, _ = E.cache_evict(cache, _cuda(both[:1]), _ints([n]), _cuda(w), _cuda(both[1:]), K)
    torch.cuda.synchronize()
    for g in range(G):
        idx = S.evict(w[0, g], n, K, 0, 0)
        assert keep[0, g].tolist() == idx
        for x, s in ((pool.k, pool.ks), (pool.v, pool.vs)):
            for blk in range(-(-K // P)):
                part = idx[blk * P:(blk + 1) * P]
                held = np.stack([S._VALUES[x[both[0][i // P], g, i % P]]
                                 * float(s[both[0][i // P], g]) for i in part])
                sc = S.block_scale(np.abs(held).max())
                x[both[1][blk], g, :len(part)] = S.to_e4m3(held / sc)
                s[both[1][blk], g] = sc
    _match(cache, pool)


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("T,lengths,max_tokens", [
    (1, [100, 7], 128), (1, [3000, 100], 3000), (1, [9000], 9000), (5, [300, 5], 2100),
    (20, [2500, 300], 2500),
])
def test_attend_large_values(dtype, T, lengths, max_tokens):
    """Values of one sign, of up to 2^127: their sum before the division by the weights' sum is
    beyond float32, their mean is not."""
    rng = np.random.default_rng(53)
    pool, table = _filled(rng, lengths, 1, 64, 64)
    pool.v &= 0x7F
    pool.vs *= np.float32(2.0 ** 122)
    q = torch.from_numpy(rng.standard_normal((len(lengths), 6, T, 64)) * 0.1).to(dtype)
    _check_attend(pool, table, lengths, q, max_tokens=max_tokens)


@pytest.mark.parametrize("T,max_tokens", [(1, 64), (1, 3000), (5, 2100), (20, 64)])
def test_attend_the_largest_held_values(T, max_tokens):
    """2^128, the largest that the cache holds, is no infinity: as a key's element where the
    query's is 0, as a value of a token that gets no weight, and of one that gets some."""
    rng = np.random.default_rng(54)
    n, P, D = 40, 16, 64
    pool, table = _filled(rng, [n], 1, P, D)
    block, other = table[0, 0], table[0, 1]
    pool.k[block, 0] = S.to_e4m3(np.zeros((P, D)))
    pool.ks[block, 0] = 2.0 ** 120
    pool.k[block, 0, 3, 7] = S.to_e4m3(np.array(256.0))              # 2^128
    pool.v[other, 0] = S.to_e4m3(np.clip(rng.standard_normal((P, D)) * 50, -200, 200))
    pool.vs[other, 0] = 2.0 ** 120
    pool.v[other, 0, 2, 11] = S.to_e4m3(np.array(256.0))
    pool.v[other, 0, 4] = S.to_e4m3(np.full(D, 256.0))
    q = torch.from_numpy(rng.standard_normal((1, 6, T, D)) * 0.1).to(FL)
    q[..., 7] = 0.0
    # token 20 (row 4 of the second page) gets no weight: a key far on the other side
    pool.k[other, 0, 4] = S.to_e4m3(np.zeros(D))
    q[..., 9] = 30.0
    pool.k[other, 0, 4, 9] = S.to_e4m3(np.array(-448.0))
    pool.ks[other, 0] = 2.0 ** 4
    _check_attend(pool, table, [n], q, max_tokens=max_tokens, causal=False)


def test_rotate_rows_that_overlap():
    """Rows one element apart (windows over one line): the output's rows do not overlap."""
    D, T, H = 64, 5, 3
    line = torch.randn(4000, generator=torch.Generator().manual_seed(5)).cuda()
    q = line.as_strided((2, H, T, D), (1000, 300, 1, 1))
    k = line.as_strided((2, T, H, D), (0, 0, 1, 1)).transpose(1, 2)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 7
    plan = E.rotary_plan(D)
    got = E.rotate_positions(q, k, pos, plan)
    want = E.rotate_positions(q.contiguous(), k.contiguous(), pos, plan)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("given", [True, False])
def test_workspace_outlives_the_object_on_another_stream(given):
    """An object that is dropped while another stream still works in its workspace: the
    allocator keeps the memory until that work is done."""
    rng = np.random.default_rng(55)
    pool, table = _filled(rng, [5000], 2, 64, 128)
    q = torch.from_numpy(rng.standard_normal((1, 4, 1, 128))).to(BF).cuda()
    cache, pages, lengths = E.PagedCache.of(*pool.tensors()), _cuda(table), _ints([5000])
    want, _ = E.cache_attend(q, cache, pages, lengths)
    torch.cuda.synchronize()
    att = E.CacheAttention(cache, 1, 4, 1, 5000)
    size, at = att.workspace.numel(), att.workspace.data_ptr()
    assert size > 0
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    if given:
        got, _ = att(q, pages, lengths, stream=side.cuda_stream)
    else:
        with torch.cuda.stream(side):
            got, _ = att(q, pages, lengths)
    assert not side.query(), "the other stream's work was to be under way still"
    del att
    new = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert new.data_ptr() != at
    side.synchronize()
    assert torch.equal(got, want)


def test_rotate_and_attend_on_a_given_stream():
    """`stream` without entering it, for every call: their work waits for what is on that
    stream, and the current one stays free."""
    rng = np.random.default_rng(56)
    pool, table = _filled(rng, [300, 5000], 2, 64, 64)
    cache, pages, lengths = E.PagedCache.of(*pool.tensors()), _cuda(table), _ints([300, 5000])
    q = torch.from_numpy(rng.standard_normal((2, 4, 2, 64))).to(BF).cuda()
    pos = torch.arange(2, dtype=torch.int32, device="cuda")
    plan = E.rotary_plan(64)
    turned, _ = E.rotate_positions(q, None, pos, plan)
    out, w = E.cache_attend(turned, cache, pages, lengths, want_weights=True)
    src = torch.zeros_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        src.copy_(q)
    a, _ = E.rotate_positions(src, None, pos, plan, stream=side.cuda_stream)
    b, w2 = E.cache_attend(a, cache, pages, lengths, want_weights=True, stream=side.cuda_stream)
    torch.cuda.current_stream().synchronize()
    assert not side.query(), "the calls were to wait for the other stream's work"
    side.synchronize()
    for x, y in ((turned, a), (out, b), (w, w2)):
        assert torch.equal(x, y)


def _grad_of_formula(x, w, pos, f, kw):
    y = x.double().requires_grad_()
    S.rotate(y, pos, f, layout=kw["layout"], inverse=kw["inverse"]).backward(w.double())
    return y.grad


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("layout,inverse", [("half", False), ("interleaved", True)])
def test_rotation_has_its_gradient(dtype, layout, inverse):
    g = torch.Generator().manual_seed(6)
    R, D = 32, 64
    x, w = (torch.randn((2, 3, 9, D), generator=g).to(dtype) for _ in range(2))
    k, wk = (torch.randn((2, 1, 9, D), generator=g).to(dtype) for _ in range(2))
    pos = torch.randint(0, 500, (2, 9), generator=g, dtype=torch.int32)
    plan, f = E.rotary_plan(D, rot_dim=R, layout=layout), S.frequencies(R, 1e4)
    kw = dict(layout=layout, inverse=inverse)
    q1, k1 = x.cuda().requires_grad_(), k.cuda().requires_grad_()
    yq, yk = E.rotate_positions(q1, k1, pos.cuda(), plan, inverse=inverse)
    with torch.no_grad():
        plain = E.rotate_positions(q1, k1, pos.cuda(), plan, inverse=inverse)
    assert torch.equal(yq, plain[0]) and torch.equal(yk, plain[1])
    assert not plain[0].requires_grad
    torch.autograd.backward([yq, yk], [w.cuda(), wk.cuda()])
    for got, a, b in ((q1.grad, x, w), (k1.grad, k, wk)):
        ref = _grad_of_formula(a, b, pos, f, kw)
        tol = S.rotate_tolerance(b.double(), ref, R, layout, dtype)
        assert ((got.cpu().double() - ref).abs() <= tol).all()
    # one of the two alone, through a loss whose gradient is one broadcast number
    q2 = x.cuda().requires_grad_()
    yq, yk = E.rotate_positions(q2, k.cuda(), pos.cuda(), plan, inverse=inverse)
    yq.sum().backward()
    ones = torch.ones_like(x)
    ref = _grad_of_formula(x, ones, pos, f, kw)
    tol = S.rotate_tolerance(ones.double(), ref, R, layout, dtype)
    assert ((q2.grad.cpu().double() - ref).abs() <= tol).all()
    # against differences: the map is linear, so a step of 1 is exact but for the roundings of
    # its two results (a half step of the type and 8 * 2^-24 of |x0| + |x1| each)
    for at in ((0, 1, 3, 5), (1, 2, 8, 30), (1, 0, 0, 50)):
        up, down = x.double(), x.double()
        up[at] += 1
        down[at] -= 1
        up, down = up.to(dtype), down.to(dtype)
        step = float(up[at].double() - down[at].double())
        with torch.no_grad():
            y1, _ = E.rotate_positions(up.cuda(), None, pos.cuda(), plan, inverse=inverse)
            y0, _ = E.rotate_positions(down.cuda(), None, pos.cuda(), plan, inverse=inverse)
        slope = float(((y1.double() - y0.double()).cpu() * w.double())[at[:3]].sum()) / step
        # only the element's own row changes, and of it the pair
        row = at[:3]
        big = 2 * (up[row].abs().max() + 1).double()
        tol = 2 * 2 * (S.HALF_STEP[dtype] + 8 * 2.0 ** -24) * float(big * w[row].double().abs().max())
        assert abs(slope - float(q1.grad[at])) <= tol / step + \
            S.HALF_STEP[dtype] * abs(slope) + 1e-6


def test_rotation_gradients_of_shared_and_strided_inputs():
    """A query that all heads share, token-major rows, a second derivative, and no gradient
    where none is asked for."""
    g = torch.Generator().manual_seed(7)
    D, T, H = 64, 11, 4
    one = torch.randn((2, 1, T, D), generator=g).cuda().requires_grad_()
    wide = torch.randn((2, T, H, D), generator=g).cuda().requires_grad_()
    w = torch.randn((2, H, T, D), generator=g).cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 31
    plan = E.rotary_plan(D)
    yq, yk = E.rotate_positions(one.expand(2, H, T, D), wide.transpose(1, 2), pos, plan)
    assert yq.requires_grad and yk.requires_grad
    gq, gk = torch.autograd.grad([yq, yk], [one, wide], [w, w], create_graph=True)
    with torch.no_grad():
        back, _ = E.rotate_positions(w, None, pos, plan, inverse=True)
    assert torch.equal(gk, back.transpose(1, 2))
    # (four heads summed in float32)
    assert ((gq - back.sum(1, keepdim=True)).abs()
            <= 8 * 2.0 ** -24 * back.abs().sum(1, keepdim=True)).all()
    # the gradient is linear in w: its own derivative is the rotation
    w2 = w.clone().requires_grad_()
    y, _ = E.rotate_positions(wide.transpose(1, 2), None, pos, plan)
    gx, = torch.autograd.grad(y, wide, w2, create_graph=True)
    v = torch.randn((2, T, H, D), generator=g).cuda()
    gw, = torch.autograd.grad(gx, w2, v)
    with torch.no_grad():
        there, _ = E.rotate_positions(v.transpose(1, 2), None, pos, plan)
    assert torch.equal(gw, there)
    with pytest.raises(ValueError):
        E.rotate_positions(wide.transpose(1, 2), None, pos, plan, q_out=torch.empty_like(w))
    out = torch.empty_like(w)
    with torch.no_grad():
        E.rotate_positions(wide.transpose(1, 2), None, pos, plan, q_out=out)
    assert torch.equal(out, y)


def test_attention_says_that_it_has_no_gradient():
    rng = np.random.default_rng(57)
    pool, table = _filled(rng, [100], 2, 16, 64)
    cache, pages, lengths = E.PagedCache.of(*pool.tensors()), _cuda(table), _ints([100])
    q = torch.from_numpy(rng.standard_normal((1, 4, 2, 64))).to(BF).cuda()
    want, ww = E.cache_attend(q, cache, pages, lengths, want_weights=True)
    q.requires_grad_()
    out, w = E.cache_attend(q, cache, pages, lengths, want_weights=True)
    assert torch.equal(out, want) and torch.equal(w, ww)
    for y in (out, w):
        with pytest.raises(RuntimeError, match="no backward"):
            y.float().sum().backward(retain_graph=True)
    acc = torch.zeros_like(ww)
    out, w = E.cache_attend(q, cache, pages, lengths, weights_in=acc, weights_out=acc)
    assert w is acc and torch.equal(acc, ww)
    with pytest.raises(RuntimeError, match="no backward"):
        out.float().sum().backward()
    with pytest.raises(ValueError):
        E.cache_attend(q, cache, pages, lengths, out=torch.empty_like(want))
    with torch.no_grad():
        given = torch.empty_like(want)
        out, _ = E.cache_attend(q, cache, pages, lengths, out=given)
    assert out is given and torch.equal(out, want) and not out.requires_grad
