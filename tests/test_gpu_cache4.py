"""The 4-bit cache: what is stored, bit for bit, what is read, and attention over it against
float64."""
import numpy as np
import pytest
import torch

import _serve_helpers as R
import _step_helpers as H
import paper_2608_23253_amd as E

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def device(x, kind, order="head"):
    """float64 [B, H, T, d] on the GPU in a layout."""
    x = x.to(H.DTYPES[kind])
    if order == "token":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    if order == "wide":
        big = torch.zeros(x.shape[0], x.shape[2], x.shape[1], x.shape[3] + 32, dtype=x.dtype,
                          device="cuda")
        big[..., 16:16 + x.shape[3]] = x.transpose(1, 2).cuda()
        return big[..., 16:16 + x.shape[3]].transpose(1, 2)
    return x.cuda()


def cache_of(pool):
    return E.PagedCache4.of(*pool.tensors())


def tables_of(cache):
    return [t.cpu().numpy() if t.dtype == torch.uint8 else t.float().cpu().numpy()
            for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------

APPENDS = [
    # d, page, Hkv, dtype, order, starts, tokens, counts
    (128, 64, 2, "bf16", "token", [0, 31, 32, 63, 200], 1, None),
    (64, 32, 3, "f16", "head", [0, 5, 31, 64], 1, None),
    (128, 32, 1, "f32", "wide", [0, 7], 70, None),
    (64, 128, 2, "bf16", "token", [3, 100, 0], 150, [150, 0, 33]),
    (128, 128, 4, "f16", "head", [1], 257, [256]),
    (64, 64, 1, "f32", "head", [0, 62], 9, [9, 4]),
    (128, 64, 2, "f32", "token", [30, 0], 3, [-4, 9]),
    (64, 32, 2, "bf16", "wide", [16], 8, None),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "-".join(map(str, c[:5])))
def test_append_holds_what_is_documented(case):
    """Old tokens stay as they were; new ones are held bit for bit; and are read as held."""
    d, P, G, kind, order, starts, T, counts = case
    rng = np.random.default_rng(d + P + T)
    B = len(starts)
    n = [T if counts is None else max(0, min(counts[b], T)) for b in range(B)]
    pool, table = H.filled(rng, B, G, P, d, starts)
    wide, pages = R.tables(rng, [s + T for s in starts], P, 2)
    # the old tokens' tables, moved to pages of the wider table
    pool2 = H.Pool4(pages, G, P, d)
    for b in range(B):
        for i in range(-(-starts[b] // P)):
            for x, y in ((pool.k, pool2.k), (pool.v, pool2.v), (pool.ks, pool2.ks),
                         (pool.vs, pool2.vs)):
                y[wide[b, i]] = x[table[b, i]]
    cache = cache_of(pool2)
    size = 2.0 ** torch.from_numpy(rng.uniform(-20, 10, (B, G, T, 1)))
    k, v = (torch.from_numpy(rng.standard_normal((B, G, T, d))) * size for _ in range(2))
    k[0, 0, 0] = 0
    v[0, 0, 0] = 0
    # elements in the middle between codes, and the largest at a border of the scale
    k[-1, -1, -1, :8] = torch.tensor([6.0, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5.0])
    k[-1, -1, -1, 8:32] = 0.125
    v[-1, -1, -1] = 0.125
    v[-1, -1, -1, :8] = torch.tensor([6.0, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5.0])
    kd, vd = device(k, kind, order), device(v, kind, order)
    E.cache4_append(cache, ints(wide), ints(starts), kd, vd,
                    count=None if counts is None else ints(counts))
    k64, v64 = kd.double().cpu().numpy(), vd.double().cpu().numpy()
    for b in range(B):
        pool2.append(list(wide[b]), starts[b], k64[b][:, :n[b]], v64[b][:, :n[b]])
    H.same_tables(pool2, tables_of(cache))
    got = E.cache4_read(cache, ints(wide), ints(starts), T,
                        count=None if counts is None else ints(counts), dtype=torch.float32)
    for b in range(B):
        for g in range(G):
            for which, x in zip("kv", got):
                ref = pool2.rows(which, list(wide[b]), starts[b] + n[b], g)[starts[b]:]
                assert np.array_equal(x[b, g, :n[b]].double().cpu().numpy(), ref)
                assert not x[b, g, n[b]:].any()
    if kind != "f32":                                 # one rounding to the rows' type
        low = E.cache4_read(cache, ints(wide), ints(starts), T,
                            count=None if counts is None else ints(counts), dtype=H.DTYPES[kind])
        for a, x in zip(low, got):
            assert torch.equal(a, x.to(H.DTYPES[kind]))


def test_append_what_the_pruner_kept():
    rng = np.random.default_rng(1)
    pool, table = H.filled(rng, 2, 2, 32, 64, [40, 0])
    wide, pages = R.tables(rng, [40 + 12, 12], 32)
    pool = H.Pool4(pages, 2, 32, 64)
    cache = cache_of(pool)
    k, v = (torch.from_numpy(rng.standard_normal((2, 2, 30, 64))).bfloat16().cuda()
            for _ in range(2))
    idx = np.sort(rng.permutation(30)[:12])[None].repeat(2, 0).astype(np.int32)
    idx[1, 3], idx[1, 7] = 30, -1                      # outside: zeros
    E.cache4_append(cache, ints(wide), ints([40, 0]), k, v, src_idx=ints(idx))
    kz, vz = (torch.cat([x, torch.zeros_like(x[:, :, :1])], 2).double().cpu().numpy()
              for x in (k, v))
    src = np.where((idx < 0) | (idx >= 30), 30, idx)
    for b in range(2):
        pool.append(list(wide[b]), [40, 0][b], kz[b][:, src[b]], vz[b][:, src[b]])
    H.same_tables(pool, tables_of(cache))


def test_values_that_are_not_finite_take_their_block_or_row():
    pool = H.Pool4(2, 1, 32, 128)
    cache = cache_of(pool)
    k, v = torch.randn(1, 1, 4, 128), torch.randn(1, 1, 4, 128)
    k[0, 0, 1, 40] = float("nan")
    k[0, 0, 2, 127] = float("-inf")
    v[0, 0, 3, 5] = float("inf")
    table = np.array([[1]], np.int32)
    E.cache4_append(cache, ints(table), ints([30]), k.cuda(), v.cuda())
    pool.append([1], 30, k[0].double().numpy(), v[0].double().numpy())
    H.same_tables(pool, tables_of(cache))
    gk, gv = E.cache4_read(cache, ints(table), ints([30]), 2, dtype=torch.float32)
    assert torch.isnan(gk[0, 0, 1, 32:64]).all() and torch.isnan(gk).sum() == 32
    assert not torch.isnan(gv).any()


def test_append_and_read_leave_what_has_no_page():
    """Pages outside the pool, tokens past the table, negative starts."""
    rng = np.random.default_rng(2)
    pool, _ = H.filled(rng, 1, 2, 32, 64, [96], spare=1)
    cache = cache_of(pool)
    before = tables_of(cache)
    pages = pool.k.shape[0]
    table = np.array([[-1, pages], [0, 1 << 30], [0, 1]], np.int32)
    k = torch.randn(3, 2, 20, 64, device="cuda")
    E.cache4_append(cache, ints(table), ints([20, 60, -1]), k, k)
    for a, b in zip(before, tables_of(cache)):
        assert np.array_equal(a, b, equal_nan=True)
    out = E.cache4_read(cache, ints(table), ints([20, 60, -1]), 20, dtype=torch.float32)
    for which, x in zip("kv", out):
        assert not x[0].any() and not x[1].any()       # no page, and past the table
        assert not x[2, :, 0].any()
        for g in range(2):
            ref = pool.rows(which, [0, 1], 19, g)
            assert np.array_equal(x[2, g, 1:].double().cpu().numpy(), ref, equal_nan=True)


def test_read_into_given_rows_leaves_the_others():
    rng = np.random.default_rng(4)
    pool, table = H.filled(rng, 2, 2, 64, 128, [70, 9])
    cache = cache_of(pool)
    wide = torch.full((2, 50, 2, 160), 7.0, device="cuda")
    k_out = wide[..., :128].transpose(1, 2)
    v_out = torch.full((2, 2, 50, 128), 7.0, device="cuda")
    E.cache4_read(cache, ints(table), ints([20, 0]), 50, count=ints([50, 9]), k_out=k_out,
                  v_out=v_out)
    for which, x in (("k", k_out), ("v", v_out)):
        for g in range(2):
            ref = pool.rows(which, list(table[0]), 70, g)[20:]
            assert np.array_equal(x[0, g].double().cpu().numpy(), ref)
            ref = pool.rows(which, list(table[1]), 9, g)
            assert np.array_equal(x[1, g, :9].double().cpu().numpy(), ref)
            assert bool((x[1, g, 9:] == 7).all())
    assert bool((wide[..., 128:] == 7).all())


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

ATTENDS = [
    # d, page, H, Hkv, dtype, T, lengths, counts, causal, order, scale
    (128, 64, 28, 4, "bf16", 1, [1, 700], None, True, "token", None),
    (128, 32, 4, 4, "f16", 1, [0, 31, 32, 33, 127, 128, 129], None, True, "head", None),
    (64, 32, 16, 2, "f32", 1, [0, 1, 300, 255], None, True, "head", None),
    (64, 128, 8, 1, "bf16", 1, [513, 2], None, False, "wide", 0.3),
    (128, 128, 6, 2, "f32", 1, [260], None, True, "token", None),
    (128, 64, 14, 2, "bf16", 4, [130, 3, 0], None, True, "token", None),       # 28 rows
    (64, 64, 4, 4, "f16", 20, [19, 20, 21, 190], [20, 7, 0, 13], True, "head", None),
    (128, 32, 8, 2, "f32", 9, [100, 5], [9, 9], False, "token", None),
    (128, 64, 28, 4, "bf16", 11, [300], [10], True, "wide", None),             # 77 rows
    (64, 32, 2, 1, "f32", 40, [45], None, True, "token", None),
    (128, 64, 3, 1, "f16", 33, [64, 500], [33, 32], True, "token", None),
    (128, 128, 32, 32, "f16", 1, [140] * 3, None, True, "token", None),
    (64, 64, 16, 1, "bf16", 1, [2600], None, True, "token", None),
    (128, 64, 17, 1, "bf16", 1, [1500], None, True, "token", 2.0),
]


def check(out, ref, tol, counts=None, T=None):
    err = np.abs(out.double().cpu().numpy() - ref)
    bad = ~(err <= tol)
    bad &= ~(np.isnan(ref) & np.isnan(out.double().cpu().numpy()))
    if bad.any():
        at = np.argwhere(bad)[0]
        raise AssertionError((at.tolist(), float(out.double().cpu().numpy()[tuple(at)]),
                              float(ref[tuple(at)]), float(tol[tuple(at)]), int(bad.sum()),
                              float(np.nanmax(err / np.maximum(tol, 1e-300)))))


@pytest.mark.parametrize("case", ATTENDS, ids=lambda c: "-".join(map(str, c[:7])))
def test_attend(case):
    d, P, Hq, G, kind, T, lengths, counts, causal, order, scale = case
    rng = np.random.default_rng(d + P + Hq + T)
    B = len(lengths)
    pool, table = H.filled(rng, B, G, P, d, lengths)
    q = torch.from_numpy(rng.standard_normal((B, Hq, T, d)) *
                         2.0 ** rng.uniform(-2, 2, (B, Hq, T, 1)))
    qd = device(q, kind, order)
    ref, tol = H.attend(pool, table, lengths, qd.double().cpu(), kind, counts, causal, scale)
    out = torch.full_like(qd, 7.0)
    E.cache4_attend(qd, cache_of(pool), ints(table), ints(lengths), scale=scale or 0.0,
                    causal=causal, out=out, q_count=None if counts is None else ints(counts))
    if counts is not None:
        for b, c in enumerate(counts):
            assert bool((out[b, :, c:] == 7).all())
            out[b, :, c:] = 0
    check(out, ref, tol)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_missing_pages_and_nan_behind_the_mask(kind, T):
    """Tokens without a page are seen by no query; what no query sees may hold NaN scales (every
    row that nothing wrote does, in a pool of 0xFF bytes)."""
    rng = np.random.default_rng(11)
    d, P, G, Hq = 128, 32, 2, 6
    lengths = [250, 40, 64]
    pool, table = H.filled(rng, 3, G, P, d, lengths)
    table = table.copy()
    table[0, 2], table[0, 5] = -1, 1 << 30
    table[1, 0], table[1, 1] = -7, pool.k.shape[0]       # nothing left
    q = torch.from_numpy(rng.standard_normal((3, Hq, T, d)))
    qd = device(q, kind)
    ref, tol = H.attend(pool, table, lengths, qd.double().cpu(), kind)
    out = E.cache4_attend(qd, cache_of(pool), ints(table), ints(lengths))
    check(out, ref, tol)
    assert not out[1].any()


@pytest.mark.parametrize("T", [3, 24])
def test_nan_reaches_the_queries_that_see_it(T):
    rng = np.random.default_rng(12)
    d, P, G, Hq = 64, 32, 2, 2
    lengths = [200, 200]
    pool, table = H.filled(rng, 2, G, P, d, lengths)
    # the key of sequence 0's last token but one, the value of sequence 1's, of head 1
    at = lengths[0] - 2
    pool.ks[table[0, at // P], 1, at % P // 16, at % 4, 1, at % 16 // 4] = 255
    pool.vs[table[1, at // P], 1, at % P] = np.nan
    q = torch.from_numpy(rng.standard_normal((2, Hq, T, d)))
    qd = device(q, "bf16")
    qd[0, 0, 0, 3] = float("nan")
    qd[1, 0, 1, 3] = float("inf")
    out = E.cache4_attend(qd, cache_of(pool), ints(table), ints(lengths)).float().cpu()
    bad = torch.isnan(out).any(-1)
    assert torch.equal(bad, torch.isnan(out).all(-1))
    want = torch.zeros(2, Hq, T, dtype=torch.bool)
    want[:, 1, T - 2:] = True                          # they see token `at`
    want[0, 0, 0] = want[1, 0, 1] = True
    assert torch.equal(bad, want)


def test_far_apart_weights_and_scales():
    """A peak among many small weights in one step, and values of very different scales."""
    rng = np.random.default_rng(13)
    d, P = 128, 64
    for kind in ("bf16", "f32"):
        pool, table = H.filled(rng, 1, 1, P, d, [900], spread=12.0)
        q = torch.from_numpy(rng.standard_normal((1, 8, 1, d)) * 2.0 ** -9)
        qd = device(q, kind)
        ref, tol = H.attend(pool, table, [900], qd.double().cpu(), kind)
        check(E.cache4_attend(qd, cache_of(pool), ints(table), ints([900])), ref, tol)


def test_a_length_that_is_too_long_is_cut():
    rng = np.random.default_rng(14)
    pool, table = H.filled(rng, 2, 1, 32, 64, [96, 64])
    q = device(torch.from_numpy(rng.standard_normal((2, 2, 1, 64))), "f32")
    ref, tol = H.attend(pool, table[:, :2], [64, 64], q.double().cpu(), "f32")
    out = E.cache4_attend(q, cache_of(pool), ints(table[:, :2].copy()), ints([1 << 30, 64]))
    check(out, ref, tol)
    out = E.cache4_attend(q, cache_of(pool), ints(table[:, :2].copy()), ints([-5, 64]))
    assert not out[0].any()
    check(out[1:], ref[1:], tol[1:])


def test_strided_pools():
    """A layer's pages within a pool that holds every layer's."""
    rng = np.random.default_rng(15)
    pool, table = H.filled(rng, 1, 2, 32, 64, [70])
    k, ks, v, vs = pool.tensors()
    kk = torch.zeros((k.shape[0], 3) + k.shape[1:], dtype=torch.uint8, device="cuda")
    vv = torch.zeros((v.shape[0], 3) + v.shape[1:], dtype=torch.uint8, device="cuda")
    kk[:, 1], vv[:, 1] = k, v
    q = device(torch.from_numpy(rng.standard_normal((1, 4, 1, 64))), "bf16")
    cache = E.PagedCache4.of(kk[:, 1], ks, vv[:, 1], vs)
    ref, tol = H.attend(pool, table, [70], q.double().cpu(), "bf16")
    check(E.cache4_attend(q, cache, ints(table), ints([70])), ref, tol)
    new = torch.from_numpy(rng.standard_normal((1, 2, 3, 64))).bfloat16()
    E.cache4_append(cache, ints(table), ints([70]), new.cuda(), new.cuda())
    pool.append(list(table[0]), 70, new[0].double().numpy(), new[0].double().numpy())
    H.same_tables(pool, [kk[:, 1].cpu().numpy(), ks.cpu().numpy(), vv[:, 1].cpu().numpy(),
                         vs.float().cpu().numpy()])
    assert not kk[:, 0].any() and not kk[:, 2].any() and not vv[:, 0].any() and not vv[:, 2].any()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,G,T,most", [(64, 32, 1, 90), (70, 8, 1, 300), (3, 4, 2, 5000)])
def test_every_split(kind, B, G, T, most):
    """One, two and four waves that part the keys, several workgroups to a sequence; sequences
    read the same pages."""
    rng = np.random.default_rng(16)
    d, P = 64, 32
    one = min(most, 320)
    pool, table = H.filled(rng, 1, G, P, d, [one])
    pages = np.array([[table[0][i % (one // P)] for i in range(-(-most // P))]] * B, np.int32)
    lengths = [int(x) for x in rng.integers(0, most + 1, B)]
    lengths[0] = most
    some = [0, 1, B - 1]                               # compared with float64
    q = torch.from_numpy(rng.standard_normal((B, G, T, d)))
    qd = device(q, kind)
    out = E.cache4_attend(qd, cache_of(pool), ints(pages), ints(lengths))
    ref, tol = H.attend(pool, pages[some], [lengths[b] for b in some], qd.double().cpu()[some],
                        kind)
    check(out[some], ref, tol)
    # and the others with calls of one sequence
    for b in range(2, B - 1, 17):
        alone = E.cache4_attend(qd[b:b + 1], cache_of(pool), ints(pages[b:b + 1]),
                                ints(lengths[b:b + 1]))
        r2, t2 = H.attend(pool, pages[b:b + 1], lengths[b:b + 1], qd.double().cpu()[b:b + 1], kind)
        check(alone, r2, t2)
        check(out[b:b + 1], r2, t2)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_value_codes_at_every_border(kind):
    """Rows of every largest element's mantissa, beside the elements around each border between
    codes: bf16 all that lie within 2^-6 of it, f16 the nearest on either side."""
    dtype, d = H.DTYPES[kind], 64
    rows = []
    for m in range(128):
        top = 1.0 + m / 128
        s = H.value_scale(top)
        near = []
        for border in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            x = torch.tensor(border * s, dtype=torch.float64).to(dtype)
            for step in range(-4, 5):
                near.append((x.view(torch.int16) + step).view(dtype).item())
        for i in range(0, len(near), d - 1):
            part = [min(v, top) for v in near[i:i + d - 1]]
            rows.append([top] + part + [-0.0] * (d - 1 - len(part)))
    v = torch.tensor(rows, dtype=torch.float64)
    v = v * torch.where(torch.arange(d) % 2 == 1, -1.0, 1.0)
    T = len(rows)
    pages = -(-T // 128)
    pool = H.Pool4(pages, 1, 128, d)
    cache = cache_of(pool)
    x = v[None, None].to(dtype)
    assert torch.equal(x.double()[0, 0], v)
    E.cache4_append(cache, ints([list(range(pages))]), ints([0]), x.cuda(), x.cuda())
    pool.append(list(range(pages)), 0, v[None].numpy(), v[None].numpy())
    H.same_tables(pool, tables_of(cache))


@pytest.mark.parametrize("d,P", [(64, 32), (128, 128)])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_every_magnitude_of_a_type(kind, d, P):
    """Rows (and blocks of 32) anywhere in the type's range, from its smallest element to its
    largest, held bit for bit; and a source row that several tokens name."""
    dtype = H.DTYPES[kind]
    info = torch.finfo(dtype)
    rng = np.random.default_rng(17)
    low = int(np.log2(info.tiny)) + int(np.log2(info.eps))
    T, N = 200, 150
    top = torch.from_numpy(rng.integers(low, int(np.log2(info.max)) + 1, (1, 1, N, d // 32, 1)))
    x = torch.from_numpy(rng.uniform(1, 2, (1, 1, N, d // 32, 32))) * \
        2.0 ** (top - torch.from_numpy(rng.integers(0, 5, (1, 1, N, d // 32, 32))))
    x = (x * torch.from_numpy(rng.choice([-1.0, 1.0], x.shape))).reshape(1, 1, N, d)
    x[0, 0, 0], x[0, 0, 1], x[0, 0, 2] = info.max, info.tiny * info.eps, 0
    x[0, 0, 3, 1::2] = -info.max
    x = x.clamp(-info.max, info.max).to(dtype)
    idx = rng.integers(0, N, (1, T)).astype(np.int32)
    idx[0, :4], idx[0, 50:60] = range(4), 7
    pages = -(-(T + 5) // P)
    pool = H.Pool4(pages, 1, P, d)
    cache = cache_of(pool)
    v = x.flip(2).contiguous()
    E.cache4_append(cache, ints([list(range(pages))]), ints([5]), x.cuda(), v.cuda(),
                    src_idx=ints(idx))
    pool.append(list(range(pages)), 5, x[0][:, idx[0]].double().numpy(),
                v[0][:, idx[0]].double().numpy())
    H.same_tables(pool, tables_of(cache))
    got = E.cache4_read(cache, ints([list(range(pages))]), ints([5]), T, dtype=torch.float32)
    for which, y in zip("kv", got):
        ref = torch.from_numpy(pool.rows(which, list(range(pages)), 5 + T, 0)[5:])
        assert torch.equal(y[0, 0].cpu(), ref.float())
