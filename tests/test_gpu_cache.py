"""GPU checks of the 8-bit cache (e2s_cache_append, e2s_cache_attend, e2s_cache_evict)
against plain float64 implementations: what is stored and kept bit for bit, attention
and its weights within the rounding that its arithmetic makes.

Bytes and scales that nothing wrote are NaN throughout, and unused entries of the page
tables name no page, so whatever reads them shows."""
import numpy as np
import pytest

import _serve_helpers as S

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E = pytest.importorskip("paper_2608_23253_amd")

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rows(rng, B, G, N, D, dtype, spread=2.0):
    x = rng.standard_normal((B, G, N, D)) * np.exp2(spread * rng.random((B, G, N, 1)))
    return torch.from_numpy(x).to(dtype)


def _filled(rng, lengths, G, P, D, spare=2, bad=None):
    """A pool whose sequences hold `lengths` tokens; (pool, table)."""
    table, pages = S.tables(rng, lengths, P, spare, bad)
    pool = S.Pool(pages, G, P, D)
    for b, n in enumerate(lengths):
        if n:
            for w in ("k", "v"):
                pool.append(w, list(table[b]), 0, rng.standard_normal((G, n, D))
                            * np.exp2(rng.random((G, 1, 1)) * 3))
    return pool, table


def _match(cache, pool, what=""):
    for name, ref in (("k", pool.k), ("v", pool.v)):
        got = getattr(cache, name).view(torch.uint8).cpu().numpy()
        assert S.same_bytes(got, ref), f"{what} {name}: bytes differ"
    for name, ref in (("k_scale", pool.ks), ("v_scale", pool.vs)):
        got = getattr(cache, name).cpu().numpy()
        assert np.array_equal(got, ref, equal_nan=True), f"{what} {name}"


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("D,P,G,starts,T", [
    (128, 64, 2, [0, 1, 63, 64, 65, 200], 1),
    (64, 16, 3, [0, 15, 16, 31, 7], 3),
    (128, 128, 1, [0, 5, 127, 128], 128),
    (128, 128, 2, [1, 130], 300),
    (64, 32, 2, [0, 31, 33], 65),
    (64, 128, 1, [0, 100], 4),
    (128, 16, 2, [9, 0], 33),
])
def test_append(dtype, D, P, G, starts, T):
    rng = np.random.default_rng(D + P + T)
    B = len(starts)
    table, pages = S.tables(rng, [s + T for s in starts], P, 1)
    pool = S.Pool(pages, G, P, D)
    for b, s in enumerate(starts):
        if s:
            for w in ("k", "v"):
                pool.append(w, list(table[b]), 0, rng.standard_normal((G, s, D)))
    cache = E.PagedCache.of(*pool.tensors())
    k, v = _rows(rng, B, G, T, D, dtype), _rows(rng, B, G, T, D, dtype)
    E.cache_append(cache, _cuda(table), _ints(starts), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    for b, s in enumerate(starts):
        pool.append("k", list(table[b]), s, k[b].double().numpy())
        pool.append("v", list(table[b]), s, v[b].double().numpy())
    _match(cache, pool)


def test_append_token_by_token_equals_at_once():
    """The scale of a block is that of all its tokens, however they came; rescaling is exact
    (values of one magnitude: none falls below e4m3's normal range)."""
    rng = np.random.default_rng(5)
    D, P, G, T = 64, 32, 2, 70
    table, pages = S.tables(rng, [T], P)
    x = torch.from_numpy(np.sign(rng.standard_normal((1, G, T, D)))
                         * (1 + rng.random((1, G, T, D))) * np.exp2(np.arange(T) // 12)[:, None]
                         ).to(BF).cuda()
    one, many = (E.PagedCache.of(*S.Pool(pages, G, P, D).tensors()) for _ in range(2))
    E.cache_append(one, _cuda(table), _ints([0]), x, x)
    for t in range(T):
        E.cache_append(many, _cuda(table), _ints([t]), x[:, :, t:t + 1], x[:, :, t:t + 1])
    torch.cuda.synchronize()
    assert torch.equal(one.k_scale, many.k_scale) and torch.equal(one.v_scale, many.v_scale)
    used = [int(p) for p in table[0]]
    for c in (one.k, one.v), (many.k, many.v):
        pass
    for i, p in enumerate(used):
        n = min(P, T - i * P)
        for a, b in ((one.k, many.k), (one.v, many.v)):
            assert torch.equal(a.view(torch.uint8)[p, :, :n], b.view(torch.uint8)[p, :, :n])


def test_append_kept_tokens_of_strided_sources():
    """prune()'s keep_idx picks the rows; token-major keys, head-major values; counts cut;
    an index outside the source appends zeros."""
    rng = np.random.default_rng(6)
    B, G, N, T, D, P = 3, 4, 50, 20, 128, 16
    starts, counts = [3, 16, 0], [20, 7, -5]
    table, pages = S.tables(rng, [s + T for s in starts], P, 1)
    pool = S.Pool(pages, G, P, D)
    for b, s in enumerate(starts):
        if s:
            for w in ("k", "v"):
                pool.append(w, list(table[b]), 0, rng.standard_normal((G, s, D)))
    cache = E.PagedCache.of(*pool.tensors())
    k = _rows(rng, B, N, G, D, BF).cuda().transpose(1, 2)
    v = _rows(rng, B, G, N + 9, D, BF).cuda()[:, :, 4:4 + N]
    idx = np.stack([np.sort(rng.choice(N, T, replace=False)) for _ in range(B)]).astype(np.int32)
    idx[0, 4], idx[0, 5], idx[1, 0] = N, -1, 2 ** 31 - 1
    E.cache_append(cache, _cuda(table), _ints(starts), k, v, count=_ints(counts),
                   src_idx=_cuda(idx))
    torch.cuda.synchronize()
    for b in range(B):
        for w, x in (("k", k), ("v", v)):
            rows = x[b].double().cpu().numpy()[:, np.clip(idx[b], 0, N - 1)]
            rows[:, (idx[b] < 0) | (idx[b] >= N)] = 0.0
            pool.append(w, list(table[b]), starts[b], rows[:, :max(counts[b], 0)])
    _match(cache, pool)


def test_append_bad_pages_ends_and_values():
    """A page outside the pool, tokens past the table, a negative start: not written.
    NaN and infinities are held as NaN and are no maximum; zeros take the smallest scale;
    the largest and smallest magnitudes."""
    rng = np.random.default_rng(7)
    D, P, G = 64, 16, 1
    table = np.array([[2, 99, 0], [-7, 3, 1], [4, 5, 6], [7, 8, 9]], np.int32)
    pool = S.Pool(10, G, P, D)
    cache = E.PagedCache.of(*pool.tensors())
    k = _rows(rng, 4, G, 60, D, FL)
    v = k.clone()
    k[0, 0, 2, 3], k[0, 0, 3, 4], k[0, 0, 5, 6] = float("nan"), float("inf"), -float("inf")
    v[0, 0, :16] = 0.0
    v[3, 0, :16] = 3.3e38
    v[3, 0, 16:32] = 1e-38
    k[3, 0, :16] = 448.0
    k[3, 0, 1, 0] = 449.0
    starts = [0, 3, -1, 0]
    E.cache_append(cache, _cuda(table), _ints(starts), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    for b in range(4):
        pool.append("k", list(table[b]), starts[b], k[b].double().numpy())
        pool.append("v", list(table[b]), starts[b], v[b].double().numpy())
    _match(cache, pool)
    assert float(cache.v_scale[2, 0]) == 2.0 ** -100


def test_append_pages_apart_in_a_pool_of_layers():
    """The cache of one layer inside a pool [pages, layers, 2, Hkv, P, d]: page strides; the
    other layer's bytes stay."""
    rng = np.random.default_rng(8)
    D, P, G, T = 64, 16, 2, 40
    table, pages = S.tables(rng, [T], P, 3)
    raw = torch.full((pages, 2, 2, G, P, D), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.ones((2, 2, pages, G), device="cuda")
    cache = E.PagedCache.of(raw[:, 1, 0].view(S.F8), raw[:, 1, 1].view(S.F8), scales[1, 0],
                            scales[1, 1])
    k, v = _rows(rng, 1, G, T, D, BF), _rows(rng, 1, G, T, D, BF)
    E.cache_append(cache, _cuda(table), _ints([0]), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    pool = S.Pool(pages, G, P, D)
    pool.k[:], pool.v[:], pool.ks[:], pool.vs[:] = 0x55, 0x55, 1.0, 1.0
    pool.append("k", list(table[0]), 0, k[0].double().numpy())
    pool.append("v", list(table[0]), 0, v[0].double().numpy())
    _match(cache, pool)
    assert (raw[:, 0] == 0x55).all()
    q = torch.randn((1, 4, 1, D), generator=torch.Generator().manual_seed(1)).to(BF)
    _check_attend(pool, table, [T], q, cache=cache)


# ---------------------------------------------------------------------------
# attend
# ---------------------------------------------------------------------------

def _check_attend(pool, table, lengths, q, counts=None, causal=True, scale=None, max_tokens=None,
                  cache=None, weights_in=None, order="head"):
    G, D = pool.k.shape[1], pool.k.shape[3]
    B, H, T = q.shape[:3]
    cache = cache or E.PagedCache.of(*pool.tensors())
    qd = q.cuda()
    if order == "token":
        qd = qd.transpose(1, 2).contiguous().transpose(1, 2)
    max_tokens = max_tokens or max(max(lengths), 1)
    out = torch.full_like(qd, 7.0)
    w = torch.full((B, G, max_tokens + 3), -5.0, device="cuda")
    win = None if weights_in is None else _cuda(weights_in)
    call = E.CacheAttention(cache, B, H, T, max_tokens, q.dtype, scale or 0.0, causal, True)
    call(qd, _cuda(table), _ints(lengths), out, None if counts is None else _ints(counts), win, w)
    plain = E.CacheAttention(cache, B, H, T, max_tokens, q.dtype, scale or 0.0, causal)
    out2 = torch.full_like(qd, 7.0)
    plain(qd, _cuda(table), _ints(lengths), out2, None if counts is None else _ints(counts))
    torch.cuda.synchronize()
    assert torch.equal(out, out2), "the outputs depend on whether weights are returned"
    lens = [min(max(n, 0), max_tokens, table.shape[1] * pool.P) for n in lengths]
    cuts = None if counts is None else [min(max(c, 0), T) for c in counts]
    ref, rw, mag, dots, big = S.attend(pool, [list(t) for t in table], lens, q.double(), cuts,
                                       causal, scale)
    got, gw = out.double().cpu().numpy(), w.double().cpu().numpy()
    for b in range(B):
        c = T if cuts is None else cuts[b]
        assert (got[b, :, c:] == 7.0).all(), "a row behind the count was written"
        n = lens[b]
        tol = S.attend_tolerance(q.dtype, D, n, ref[b], mag[b], dots[b], big[b])
        err = np.abs(got[b] - ref[b])[:, :c]
        assert (err <= tol[:, :c]).all(), (b, float((err / tol[:, :c]).max()))
        assert (gw[b, :, n:] == -5.0).all(), "a weight behind the length was written"
        was = 0.0 if weights_in is None else weights_in[b, :, :n].astype(np.float64)
        rows = H // G * c
        rel = S.weight_error(D, n, dots[b].max(initial=0), big[b].max(initial=0)) + \
            rows * 2.0 ** -24
        # (hardware exponentials below 2^-126 are 0)
        tol = rw[b, :, :n] * rel + 2.0 ** -24 * np.abs(was + rw[b, :, :n]) + rows * 2.0 ** -125
        err = np.abs(gw[b, :, :n] - was - rw[b, :, :n])
        assert (err <= tol).all(), (b, float((err / np.maximum(tol, 1e-300)).max()))


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("D,P,G,group,T,lengths", [
    (128, 64, 4, 7, 1, [0, 1, 2, 31, 32, 33, 63, 64, 65, 300]),
    (64, 16, 2, 1, 1, [1, 15, 16, 17, 1023, 1024, 1025, 1400]),
    (128, 128, 1, 16, 1, [127, 129, 513]),
    (128, 32, 2, 17, 1, [40, 255, 257]),             # 17 rows: two tiles
    (64, 64, 1, 2, 5, [3, 4, 5, 6, 200]),            # the first queries see nothing
    (128, 16, 2, 3, 33, [10, 33, 34, 400]),          # 99 rows: several row groups
    (128, 64, 8, 1, 1, [90, 700]),
])
def test_attend(dtype, D, P, G, group, T, lengths):
    rng = np.random.default_rng(D + P + group + T)
    pool, table = _filled(rng, lengths, G, P, D, bad=1 << 30)
    q = torch.from_numpy(rng.standard_normal((len(lengths), G * group, T, D)) * 2).to(dtype)
    _check_attend(pool, table, lengths, q, order="token" if group % 2 else "head")


@pytest.mark.parametrize("dtype,D,P,causal", [(BF, 128, 64, True), (HF, 64, 16, False),
                                              (FL, 128, 32, True)])
def test_attend_many_rows(dtype, D, P, causal):
    """More than 32 rows to a key head, with ragged counts, missing pages and given weights:
    the weights' own products."""
    rng = np.random.default_rng(D + P)
    lengths, counts = [700, 33, 12, 0, 260], [13, 0, 13, 4, 7]
    pool, table = _filled(rng, lengths, 2, P, D)
    table[0, 3], table[4, 0] = -1, 1 << 29
    q = torch.from_numpy(rng.standard_normal((5, 10, 13, D)) * 2).to(dtype)
    _check_attend(pool, table, lengths, q, counts=counts, causal=causal,
                  weights_in=rng.random((5, 2, 700)).astype(np.float32))


@pytest.mark.parametrize("dtype", [BF, FL])
def test_attend_some_rows_of_many_keys(dtype):
    """17 to 32 rows where the keys are many enough that the rows are parted."""
    rng = np.random.default_rng(23)
    lengths = [33000, 700, 0, 32999]
    pool, table = _filled(rng, lengths, 1, 128, 64)
    q = torch.from_numpy(rng.standard_normal((4, 7, 3, 64))).to(dtype)
    _check_attend(pool, table, lengths, q, max_tokens=33001, counts=[3, 1, 3, 2])


def test_attend_many_splits():
    """A long sequence over many workgroups beside short ones; lengths above max_tokens are
    cut; added onto given weights."""
    rng = np.random.default_rng(20)
    lengths = [5000, 1, 0, 2600]
    pool, table = _filled(rng, lengths, 1, 64, 64)
    q = torch.from_numpy(rng.standard_normal((4, 2, 1, 64)) * 3).to(BF)
    _check_attend(pool, table, lengths, q, weights_in=rng.random((4, 1, 5000)).astype(np.float32))
    _check_attend(pool, table, [5000, 1, -4, 5000], q, max_tokens=2000)


@pytest.mark.parametrize("causal", [True, False])
def test_attend_counts_and_mask(causal):
    rng = np.random.default_rng(21)
    lengths, counts = [50, 7, 300, 12, 90], [9, 9, 0, 20, 1]
    pool, table = _filled(rng, lengths, 2, 16, 128)
    q = torch.from_numpy(rng.standard_normal((5, 6, 9, 128))).to(HF)
    _check_attend(pool, table, lengths, q, counts, causal, scale=0.3)


def test_attend_missing_pages():
    """Tokens whose page is not there are seen by no query, also at a tile's half."""
    rng = np.random.default_rng(22)
    lengths = [200, 100, 40]
    pool, table = _filled(rng, lengths, 2, 16, 64)
    table[0, 3], table[0, 4], table[0, 9], table[1, :7], table[2, 2] = -1, 999, -2 ** 31, -1, 77
    q = torch.from_numpy(rng.standard_normal((3, 4, 3, 64))).to(FL)
    _check_attend(pool, table, lengths, q)


def test_attend_nan_reaches_only_who_sees_it():
    """A NaN key or value of a late token: earlier queries of the same call are untouched,
    later ones get NaN (all dimensions for a key, one for a value)."""
    rng = np.random.default_rng(23)
    lengths = [70]
    pool, table = _filled(rng, lengths, 1, 64, 64)
    q = torch.from_numpy(rng.standard_normal((1, 2, 8, 64))).to(FL)
    _, _, mag, dots, big = S.attend(pool, [list(table[0])], lengths, q.double())
    clean, _ = E.cache_attend(q.cuda(), E.PagedCache.of(*pool.tensors()), _cuda(table),
                              _ints(lengths))
    p, r = table[0][66 // 64], 66 % 64               # token 66: seen by queries 4 .. 7
    pool.v[p, 0, r, 37] = 0x7F
    got, _ = E.cache_attend(q.cuda(), E.PagedCache.of(*pool.tensors()), _cuda(table),
                            _ints(lengths))
    assert torch.equal(got[:, :, :4], clean[:, :, :4])
    assert got[:, :, 4:, 37].isnan().all()
    rest = [i for i in range(64) if i != 37]
    assert torch.equal(got[:, :, 4:][..., rest], clean[:, :, 4:][..., rest])
    pool.v[p, 0, r, 37] = 0
    pool.k[p, 0, r, 5] = 0xFF
    got, _ = E.cache_attend(q.cuda(), E.PagedCache.of(*pool.tensors()), _cuda(table),
                            _ints(lengths))
    assert got[:, :, 4:].isnan().all() and not got[:, :, :4].isnan().any()


@pytest.mark.parametrize("length", [64, 4000])
def test_attend_all_nan_and_growing_logits(length):
    """Logits that grow along the sequence (the maximum is raised again and again), and a
    sequence of NaN keys alone, over one and over several workgroups."""
    rng = np.random.default_rng(24)
    pool, table = _filled(rng, [length], 1, 64, 64)
    q = torch.from_numpy(np.abs(rng.standard_normal((1, 3, 1, 64)))).to(FL)
    for i in range(length):
        p = table[0][i // 64]
        pool.k[p, 0, i % 64] = S.to_e4m3(np.full(64, min(448.0, i * 448.0 / length)))
        pool.ks[p, 0] = 2.0 ** -4
    _check_attend(pool, table, [length], q)
    pool.k[:] = 0x7F
    got, w = E.cache_attend(q.cuda(), E.PagedCache.of(*pool.tensors()), _cuda(table),
                            _ints([length]), want_weights=True)
    assert got.isnan().all() and w[:, :, :length].isnan().all()


def test_attend_pool_beyond_32_bits():
    """Pages more than 2^32 bytes into the pool."""
    if torch.cuda.get_device_properties(0).total_memory < 24 << 30:
        pytest.skip("needs 12 GB")
    rng = np.random.default_rng(25)
    D, P, G = 128, 128, 8
    pages = (1 << 32) // (D * P * G) + 40
    small, stable = _filled(rng, [300], G, P, D)
    big = torch.zeros((pages, G, P, D), dtype=torch.uint8, device="cuda")
    bigv = torch.zeros_like(big)
    ks, vs = torch.ones((pages, G), device="cuda"), torch.ones((pages, G), device="cuda")
    table = np.array([[pages - 1, pages - 30, pages - 7]], np.int32)
    for i in range(3):
        p = int(stable[0, i])
        big[int(table[0, i])] = _cuda(small.k[p])
        bigv[int(table[0, i])] = _cuda(small.v[p])
        ks[int(table[0, i])], vs[int(table[0, i])] = _cuda(small.ks[p]), _cuda(small.vs[p])
    q = torch.from_numpy(rng.standard_normal((1, 8, 1, 128))).to(BF)
    cache = E.PagedCache.of(big.view(S.F8), bigv.view(S.F8), ks, vs)
    got, _ = E.cache_attend(q.cuda(), cache, _cuda(table), _ints([300]))
    ref, _ = E.cache_attend(q.cuda(), E.PagedCache.of(*small.tensors()), _cuda(stable),
                            _ints([300]))
    assert torch.equal(got, ref)


# ---------------------------------------------------------------------------
# evict
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("D,P,G,lengths,K,sinks,recent", [
    (128, 64, 2, [0, 1, 99, 100, 101, 700], 100, 4, 16),
    (64, 16, 3, [5, 40, 1200], 1, 0, 0),
    (64, 16, 1, [2000, 33], 17, 1, 16),              # no token to choose
    (128, 128, 2, [3000, 129], 400, 0, 100),
    (64, 32, 1, [90, 64], 64, 10, 0),
    (128, 64, 1, [20000], 5000, 4, 1000),
])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict(D, P, G, lengths, K, sinks, recent, kind):
    rng = np.random.default_rng(D + P + K)
    B = len(lengths)
    both, pages = S.tables(rng, lengths + [K] * B, P, 1)
    pool = S.Pool(pages, G, P, D)
    for b, n in enumerate(lengths):
        if n:
            for w in ("k", "v"):
                pool.append(w, list(both[b]), 0, rng.standard_normal((G, n, D))
                            * np.exp2(rng.random((G, n, 1)) * 12))
    N = max(lengths)
    if kind == "ties":
        w = rng.integers(0, 4, (B, G, N)).astype(np.float32) / 4
        w[rng.random(w.shape) < 0.1] = -0.0
        w[rng.random(w.shape) < 0.02] = np.nan
        w[rng.random(w.shape) < 0.02] = np.inf
        w[rng.random(w.shape) < 0.02] = -np.inf
    else:
        w = np.exp(2 * rng.standard_normal((B, G, N))).astype(np.float32)
    table, new = both[:B], both[B:]
    cache = E.PagedCache.of(*pool.tensors())
    left = torch.full((B, G, K + 5), 3.0, device="cuda")
    keep, kept, left2 = E.cache_evict(cache, _cuda(table), _ints(lengths), _cuda(w), _cuda(new), K,
                                      sinks, recent, weights_left=left)
    torch.cuda.synchronize()
    assert left2 is left
    assert kept.tolist() == [min(n, K) for n in lengths]
    keep, left = keep.cpu().numpy(), left.cpu().numpy()
    old = {"k": pool.k.copy(), "v": pool.v.copy()}, {"k": pool.ks.copy(), "v": pool.vs.copy()}
    for b, n in enumerate(lengths):
        for g in range(G):
            idx = S.evict(w[b, g], n, K, sinks, recent)
            assert keep[b, g].tolist() == idx + [-1] * (K - len(idx)), (b, g)
            assert np.array_equal(left[b, g, :len(idx)], w[b, g, idx], equal_nan=True)
            assert (left[b, g, len(idx):] == 0).all()
            for which in ("k", "v"):
                x, s = (pool.k, pool.ks) if which == "k" else (pool.v, pool.vs)
                for blk in range(-(-len(idx) // P)):
                    part = idx[blk * P:(blk + 1) * P]
                    src = [both[b][i // P] for i in part]
                    rows = np.stack([S._VALUES[old[0][which][p, g, i % P]]
                                     * float(old[1][which][p, g]) for p, i in zip(src, part)])
                    sc = S.block_scale(np.abs(rows).max())
                    x[new[b][blk], g, :len(part)] = S.to_e4m3(rows / sc)
                    s[new[b][blk], g] = sc
    _match(cache, pool)


def test_evict_missing_pages_and_nan():
    """A kept row whose page is not there becomes zeros, a new page that is not there is not
    written; NaN bytes move as NaN and are no maximum."""
    rng = np.random.default_rng(31)
    D, P, G = 64, 16, 1
    pool, table = _filled(rng, [64, 64], G, P, D, spare=6)
    free = [p for p in range(pool.k.shape[0]) if p not in set(table.ravel().tolist())]
    table[0, 1] = 500
    new = np.array([[free[0], free[1]], [free[2], -3]], np.int32)
    src = table[1][0]
    pool.k[src, 0, 3, 7] = 0xFF
    w = np.arange(64, dtype=np.float32)[None, None].repeat(2, 0)
    w[1] = -w[1]
    cache = E.PagedCache.of(*pool.tensors())
    keep, _, _ = E.cache_evict(cache, _cuda(table), _ints([64, 64]), _cuda(w), _cuda(new), 32,
                               sinks=20)
    torch.cuda.synchronize()
    got = cache.k.view(torch.uint8).cpu().numpy()
    assert keep[0, 0].tolist() == list(range(20)) + list(range(52, 64))
    assert (got[free[0], 0] == pool.k[table[0, 0], 0]).all()
    assert (got[free[1], 0, :4] == 0).all()          # tokens 16 .. 19: the missing page
    assert keep[1, 0].tolist() == list(range(32))
    assert (got[free[2], 0, 3, 7] & 0x7F) == 0x7F
    keepable = [p for p in range(pool.k.shape[0]) if p not in (free[0], free[1], free[2])]
    assert S.same_bytes(got[keepable], pool.k[keepable])


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def _generate(steps, capture=False):
    """Prune an image, put the kept tokens' rotated keys into the cache, decode with
    accumulated weights, evict, go on: what a serving loop does."""
    g = torch.Generator(device="cuda").manual_seed(77)
    B, H, G, D, P, gh, K, T = 2, 8, 2, 128, 16, 12, 40, 6
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF)       # noqa: E731
    plan = E.rotary_plan(D, base=1e6, sections=(16, 24, 24))
    at = torch.arange(gh * gh, device="cuda", dtype=torch.int32)
    vis = torch.stack([torch.zeros_like(at), at // gh, at % gh])
    txt = (gh + torch.arange(T, device="cuda", dtype=torch.int32)).expand(3, T)
    kv, vv = rnd(B, gh * gh, G, D).transpose(1, 2), rnd(B, gh * gh, G, D).transpose(1, 2)
    qt, kt, vt = rnd(B, H, T, D), rnd(B, G, T, D), rnd(B, G, T, D)
    _, kv = E.rotate_positions(None, kv, vis, plan)
    qt, kt = E.rotate_positions(qt, kt, txt, plan)
    keep, _, _ = E.prune_views([qt], [kv], gh, gh, K)
    budget = 48
    pages = torch.randperm(16, generator=g, device="cuda").to(torch.int32).view(B, 8)
    table, fresh = pages[:, :5].contiguous(), pages[:, 5:].contiguous()
    cache = E.PagedCache(16, G, D, P)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    E.cache_append(cache, table, zero, kv, vv, src_idx=keep)
    E.cache_append(cache, table, zero + K, kt, vt)
    length = zero + K + T
    acc = torch.zeros((B, G, 80), device="cuda")
    outs = [E.cache_attend(qt, cache, table, length, 80, weights_in=acc, weights_out=acc)[0]]
    one = E.CacheAttention(cache, B, H, 1, 80, BF, weights=True)
    for s in range(steps):
        if s == steps // 2:
            _, length, acc2 = E.cache_evict(cache, table, length, acc, fresh, budget, 4, 8)
            acc = torch.zeros_like(acc)
            acc[:, :, :budget] = acc2
            table = fresh
        pos = (length + 20).view(1, B, 1).expand(3, B, 1)
        q, k = E.rotate_positions(rnd(B, H, 1, D), rnd(B, G, 1, D), pos, plan)
        E.cache_append(cache, table, length, k, rnd(B, G, 1, D))
        length = length + 1
        outs.append(one(q, table, length, weights_in=acc, weights_out=acc)[0])
    torch.cuda.synchronize()
    return outs, acc, length, cache, table


def test_a_serving_loop():
    outs, acc, length, cache, table = _generate(12)
    assert all(bool(torch.isfinite(o.float()).all()) for o in outs)
    # 46 tokens, 6 steps to 52, cut to 48, 6 more
    assert length.tolist() == [54, 54]
    # every query of every head gave its weight of 1 to some token; what eviction dropped is gone
    total = acc.sum((1, 2))
    assert bool((total > 0).all()) and bool((acc[:, :, 54:] == 0).all())
    again = _generate(12)
    assert all(torch.equal(a, b) for a, b in zip(outs, again[0])), "not the same twice"
    assert torch.equal(acc, again[1])
    # and the cache holds what the last outputs say: one more step against float64
    pool = S.Pool(16, 2, 16, 128)
    pool.k, pool.v = (t.view(torch.uint8).cpu().numpy() for t in (cache.k, cache.v))
    pool.ks, pool.vs = cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
    q = torch.randn((2, 8, 1, 128), generator=torch.Generator().manual_seed(2)).to(BF)
    _check_attend(pool, table.cpu().numpy(), [54, 54], q, cache=cache)


def test_captured_steps_replay_exactly():
    """Rotate, append, attend and evict captured in one graph: replays on new inputs equal
    eager calls, with eager work between."""
    B, H, G, D, P, n = 2, 6, 2, 64, 16, 300
    rng = np.random.default_rng(41)
    pool, table = _filled(rng, [n + 1] * B, G, P, D, spare=2 * 4)
    free = [p for p in range(pool.k.shape[0]) if p not in set(table.ravel().tolist())]
    new = np.array(free[:8], np.int32).reshape(2, 4)
    inputs = [[_rows(np.random.default_rng(50 + i), B, h, 1, D, HF).cuda() for h in (H, G, G)]
              for i in range(3)]
    q, k, v = (x.clone() for x in inputs[0])
    plan = E.rotary_plan(D, rot_dim=32)
    start, length = _ints([n, n - 40]), _ints([n + 1, n - 39])
    pages, fresh = _cuda(table), _cuda(new)

    def make():
        cache = E.PagedCache.of(*pool.tensors())
        return cache, E.CacheAttention(cache, B, H, 1, 320, HF, weights=True)

    def step(cache, att, q, k, v):
        qr, kr = E.rotate_positions(q, k, start.view(B, 1), plan)
        E.cache_append(cache, pages, start, kr, v)
        out, w = att(qr, pages, length)
        keep, kept, left = E.cache_evict(cache, pages, length, w, fresh, 60, 2, 5)
        return out, w, keep, kept, left, cache.k.view(torch.uint8), cache.k_scale

    cache, att = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, att, q, k, v)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache, att, q, k, v)
    first = [t.clone() for t in (cache.k.view(torch.uint8), cache.v.view(torch.uint8),
                                 cache.k_scale, cache.v_scale)]
    for rep in range(6):
        for t, s in zip((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale,
                         cache.v_scale), first):
            t.copy_(s)
        for t, s in zip((q, k, v), inputs[rep % 3]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        here = [t.clone() for t in got]
        c2 = E.PagedCache.of(first[0].clone().view(S.F8), first[1].clone().view(S.F8),
                             first[2].clone(), first[3].clone())
        want = step(c2, E.CacheAttention(c2, B, H, 1, 320, HF, weights=True), *inputs[rep % 3])
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(here, want)):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)), (rep, i)


def test_on_another_stream():
    rng = np.random.default_rng(42)
    pool, table = _filled(rng, [500], 2, 32, 128)
    q = torch.from_numpy(rng.standard_normal((1, 4, 1, 128))).to(BF).cuda()
    cache = E.PagedCache.of(*pool.tensors())
    want, _ = E.cache_attend(q, cache, _cuda(table), _ints([500]))
    pages, lengths = _cuda(table), _ints([500])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, _ = E.cache_attend(q, cache, pages, lengths)
    s.synchronize()
    assert torch.equal(got, want)


def test_on_a_given_stream():
    """`stream` without entering it: what the calls allocate and fill belongs to it."""
    rng = np.random.default_rng(43)
    pool, table = _filled(rng, [500, 90], 2, 32, 128, spare=4)
    q = torch.from_numpy(rng.standard_normal((2, 4, 3, 128))).to(BF).cuda()
    cache = E.PagedCache.of(*pool.tensors())
    free = [p for p in range(pool.k.shape[0]) if p not in set(table.ravel().tolist())]
    fresh = _cuda(np.array(free[:4], np.int32).reshape(2, 2))
    pages, lengths, counts = _cuda(table), _ints([500, 90]), _ints([3, 1])
    att = E.CacheAttention(cache, 2, 4, 3, 512, weights=True)
    out, w = att(q, pages, lengths, q_count=counts)
    keep, kept, left = E.cache_evict(cache, pages, lengths, w, fresh, 40, 2, 5)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out2, w2 = att(q, pages, lengths, q_count=counts, stream=s.cuda_stream)
    s.synchronize()
    k2, n2, left2 = E.cache_evict(cache, pages, lengths, w2, fresh, 40, 2, 5,
                                  stream=s.cuda_stream)
    s.synchronize()
    for a, b in ((out, out2), (w, w2), (keep, k2), (kept, n2), (left, left2)):
        assert torch.equal(a, b)


def test_no_empty_cache():
    with pytest.raises(ValueError):
        E.PagedCache(0, 2, 64, 16)
