"""GPU checks of the operators of e2s_serve.h as programs run them: two calls at once,
captured and replayed calls of every way to part the work, a source row used twice, and the
longest sequences that the header allows."""
import numpy as np
import pytest

import _serve_helpers as S
from test_gpu_cache import _cuda, _ints, _match, _rows
from test_gpu_cache_variants import DTYPES, _pool, _reference

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E = pytest.importorskip("paper_2608_23253_amd")

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32

# dtype, batch, heads, kv_heads, queries, head_dim, max_tokens, lengths: one workgroup of eight
# waves, few and many parts, a launch for the weights, rows parted in 16 and in 32 to a wave
CALLS = {
    "eight waves": ("bf16", 2, 8, 2, 1, 128, 500, [500, 40]),
    "few parts": ("f16", 20, 32, 8, 1, 128, 3000, [3000, 1500] + [70] * 18),
    "many parts": ("f32", 2, 8, 2, 1, 64, 9000, [9000, 10]),
    "full": ("bf16", 128, 8, 8, 2, 64, 300, [300, 1] + [64] * 126),
    "rows": ("bf16", 2, 14, 2, 20, 128, 2500, [2500, 30]),
    "many rows": ("bf16", 8, 64, 64, 70, 64, 200, [200, 70] + [90] * 6),
}


def _setup(name, seed):
    dt, B, H, G, T, D, N, lengths = CALLS[name]
    cache, table = _pool(seed, lengths, G, 32, D, -(-N // 32))
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((B, H, T, D), generator=g, device="cuda").to(DTYPES[dt])
    return cache, table, _ints(lengths), q, lambda: E.CacheAttention(
        cache, B, H, T, N, DTYPES[dt], weights=True)


@pytest.mark.parametrize("name", CALLS)
def test_captured_attention_replays_exactly(name):
    """Several replays on changing queries and lengths, each against an eager call, with eager
    work between them; weights added up in place."""
    cache, table, lengths, q, make = _setup(name, 3)
    att = make()
    B, H, G = q.shape[0], q.shape[1], cache.num_kv_heads
    acc = torch.zeros((B, G, att.max_tokens), device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        att(q, table, lengths, out, weights_in=acc, weights_out=acc)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(q, table, lengths, out, weights_in=acc, weights_out=acc)
    acc.zero_()
    full, other = lengths.clone(), make()
    want = torch.zeros_like(acc)
    for rep in range(5):
        q.copy_(torch.randn(q.shape, device="cuda", generator=torch.Generator("cuda")
                            .manual_seed(rep)))
        lengths.copy_(full - torch.arange(B, device="cuda", dtype=torch.int32) % (rep + 1))
        lengths.clamp_(min=0)
        eager, _ = other(q, table, lengths, weights_in=want, weights_out=want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), rep
        assert torch.equal(acc, want), rep


def test_two_calls_at_once():
    """Each pair of kinds on two streams, again and again: as one after the other."""
    names = list(CALLS)
    sets = {n: _setup(n, 7) for n in names}
    calls = {n: s[4]() for n, s in sets.items()}
    want = {n: calls[n](s[3], s[1], s[2]) for n, s in sets.items()}
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for x, y in zip(names, names[1:] + names[:1]):
        got = []
        for _ in range(4):
            for n, st in ((x, a), (y, b)):
                with torch.cuda.stream(st):
                    got.append((n, calls[n](sets[n][3], sets[n][1], sets[n][2])))
        torch.cuda.synchronize()
        for n, (out, w) in got:
            assert torch.equal(out, want[n][0]) and torch.equal(w, want[n][1]), (x, y)


def test_append_a_source_row_twice():
    rng = np.random.default_rng(61)
    D, P, G, N = 64, 16, 2, 7
    idx = np.array([[3, 3, 0, 6, 3, 6, 6, 1, 1, 0, 5, 5, 5, 5, 2, 4, 4, 3, 3, 3]], np.int32)
    table, pages = S.tables(rng, [idx.size], P, 1)
    pool = S.Pool(pages, G, P, D)
    cache = E.PagedCache.of(*pool.tensors())
    k, v = _rows(rng, 1, G, N, D, HF), _rows(rng, 1, G, N, D, HF)
    E.cache_append(cache, _cuda(table), _ints([0]), k.cuda(), v.cuda(), src_idx=_cuda(idx))
    torch.cuda.synchronize()
    pool.append("k", list(table[0]), 0, k[0].double().numpy()[:, idx[0]])
    pool.append("v", list(table[0]), 0, v[0].double().numpy()[:, idx[0]])
    _match(cache, pool)


def test_the_longest_sequence():
    """2^20 tokens: appended in two calls, attended to with their weights, cut to some."""
    N, D, P, K = 1 << 20, 64, 128, 5000
    g = torch.Generator(device="cuda").manual_seed(8)
    pages = N // P
    perm = torch.randperm(pages + 40, generator=g, device="cuda").to(torch.int32)
    table, new = perm[None, :pages].contiguous(), perm[None, pages:].contiguous()
    cache = E.PagedCache(pages + 40, 1, D, P)
    k, v = (torch.randn((1, 1, N, D), generator=g, device="cuda").to(BF) for _ in range(2))
    half = N // 2 + 33
    E.cache_append(cache, table, _ints([0]), k[:, :, :half], v[:, :, :half])
    E.cache_append(cache, table, _ints([half]), k[:, :, half:], v[:, :, half:])
    i = torch.arange(N, device="cuda")
    for x, held, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        page = table[0].long()[i // P]
        row = held.view(torch.uint8)[page, 0, i % P].view(S.F8).double()
        s = scale[page, 0].double()[:, None]
        # a half step of 4 bits, or of the smallest numbers
        assert bool(((row * s - x[0, 0].double()).abs()
                     <= torch.maximum(2.0 ** -4 * x[0, 0].double().abs(), 2.0 ** -10 * s)).all())
    q = (torch.randn((1, 2, 2, D), generator=g, device="cuda") * 2).to(FL)
    out, w = E.cache_attend(q, cache, table, _ints([N]), max_tokens=N, want_weights=True)
    ref, rw, mag, dots, big = _reference(cache, table[0], N, 0, q[0].double(), True)
    tol = S.attend_tolerance(FL, D, N, ref, mag, dots, big)
    assert (np.abs(out[0].double().cpu().numpy() - ref) <= tol).all()
    rel = S.weight_error(D, N, dots.max(), big.max()) + 4 * 2.0 ** -24
    assert (np.abs(w[0, 0].double().cpu().numpy() - rw) <= rw * rel + 4 * 2.0 ** -125).all()
    keep, kept, left = E.cache_evict(cache, table, _ints([N]), w, new, K, 4, 100)
    assert kept.tolist() == [K]
    host = w[0, 0, 4:N - 100].double().cpu().numpy()
    order = np.lexsort((np.arange(host.size), -host))[:K - 104] + 4
    idx = np.sort(np.concatenate([np.arange(4), order, np.arange(N - 100, N)]))
    assert np.array_equal(keep[0, 0].cpu().numpy(), idx)
    assert torch.equal(left[0, 0], w[0, 0, torch.from_numpy(idx).cuda()])
