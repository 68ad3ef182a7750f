"""GPU checks that reach every kernel of the 4-bit attention's dispatch (the calls of
_step_variants.py, whose plans test_step_plan.py holds to their kernels), every sequence and
head against float64; and the longest sequence and a pool that 32 bits do not number.

What nothing wrote has NaN scales, and unused entries of the page tables name no page."""
import numpy as np
import pytest
import torch

import _serve_helpers as R
import _step_helpers as H
import _step_variants as V
import paper_2608_23253_amd as E

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def random_tables(seed, pages, G, P, d):
    """Any codes; key scales of 1/8 to 1, value scales of 1/4 to 2 with any mantissa."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def whole(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda")
    k = whole(0, 256, pages, G, P, d // 2).to(torch.uint8)
    v = whole(0, 256, pages, G, P // 32, d, 16).to(torch.uint8)
    ks = whole(124, 128, pages, G, P // 16, 4, d // 32, 4).to(torch.uint8)
    vs = (1 + whole(0, 128, pages, G, P) / 128.0) * torch.exp2(whole(-2, 1, pages, G, P).float())
    return k, ks, v, vs.to(torch.bfloat16)


def sequences(seed, lengths, G, P, d, width):
    """Tables and a page table of `width` columns; tokens behind a sequence have NaN scales."""
    table, pages = R.tables(np.random.default_rng(seed), lengths, P, 2)
    wide = np.full((len(lengths), width), -1, np.int32)
    wide[:, :table.shape[1]] = table
    written = np.zeros((pages, P), bool)
    for b, n in enumerate(lengths):
        for i in range(-(-n // P)):
            written[table[b, i], :min(P, n - i * P)] = True
    k, ks, v, vs = random_tables(seed, pages, G, P, d)
    live = torch.from_numpy(written).cuda()
    vs.masked_fill_(~live[:, None], float("nan"))
    tokens = live.view(pages, 1, P // 16, 4, 4, 1).permute(0, 1, 2, 4, 5, 3)     # n, u, r -> n, r, u
    ks.masked_fill_(~tokens, 255)
    return (k, ks, v, vs), wide


def compare(out, ref, tol, what):
    err = (out.double() - ref).abs()
    bad = ~(err <= tol)
    if bool(bad.any()):
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError((what, at, float(out[at]), float(ref[at]), float(tol[at]),
                              int(bad.sum())))


@pytest.mark.parametrize("d", V.HEAD_DIMS)
@pytest.mark.parametrize("kind", V.DTYPES)
@pytest.mark.parametrize("name", V.CALLS)
def test_every_kernel(name, kind, d):
    c = V.CALLS[name]
    B, Hq, G, T, P = c["batch"], c["heads"], c["kv_heads"], c["queries"], c["page"]
    lengths = V.lengths_of(c)
    counts, causal = c.get("counts"), c.get("causal", True)
    tables, pages = sequences(21, lengths, G, P, d, -(-c["max_tokens"] // P))
    for b, token in c.get("missing", ()):
        pages[b, token // P] = (-1, 1 << 30)[token % 2]
    g = torch.Generator(device="cuda").manual_seed(22)
    q = torch.randn((B, T, Hq, d), generator=g, device="cuda")
    q = (q * torch.exp2(2 * torch.rand((B, T, Hq, 1), generator=g, device="cuda") - 1))
    q = q.to(H.DTYPES[kind]).transpose(1, 2)
    out = torch.full_like(q, 7.0)
    E.cache4_attend(q, E.PagedCache4.of(*tables), ints(pages), ints(lengths),
                    max_tokens=c["max_tokens"], causal=causal, out=out,
                    q_count=None if counts is None else ints(counts))
    for b in range(B):
        n = T if counts is None else counts[b]
        held = H.held_rows(tables, torch.from_numpy(pages[b]), lengths[b])
        ref, tol = H.attend_rows(held, q[b].double(), n, kind, causal)
        compare(out[b, :, :n], ref[:, :n], tol[:, :n], f"sequence {b}")
        assert bool((out[b, :, n:] == 7).all())


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_the_longest_sequence(kind, d):
    """2^20 tokens of three pages in turn."""
    n, P, G, Hq, T = 1 << 20, 128, 1, 3, 2
    tables = random_tables(23, 3, G, P, d)
    pages = np.arange(n // P, dtype=np.int32)[None] % 3
    pages[0, 5000] = -1
    q = torch.randn((1, Hq, T, d), generator=torch.Generator(device="cuda").manual_seed(24),
                    device="cuda").to(H.DTYPES[kind])
    out = E.cache4_attend(q, E.PagedCache4.of(*tables), ints(pages), ints([n]))
    held = H.held_rows(tables, torch.from_numpy(pages[0]), n)
    ref, tol = H.attend_rows(held, q[0].double(), T, kind)
    compare(out[0], ref, tol, kind)


def test_pages_further_apart_than_32_bits_number():
    """Four pages of k and of v 2.3 GB apart: tokens appended, read and attended to, as in pages
    side by side."""
    pages, G, P, d, gap = 4, 2, 64, 128, (1 << 31) + (1 << 28)
    size = G * P * d // 2
    big = torch.empty(pages * gap, dtype=torch.uint8, device="cuda")
    far = [big[at:].as_strided((pages, *shape), (gap, *torch.empty(shape).stride()))
           for at, shape in ((0, (G, P, d // 2)), (size, (G, P // 32, d, 16)))]
    k, ks, v, vs = random_tables(25, pages, G, P, d)
    far[0].copy_(k)
    far[1].copy_(v)
    near, apart = E.PagedCache4.of(k, ks, v, vs), E.PagedCache4.of(far[0], ks.clone(), far[1],
                                                                   vs.clone())
    g = torch.Generator(device="cuda").manual_seed(26)
    new = torch.randn((1, G, 70, d), generator=g, device="cuda").bfloat16()
    q = torch.randn((1, 4, 1, d), generator=g, device="cuda").bfloat16()
    table, start, n = ints([[2, 0, 3, 1]]), ints([150]), ints([220])
    got = []
    for cache in (near, apart):
        E.cache4_append(cache, table, start, new, -new)
        got.append((*E.cache4_read(cache, table, ints([0]), 256, dtype=torch.float32),
                    E.cache4_attend(q, cache, table, n)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(apart.k, near.k) and torch.equal(apart.v, near.v)
    held = H.held_rows((k, ks, v, vs), table[0], 220)
    ref, tol = H.attend_rows(held, q[0].double(), 1, "bf16")
    compare(got[0][2][0], ref, tol, "bf16")
