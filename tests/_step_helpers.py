"""Plain implementations, in float64 on the CPU, of the operators of e2s_step.h, and the
tolerances that their arithmetic gives."""
import math

import numpy as np
import torch

import _serve_helpers as R

LOWEST = -100
U = 2.0 ** -24                          # half a step of float32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# norms and positions
# ---------------------------------------------------------------------------

def pair_sum(x, rot, layout):
    """|x0| + |x1| of every turned pair at both its elements; |x| of the others."""
    out, a, half = x.abs().clone(), x[..., :rot].abs(), rot // 2
    if layout == "half":
        both = a[..., :half] + a[..., half:]
        out[..., :half], out[..., half:rot] = both, both
    else:
        both = a[..., 0::2] + a[..., 1::2]
        out[..., 0:rot:2], out[..., 1:rot:2] = both, both
    return out


def norm_rotate(x, w, positions, f, eps, axis=None, layout="half", amplitude=1.0):
    """x [B, H, T, d], w [d] float64 (or None): the result, and what is turned."""
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    y = y if w is None else y * w
    return R.rotate(y, positions, f, axis, layout, amplitude), y


def norm_tolerance(ref, y, rot, layout, dtype, amplitude=1.0):
    """One rounding of the result.  Float32's before the rotation: of the squares' sum, 16 of
    them in a lane and 6 steps across, halved by the root (11), of the mean and eps (1), of
    root and quotient (2), of the two products (2): 16 half steps of y; and the rotation's 8 of
    a pair's sum."""
    return (R.HALF_STEP[dtype] * torch.clamp(ref.abs(), min=R.TINY[dtype]) +
            24 * U * amplitude * pair_sum(y, rot, layout))


def norm_back(g, x, w, positions, f, eps, axis=None, layout="half", amplitude=1.0):
    """(dx, dw, and the sizes that the tolerances need) by the formula."""
    gb = R.rotate(g, positions, f, axis, layout, amplitude, inverse=True)
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    unit = x * r
    wt = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w
    u = gb * wt
    mean = (u * unit).mean(-1, keepdim=True)
    return r * (u - unit * mean), (gb * unit).sum((0, 1, 2)), dict(gb=gb, r=r, unit=unit, wt=wt,
                                                                   u=u, mean=mean)


def back_tolerances(dx, dw, g, z, rot, layout, dtype, wdtype, amplitude=1.0):
    """The gradient of what was turned, gb: 8 half steps of a pair's sum (rotation).  The dot
    product: one more for w, 24 for its sum (16 in a lane, 6 across, the products), 16 for r,
    all of sum |u unit|, and gb's.  dx: that mean times unit (17 more), u times r (17).  dw:
    gb's, unit's 17 and the sum's: at most as many additions as rows, of a thread, and 150 of
    the joins."""
    eg = 8 * U * amplitude * pair_sum(g, rot, layout)
    eu = eg * z["wt"].abs() + U * z["u"].abs()
    uu = (z["u"] * z["unit"]).abs()
    em = (eu * z["unit"].abs() + 41 * U * uu).mean(-1, keepdim=True)
    tx = (R.HALF_STEP[dtype] * torch.clamp(dx.abs(), min=R.TINY[dtype]) +
          z["r"] * (eu + 18 * U * z["u"].abs() + z["unit"].abs() * em +
                    20 * U * (z["unit"] * z["mean"]).abs()))
    rows = g.shape[0] * g.shape[1] * g.shape[2]
    size = (z["gb"] * z["unit"]).abs().sum((0, 1, 2))
    tw = (R.HALF_STEP[wdtype] * torch.clamp(dw.abs(), min=R.TINY[wdtype]) +
          (17 + min(rows, 4096) + 150) * U * size + (eg * z["unit"].abs()).sum((0, 1, 2)))
    return tx, tw


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------

def to_codes(y):
    """Elements over their scale, float64: nearest, ties to the even code; sign in bit 3."""
    m = np.minimum(np.abs(y), 6.0)
    hi = np.clip(np.searchsorted(GRID, m), 1, 7)
    lo = hi - 1
    down, up = m - GRID[lo], GRID[hi] - m
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    return code.astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)


def key_exponent(m):
    """The byte of a block whose largest magnitude is m."""
    if not math.isfinite(m):
        return 255
    e = LOWEST
    if m > 0:
        e = math.frexp(m)[1] - 4
        while 6.0 * 2.0 ** e < m:
            e += 1
    return max(e, LOWEST) + 127


def value_scale(m):
    if not math.isfinite(m):
        return math.nan
    if m == 0:
        return 2.0 ** LOWEST
    f, x = math.frexp(m)
    n = int(f * 2 ** 40)                 # m = n 2^(x - 40), and m / 6 in [85, 171) 2^(x - 10)
    for shift in (11, 10):               # the finer 8-bit grid where it reaches
        c = -(-n // (6 * 2 ** (40 - shift)))
        if c <= 256:
            return max(math.ldexp(c, x - shift), 2.0 ** LOWEST)
    raise AssertionError(m)


class Pool4:
    """The tables as numpy arrays; what nothing wrote is 0xFF: NaN scales."""

    def __init__(self, pages, G, P, D):
        self.k = np.full((pages, G, P, D // 2), 0xFF, np.uint8)
        self.v = np.full((pages, G, P // 32, D, 16), 0xFF, np.uint8)
        self.ks = np.full((pages, G, P // 16, 4, D // 32, 4), 0xFF, np.uint8)
        self.vs = np.full((pages, G, P), np.nan, np.float32)
        self.P, self.D = P, D

    def tensors(self, device="cuda"):
        k, ks, v = (torch.from_numpy(x.copy()).to(device) for x in (self.k, self.ks, self.v))
        return k, ks, v, torch.from_numpy(self.vs.copy()).to(device).to(torch.bfloat16)

    def put(self, p, g, r, key, value):
        """One token's float64 key and value at row r of a page."""
        D = self.D
        blocks = key.reshape(D // 32, 32)
        for c in range(D // 32):
            e = key_exponent(np.abs(blocks[c]).max() if np.isfinite(blocks[c]).all() else math.inf)
            self.ks[p, g, r // 16, r % 4, c, r % 16 // 4] = e
            if e != 255:
                q = to_codes(blocks[c] / 2.0 ** (e - 127))
                self.k[p, g, r, 16 * c:16 * c + 16] = q[0::2] | (q[1::2] << 4)
        s = value_scale(np.abs(value).max() if np.isfinite(value).all() else math.inf)
        self.vs[p, g, r] = s
        if not math.isnan(s):
            q, i = to_codes(value / s), r % 32 // 2
            b = self.v[p, g, r // 32, :, i]
            self.v[p, g, r // 32, :, i] = ((b & 0x0F) | (q << 4)) if r % 2 else ((b & 0xF0) | q)

    def append(self, table, start, k, v):
        """k, v [G, n, D] float64 as tokens start ..; tokens without a page are not written."""
        for j in range(k.shape[1] if start >= 0 else 0):
            n = start + j
            if n >= len(table) * self.P or not 0 <= table[n // self.P] < self.k.shape[0]:
                continue
            for g in range(k.shape[0]):
                self.put(table[n // self.P], g, n % self.P, k[g, j], v[g, j])

    def row(self, which, p, g, r):
        D = self.D
        signed = np.concatenate([GRID, -GRID])
        if which == "k":
            b = self.k[p, g, r]
            q = np.stack([b & 15, b >> 4], -1).reshape(D)
            e = self.ks[p, g, r // 16, r % 4, :, r % 16 // 4].astype(np.float64)
            s = np.where(e == 255, np.nan, 2.0 ** (e - 127))
            return signed[q] * np.repeat(s, 32)
        b = self.v[p, g, r // 32, :, r % 32 // 2]
        return signed[(b >> 4) if r % 2 else (b & 15)] * float(self.vs[p, g, r])

    def rows(self, which, table, n, g):
        """The first n cached rows of a sequence and head; NaN where there is no page."""
        out = np.full((n, self.D), np.nan)
        for i in range(n):
            p = table[i // self.P] if i // self.P < len(table) else -1
            if 0 <= p < self.k.shape[0]:
                out[i] = self.row(which, p, g, i % self.P)
        return out


def same_tables(pool, got):
    """The tables `got` (k, ks, v, vs numpy, vs float32) hold what the pool does: the same
    scales everywhere, and the same bytes but for codes under a NaN scale."""
    k, ks, v, vs = got
    assert np.array_equal(ks, pool.ks)
    assert np.array_equal(vs, pool.vs, equal_nan=True)
    live = pool.ks != 255                                # [p, G, P/16, r, c, u]
    p, G, n, _, c, _ = live.shape
    live = live.transpose(0, 1, 2, 5, 3, 4).reshape(p, G, n * 16, c)
    assert np.array_equal(np.where(np.repeat(live, 16, -1), k, 0),
                          np.where(np.repeat(live, 16, -1), pool.k, 0))
    one = (~np.isnan(pool.vs)).reshape(p, G, -1, 1, 16, 2).astype(np.uint8)
    mask = one[..., 0] * 15 + one[..., 1] * 240
    assert np.array_equal(v & mask, pool.v & mask)


# Terms of 4 bits on a scale that takes the largest to 1.93 .. 3.88, each the last one's residual
# on a scale 2^-4 of its: n terms hold 4 n bits, or, e4m3's smallest step being 2^-9, leave half
# of 2^-9 2^-4(n - 1) of a largest that is near 2 at least: 2^-11 - 4 (n - 1) of it, and 4%.
# n = 2, 3, 6 for queries, 3, 4, 6 for weights.
Q_FLOOR = {"bf16": 1.04 * 2.0 ** -15, "f16": 1.04 * 2.0 ** -19, "f32": 1.04 * 2.0 ** -31}
P_STEP = {"bf16": 2.0 ** -12, "f16": 2.0 ** -16, "f32": 2.0 ** -24}
P_FLOOR = {"bf16": 1.04 * 2.0 ** -19, "f16": 1.04 * 2.0 ** -23, "f32": 1.04 * 2.0 ** -31}


def attend(pool, table, lengths, q, kind, counts=None, causal=True, scale=None):
    """q [B, H, T, d] float64: outputs, and their tolerances for queries of type `kind`.

    A logit: d float32 additions over sum |q k|, what the queries' terms leave of an element
    (Q_FLOOR of its block's largest, times sum |k|), and 4 roundings of its own size in log2.
    A weight: that, the exponential's 2^-22 and the sum's (N / 32 + 64 additions), twice over
    for numerator and denominator, and the rounding of what multiplies the codes: P_STEP of
    it, or P_FLOOR of the largest of its 128 keys."""
    B, H, T, D = q.shape
    G, P = pool.k.shape[1], pool.P
    scale = D ** -0.5 if scale is None else scale
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    half = R.HALF_STEP[DTYPES[kind]]
    q = q.numpy()
    for b in range(B):
        n = max(0, min(lengths[b], len(table[b]) * P))
        c = T if counts is None else max(0, min(counts[b], T))
        there = np.array([0 <= table[b][i // P] < pool.k.shape[0] for i in range(n)], bool)
        for g in range(G):
            k, v = pool.rows("k", table[b], n, g), pool.rows("v", table[b], n, g)
            s = np.array([pool.vs[table[b][i // P], g, i % P] if there[i] else 0
                          for i in range(n)], np.float64)
            for h in range(g * H // G, (g + 1) * H // G):
                for t in range(c):
                    m = n - (c - 1 - t) if causal else n
                    seen = np.flatnonzero(there[:max(m, 0)])
                    if seen.size == 0:
                        continue
                    x = k[seen] @ q[b, h, t] * scale
                    with np.errstate(invalid="ignore"):
                        p = np.exp(x - np.max(x))
                        p /= p.sum()
                        out[b, h, t] = p @ v[seen]
                        mag = p @ np.abs(v[seen])
                        dots = (np.abs(k[seen]) @ np.abs(q[b, h, t])).max() * scale
                        top = np.repeat(np.abs(q[b, h, t]).reshape(-1, 32).max(1), 32)
                        miss = (np.abs(k[seen]) @ top).max() * scale * Q_FLOOR[kind]
                        logit = D * U * dots + miss + 4 * U * np.abs(x).max() * 1.45
                        err = 2 * (logit + 2.0 ** -22 + (n / 32 + 64) * U)
                        low = 0.0
                        for j in range(0, n, 128):
                            of = (seen >= j) & (seen < j + 128)
                            if of.any():
                                low += (p[of] * s[seen[of]]).max() * 6 * of.sum()
                    tol[b, h, t] = (half * np.maximum(np.abs(out[b, h, t]), R.TINY[DTYPES[kind]]) +
                                    mag * (P_STEP[kind] + err) + P_FLOOR[kind] * low)
    return out, tol


def filled(rng, B, G, P, D, lengths, spare=2, bad=None, spread=2.0):
    """A pool whose sequences hold normal rows of several sizes, and their page table."""
    table, pages = R.tables(rng, [max(n, 0) for n in lengths], P, spare, bad)
    pool = Pool4(pages, G, P, D)
    for b in range(B):
        n = max(lengths[b], 0)
        k, v = (rng.standard_normal((G, n, D)) * 2.0 ** rng.uniform(-spread, spread, (G, n, 1))
                for _ in range(2))
        pool.append(list(table[b]), 0, k, v)
    return pool, table


def held_rows(tables, row_of_pages, n):
    """The first n cached tokens of a sequence by (k, k_scale, v, v_scale) and its row of the
    page table, all on one device: keys and values [Hkv, n, d] and the values' scales [Hkv, n] in
    float64, and which tokens have a page [n] (what the others hold is zeros)."""
    k, ks, v, vs = tables
    P, D = k.shape[2], 2 * k.shape[3]
    i = torch.arange(n, device=k.device)
    page, row = row_of_pages.to(k.device).long()[i // P], i % P
    there = (page >= 0) & (page < k.shape[0])
    page = torch.where(there, page, 0)
    grid = torch.from_numpy(np.concatenate([GRID, -GRID])).to(k.device)
    byte = k[page, :, row]                                             # [n, Hkv, d / 2]
    codes = torch.stack([byte & 15, byte >> 4], -1).flatten(-2)
    e = ks[page, :, row // 16, row % 4, :, row % 16 // 4].double()     # [n, Hkv, d / 32]
    scale = torch.where(e == 255, math.nan, torch.exp2(e - 127)).repeat_interleave(32, -1)
    keys = grid[codes.long()] * scale
    byte = v[page, :, row // 32, :, row % 32 // 2]                     # [n, Hkv, d]
    codes = torch.where((row % 2 == 1)[:, None, None], byte >> 4, byte & 15)
    s = vs[page, :, row].double()                                      # [n, Hkv]
    values = grid[codes.long()] * s[..., None]
    none = ~there
    keys[none], values[none], s[none] = 0.0, 0.0, 0.0
    return keys.transpose(0, 1), values.transpose(0, 1), s.t(), there


def attend_rows(held, q, count, kind, causal=True, scale=None):
    """attend() of one sequence, from held_rows() and its queries q [H, T, d] in float64 on the
    same device: outputs [H, T, d] (queries behind the count: zeros) and their tolerances."""
    k, v, s, there = held
    G, n, D = k.shape
    H, T = q.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    half = R.HALF_STEP[DTYPES[kind]]
    if n == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    x = q.reshape(G, H // G * T, D)
    t = torch.arange(T, device=q.device).repeat(H // G)
    limit = n - (count - 1 - t) if causal else torch.full_like(t, n)
    limit = torch.where(t < count, limit, 0)
    seen = there & (torch.arange(n, device=q.device) < limit[:, None])         # [rows, n]
    some = seen.any(-1)[:, None]

    def times(a, b):                                     # [G, rows, d] by [G, n, d]
        return torch.matmul(a, b.transpose(1, 2).contiguous())

    def most(a):                                         # of what is seen, zeros of nothing
        return torch.where(seen, a, 0.0).amax(-1, keepdim=True)
    logit = torch.where(seen, times(x, k) * scale, -math.inf)
    p = torch.exp(logit - torch.where(some, logit.amax(-1, keepdim=True), 0.0))
    p = p / torch.where(some, p.sum(-1, keepdim=True), 1.0)
    out, mag = torch.matmul(p, v), torch.matmul(p, v.abs())
    top = x.abs().reshape(G, -1, D // 32, 32).amax(-1).repeat_interleave(32, -1)
    dots = most(times(x.abs(), k.abs())) * scale
    miss = most(times(top, k.abs())) * scale * Q_FLOOR[kind]
    err = 2 * (D * U * dots + miss + 4 * U * most(logit.abs()) * 1.45 + 2.0 ** -22 +
               (n / 32 + 64) * U)
    blocks = -(-n // 128)
    pad = blocks * 128 - n
    weight = torch.nn.functional.pad(p * s[:, None], (0, pad)).unflatten(-1, (blocks, 128))
    number = torch.nn.functional.pad(seen.double(), (0, pad)).unflatten(-1, (blocks, 128)).sum(-1)
    low = (weight.amax(-1) * 6 * number).sum(-1, keepdim=True)
    tol = (half * torch.clamp(out.abs(), min=R.TINY[DTYPES[kind]]) + mag * (P_STEP[kind] + err) +
           P_FLOOR[kind] * low)
    tol = torch.where(some, tol, 0.0)
    return out.reshape(H, T, D), tol.reshape(H, T, D)
