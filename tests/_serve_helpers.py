"""Plain implementations, in float64 on the CPU, of the operators of e2s_serve.h, and
the tolerances that their arithmetic gives."""
import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn
LOWEST = -100
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# smallest normal numbers: below them a rounding is off by an absolute half step
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -14, torch.float32: 2.0 ** -126}


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

def frequencies(R, base, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    if scaling == "base" and R > 2:
        base = base * factor ** (R / (R - 2))
    f = np.array([base ** (-2.0 * j / R) for j in range(R // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        g = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = (1 - g) * f / factor + g * f
    return f


def rotate(x, positions, f, axis=None, layout="half", amplitude=1.0, inverse=False):
    """x [B, H, T, d] float64, positions [B, T] or [3, B, T]; angles in float64."""
    R = 2 * len(f)
    y = x.clone()
    for j in range(R // 2):
        p = positions[axis[j]] if axis is not None else positions
        a = p.double() * f[j] * (-1 if inverse else 1)
        c, s = amplitude * torch.cos(a)[:, None], amplitude * torch.sin(a)[:, None]
        i0, i1 = (j, j + R // 2) if layout == "half" else (2 * j, 2 * j + 1)
        y[..., i0] = x[..., i0] * c - x[..., i1] * s
        y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


def rotate_tolerance(x, ref, R, layout, dtype, amplitude=1.0):
    """One rounding of the result, and float32's of the angle within a turn (pi * 2^-25), of
    sine and cosine (2 steps of 2^-24), of the amplitude (2) and of the product's three
    operations: under 8 * 2^-24 of |x0| + |x1|."""
    pair = torch.zeros_like(ref)
    half = R // 2
    a = x[..., :R].abs()
    if layout == "half":
        both = a[..., :half] + a[..., half:]
        pair[..., :half], pair[..., half:R] = both, both
    else:
        both = a[..., 0::2] + a[..., 1::2]
        pair[..., 0:R:2], pair[..., 1:R:2] = both, both
    step = HALF_STEP[dtype]
    return step * torch.clamp(ref.abs(), min=TINY[dtype]) + 8 * 2.0 ** -24 * amplitude * pair


# ---------------------------------------------------------------------------
# the 8-bit cache
# ---------------------------------------------------------------------------

def e4m3_values():
    return torch.arange(256, dtype=torch.uint8).view(F8).double().numpy()


_VALUES = e4m3_values()
_GRID = np.array(sorted(v for v in _VALUES[:128] if not math.isnan(v)))   # 0 .. 448


def to_e4m3(x):
    """float64 array, |x| <= 448 or NaN, to bytes: nearest, ties to the even mantissa."""
    x = np.asarray(x, dtype=np.float64)
    m = np.abs(np.where(np.isnan(x), 0.0, x))
    hi = np.clip(np.searchsorted(_GRID, m), 1, len(_GRID) - 1)
    lo = hi - 1
    down = m - _GRID[lo]
    up = _GRID[hi] - m
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isnan(x), 0x7F, code).astype(np.uint8)
    return code | (np.signbit(x) & ~np.isnan(x)).astype(np.uint8) << 7


def block_scale(amax):
    if amax == 0:
        return 2.0 ** LOWEST
    e = math.frexp(amax)[1] - 10
    while 448.0 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** max(e, LOWEST)


class Pool:
    """A cache as numpy bytes and scales; every byte that nothing wrote is a NaN."""

    def __init__(self, pages, G, P, D):
        self.k, self.v = (np.full((pages, G, P, D), 0x7F, np.uint8) for _ in range(2))
        self.ks, self.vs = (np.full((pages, G), np.nan, np.float32) for _ in range(2))
        self.P = P

    def tensors(self, device="cuda"):
        k, v = (torch.from_numpy(x.copy()).to(device).view(F8) for x in (self.k, self.v))
        return k, v, *(torch.from_numpy(x.copy()).to(device) for x in (self.ks, self.vs))

    def rows(self, which, table, n, g):
        """The first n cached rows of a sequence and head, float64 [n, D]; NaN where the
        page does not exist."""
        x, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        out = np.full((n, x.shape[3]), np.nan)
        for i in range(n):
            p = table[i // self.P]
            if 0 <= p < x.shape[0]:
                out[i] = _VALUES[x[p, g, i % self.P]] * float(s[p, g])
        return out

    def append(self, which, table, start, rows):
        """rows [G, n, D] float64 as tokens start ..; token by block, as documented."""
        x, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        P, n = self.P, rows.shape[1]
        end = min(start + n, len(table) * P)
        if start < 0:
            return
        for blk in range(start // P, -(-end // P) if end > start else 0):
            p = table[blk]
            if not 0 <= p < x.shape[0]:
                continue
            r0, r1 = max(start - blk * P, 0), min(end - blk * P, P)
            new = rows[:, blk * P + r0 - start:blk * P + r1 - start]
            for g in range(rows.shape[0]):
                fin = np.abs(new[g][np.isfinite(new[g])])
                want = block_scale(fin.max() if fin.size else 0.0)
                if r0 > 0:
                    want = max(want, float(s[p, g]))
                    if want > s[p, g]:
                        x[p, g, :r0] = to_e4m3(_VALUES[x[p, g, :r0]] * float(s[p, g]) / want)
                y = np.where(np.isinf(new[g]), np.nan, new[g])
                x[p, g, r0:r1] = to_e4m3(y / want)
                s[p, g] = want


def same_bytes(got, ref):
    """Equal, or both NaN."""
    got, ref = np.asarray(got), np.asarray(ref)
    return bool(np.all((got == ref) | (((got & 0x7F) == 0x7F) & ((ref & 0x7F) == 0x7F))))


def attend(pool, table, lengths, q, counts=None, causal=True, scale=None):
    """q [B, H, T, d] float64: outputs, per-token weights, and per (b, h, t) what the
    tolerances need: sum p|v| per dimension, the largest sum |q k| scale, the largest
    |logit|."""
    B, H, T, D = q.shape
    G = pool.k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    N = max(max(lengths), 1)
    out = np.zeros(q.shape)
    mag, dots, big = np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape[:3])
    w = np.zeros((B, G, N))
    q = q.numpy()
    for b in range(B):
        n = max(0, min(lengths[b], len(table[b]) * pool.P))
        c = T if counts is None else counts[b]
        there = np.array([0 <= table[b][i // pool.P] < pool.k.shape[0] for i in range(n)], bool)
        for g in range(G):
            k, v = pool.rows("k", table[b], n, g), pool.rows("v", table[b], n, g)
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
                    mag[b, h, t] = p @ np.abs(v[seen])
                    dots[b, h, t] = (np.abs(k[seen]) @ np.abs(q[b, h, t])).max() * scale
                    big[b, h, t] = np.abs(x).max()
                    w[b, g, seen] += p
    return out, w, mag, dots, big


P_STEP = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -16, torch.float32: 2.0 ** -24}


def weight_error(D, N, dots, big):
    """Relative error of a softmax weight: the logit's (D float32 additions over sum |q k|,
    and 4 roundings of its size: the scale, its product, log2(e), the distance to the
    maximum), the hardware exponential's 2^-22, the sum's over N tokens (32 at a time, then
    64 more), twice over for numerator and denominator."""
    logit = (D * 2.0 ** -24) * dots + 4 * 2.0 ** -24 * big * 1.45
    return 2 * (logit + 2.0 ** -22 + (N / 32 + 64) * 2.0 ** -24)


def attend_tolerance(dtype, D, N, ref, mag, dots, big):
    err = weight_error(D, N, dots, big)[..., None]
    return HALF_STEP[dtype] * np.maximum(np.abs(ref), TINY[dtype]) + mag * (P_STEP[dtype] + err)


def evict(weights, n, K, sinks, recent):
    """Kept indices of one head, ascending."""
    if n <= K:
        return list(range(n))
    ends = [i for i in range(n) if i < sinks or i >= n - recent]
    mid = [i for i in range(sinks, n - recent)]
    mid.sort(key=lambda i: (math.isnan(weights[i]),
                            -weights[i] if not math.isnan(weights[i]) else 0.0, i))
    return sorted(ends + mid[:K - len(ends)])


def tables(rng, counts, P, spare=0, bad=None):
    """Disjoint pages in random order for sequences of `counts` tokens; (table, pages).
    Entries beyond a sequence's pages are `bad`."""
    need = [-(-n // P) for n in counts]
    total = max(sum(need) + spare, 1)
    perm = rng.permutation(total)
    width = max(max(need), 1)
    t = np.full((len(counts), width), -1 if bad is None else bad, np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n]
        at += n
    return t, total
