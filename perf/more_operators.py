"""Performance cases of the operators that a layer's step takes beside those of
perf/operators.py: the norms of every head's queries and keys with the rotation of their
positions, forward and back, and a key/value cache held in 4 bits, filled, read and
attended to.

A case is a dict of plain values.  `entry` names the public call:

  norm    norm_rotate on the queries and keys of a call; with `train`, the backward pass
          as well, to the gradients of q, k and both weights
  append  cache4_append: new tokens (all, or the kept ones of a source) into their pages,
          and cache4_read, which gives the values that they are held as
  attend  a Cache4Attention kept by the program: queries against the cached tokens

`order` is how the model holds its rows: "head" [B, H, T, d], "token" [B, T, H, d].
`weight` is the type of the norms' weights: the rows' own, "f32", or "none".  Lengths,
counts and start positions are drawn from `sizes_seed`, tensors from the seed of prepare().

The 4-bit cache holds elements of one sign, two exponent and one mantissa bit (0, 1/2, 1,
3/2, 2, 3, 4, 6).  Keys have a power-of-two scale for every 32 elements of a row, a byte of
its exponent + 127; values have a bfloat16 scale for a row.  Tables, for pages of P tokens:
  k        [pages, Hkv, P, d / 2]: elements 2 i, 2 i + 1 in the low and high half of byte i
  k_scale  [pages, Hkv, P / 16, 4, d / 32, 4]: [.., n, r, c, u] is block c of token 16 n +
           4 u + r
  v        [pages, Hkv, P / 32, d, 16]: byte i of [.., n, j] is element j of tokens
           32 n + 2 i (low half) and 32 n + 2 i + 1
  v_scale  [pages, Hkv, P]
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
LOWEST = -100          # exponent of the smallest scale


def _case(name, entry, **kw):
    c = dict(name=name, entry=entry, batch=1, heads=32, kv_heads=32, head_dim=128, dtype="bf16",
             sizes_seed=1, order="token")
    c.update({"norm": dict(tokens=1, rot_dim=128, layout="half", axes=1, far=0, weight="own",
                           train=False),
              "append": dict(tokens=1, source=0, page=64, start_max=0, ragged=False),
              "attend": dict(queries=1, len_min=1, len_max=1, page=64, ragged=False)}[entry])
    c.update(kw)
    return c


def listed():
    qwen = dict(heads=28, kv_heads=4)
    return [
        # one decoding step of one sequence: grid positions on three axes, latency only
        _case("norm_decode", "norm", axes=3, far=40000, **qwen),
        # a prefill batch of the LLaVA-1.5-7B shape (image and text tokens)
        _case("norm_prefill", "norm", batch=32, tokens=1024),
        # a training step of grouped heads, the largest
        _case("norm_train", "norm", batch=8, tokens=2048, kv_heads=8, train=True, weight="f32"),
        # gradients in full precision: interleaved and partly turned rows, odd length
        _case("norm_train_f32", "norm", batch=3, heads=12, kv_heads=2, dtype="f32", tokens=1777,
              rot_dim=64, layout="interleaved", order="head", far=100000, train=True),
        # a serving batch appends one token per sequence
        _case("append_decode", "append", batch=64, start_max=2000, **qwen),
        # the 128 kept tokens of 64 LLaVA images, out of 576, into the cache of a layer
        _case("append_kept", "append", batch=64, tokens=128, source=576, start_max=60,
              order="head"),
        # one interactive sequence, where latency counts
        _case("attend_single", "attend", len_min=700, len_max=1100, **qwen),
        # a few long documents: one query against up to 131072 tokens
        _case("attend_long", "attend", batch=4, len_min=60000, len_max=131072, **qwen),
        # the LLaVA serving batch
        _case("attend_batch", "attend", batch=64, dtype="f16", len_min=130, len_max=1200),
        # text queries after an image, in one causal call of ragged counts
        _case("attend_chunk", "attend", batch=16, queries=48, len_min=300, len_max=4200,
              ragged=True, **qwen),
        # full-precision queries, small heads and pages, sequences that may be empty
        _case("attend_f32", "attend", batch=9, heads=16, kv_heads=2, head_dim=64, dtype="f32",
              len_min=0, len_max=3001, page=32, order="head"),
        # long prompts: many queries at once
        _case("attend_prompt", "attend", batch=2, queries=1024, len_min=2048, len_max=2048, **qwen),
    ]


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _sizes(c):
    """The per-sequence numbers of a case, as lists."""
    rng = random.Random(c["sizes_seed"])
    B = c["batch"]
    if c["entry"] == "append":
        start = [rng.randint(0, c["start_max"]) for _ in range(B)]
        count = [rng.randint(0, c["tokens"]) if c["ragged"] else c["tokens"] for _ in range(B)]
        return {"start": start, "count": count, "end": [s + n for s, n in zip(start, count)]}
    if c["entry"] == "attend":
        length = [rng.randint(c["len_min"], c["len_max"]) for _ in range(B)]
        return {"length": length,
                "count": [rng.randint(1, c["queries"]) if c["ragged"] else c["queries"]
                          for _ in range(B)]}
    return {}


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    H, G, D, B = c["heads"], c["kv_heads"], c["head_dim"], c["batch"]
    held = D + D / 32 + 2                      # bytes of a token's key and value of one head
    z = _sizes(c)
    if c["entry"] == "norm":
        n = float(B * c["tokens"] * (H + G)) * D
        return {"bytes": (5 if c["train"] else 2) * n * es + 4.0 * c["axes"] * B * c["tokens"],
                "flops": (24 if c["train"] else 7) * n}
    if c["entry"] == "append":
        n = float(sum(z["count"])) * G
        return {"bytes": 2 * n * (2 * D * es + held) + 1.0, "flops": 12 * n * D}
    n, q = float(sum(z["length"])), float(sum(z["count"]))
    pairs = float(sum(max(0, a - (b - 1) / 2) * b for a, b in zip(z["length"], z["count"])))
    return {"bytes": n * G * held + 2 * q * H * D * es, "flops": 4 * pairs * H * D + 1.0}


# ---------------------------------------------------------------------------
# further cases of the same ranges
# ---------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """A case whose cost stays within the largest listed one of its entry."""
    entry = rng.choice(["norm", "norm", "append", "attend", "attend", "attend"])
    most = max(_cost(c) for c in listed() if c["entry"] == entry)
    while True:
        heads, kv = rng.choice([(28, 4), (16, 2), (32, 8), (12, 2), (32, 32), (16, 16), (4, 4)])
        c = dict(entry=entry, batch=_log_int(rng, 1, 64), heads=heads, kv_heads=kv,
                 head_dim=rng.choice([64, 128, 128]),
                 dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                 sizes_seed=rng.randrange(1 << 20), order=rng.choice(["token", "head"]))
        page = rng.choice([32, 64, 128])
        if entry == "norm":
            d = rng.choice([64, 128, 128, 128, 80, 96, 256])
            c.update(head_dim=d, tokens=_log_int(rng, 1, 4096),
                     rot_dim=rng.choice([d, d, d // 2, d // 4]),
                     layout=rng.choice(["half", "interleaved"]), axes=rng.choice([1, 1, 3]),
                     far=rng.choice([0, 1000, 500000]), weight=rng.choice(["own", "f32", "none"]),
                     train=rng.random() < 0.5)
        elif entry == "append":
            t = _log_int(rng, 1, 2000)
            c.update(tokens=t, source=rng.choice([0, t + _log_int(rng, 1, 2000)]), page=page,
                     start_max=_log_int(rng, 1, 2000), ragged=rng.random() < 0.5)
        else:
            most_len = _log_int(rng, 1, 60000)
            t = rng.choice([1, 1, 1, _log_int(rng, 2, 512)])
            c.update(queries=t, len_max=most_len, len_min=rng.choice([0, most_len // 2, most_len]),
                     page=page, ragged=t > 1 and rng.random() < 0.5)
        scores = c["batch"] * heads * c.get("queries", 0) * c.get("len_max", 0)
        if _cost(c) <= most and scores <= 1 << 28:
            return c


# ---------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------

def _rows(c, g, heads, tokens):
    """[B, heads, tokens, d] as the model holds it."""
    B, D = c["batch"], c["head_dim"]
    shape = (B, heads, tokens, D) if c["order"] == "head" else (B, tokens, heads, D)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(DTYPES[c["dtype"]])
    return x if c["order"] == "head" else x.transpose(1, 2)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(g, page, tokens):
    """A page table of pages in no order for sequences of so many tokens; the number of pages."""
    need = [-(-n // page) for n in tokens]
    total = sum(need) + 1
    perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    t = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n]
        at += n
    return t, total


def _pool(c, g, pages):
    """The tables of a cache whose pages are all filled."""
    P, G, D = c["page"], c["kv_heads"], c["head_dim"]
    s = dict(k=torch.empty((pages, G, P, D // 2), dtype=torch.uint8, device="cuda"),
             k_scale=torch.empty((pages, G, P // 16, 4, D // 32, 4), dtype=torch.uint8,
                                 device="cuda"),
             v=torch.empty((pages, G, P // 32, D, 16), dtype=torch.uint8, device="cuda"),
             v_scale=torch.empty((pages, G, P), dtype=torch.bfloat16, device="cuda"))
    step = max(1, (1 << 25) // (G * P * D))
    for a in range(0, pages, step):
        n = min(step, pages - a)
        for name in ("k", "v"):
            x = torch.randn((n, G, P, D), generator=g, device="cuda")
            x = x * torch.exp2(torch.rand((n, G, P, 1), generator=g, device="cuda"))
            _put(s, name, slice(a, a + n), x)
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, G, H, D = c["batch"], c["kv_heads"], c["heads"], c["head_dim"]
    z = _sizes(c)
    s = dict(case=c)
    if c["entry"] == "norm":
        T = c["tokens"]
        s["q"], s["k"] = _rows(c, g, H, T), _rows(c, g, G, T)
        lead = (3, B) if c["axes"] == 3 else (B,)
        first = torch.randint(0, c["far"] + 1, lead + (1,), generator=g, device="cuda")
        step = torch.randint(0, 2, lead + (T,), generator=g, device="cuda")
        s["positions"] = (first + torch.cumsum(step, -1)).to(torch.int32)
        half = c["rot_dim"] // 2
        third = 3 * half // 8
        s["rotary"] = dict(rot_dim=c["rot_dim"], base=1e6, layout=c["layout"],
                           sections=(half - 2 * third, third, third) if c["axes"] == 3 else None)
        s["q_weight"] = s["k_weight"] = None
        if c["weight"] != "none":
            kind = torch.float32 if c["weight"] == "f32" else DTYPES[c["dtype"]]
            for n in ("q_weight", "k_weight"):
                w = 1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")
                s[n] = w.to(kind)
        if c["train"]:
            s["q_grad"], s["k_grad"] = _rows(c, g, H, T), _rows(c, g, G, T)
        if own:
            import paper_2608_23253_amd as E
            s["plan"] = E.rotary_plan(D, **s["rotary"])
            if c["train"]:
                for n in ("q", "k", "q_weight", "k_weight"):
                    if s[n] is not None:
                        s[n].requires_grad_(True)
        return s
    if c["entry"] == "append":
        s["pages"], n = _table(g, c["page"], z["end"])
        s.update(_pool(c, g, n))
        s["start"], s["count"] = _ints(z["start"]), _ints(z["count"]) if c["ragged"] else None
        src = c["source"] or c["tokens"]
        s["new_k"], s["new_v"] = _rows(c, g, G, src), _rows(c, g, G, src)
        s["index"] = None
        if c["source"]:
            order = torch.rand((B, src), generator=g, device="cuda").argsort(1)[:, :c["tokens"]]
            s["index"] = order.sort(1).values.to(torch.int32)
    else:
        s["pages"], n = _table(g, c["page"], z["length"])
        s.update(_pool(c, g, n))
        s["lengths"], s["count"] = _ints(z["length"]), _ints(z["count"]) if c["ragged"] else None
        s["q"] = _rows(c, g, H, c["queries"])
        s["out"] = torch.zeros(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    if own:
        import paper_2608_23253_amd as E
        s["cache"] = E.PagedCache4.of(s["k"], s["k_scale"], s["v"], s["v_scale"])
        if c["entry"] == "attend":
            s["attention"] = E.Cache4Attention(s["cache"], B, H, c["queries"],
                                               max(c["len_max"], 1), DTYPES[c["dtype"]])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2608_23253_amd as E
        if c["entry"] == "norm":
            y = E.norm_rotate(s["q"], s["k"], s["positions"], s["plan"], s["q_weight"],
                              s["k_weight"], eps=EPS)
            if not c["train"]:
                return list(y)
            at = [s[n] for n in ("q", "k", "q_weight", "k_weight") if s[n] is not None]
            return [*y, *torch.autograd.grad(y, at, [s["q_grad"], s["k_grad"]])]
        if c["entry"] == "append":
            E.cache4_append(s["cache"], s["pages"], s["start"], s["new_k"], s["new_v"],
                            count=s["count"], src_idx=s["index"])
            return list(E.cache4_read(s["cache"], s["pages"], s["start"], c["tokens"],
                                      count=s["count"], dtype=DTYPES[c["dtype"]]))
        return s["attention"](s["q"], s["pages"], s["lengths"], out=s["out"], q_count=s["count"])
    return {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend}[c["entry"]](s, c)


# ---- norms and positions ----

def _turn(y, r, axes, positions, back=False):
    """Rows [B, H, T, d] in float32, turned."""
    R = r["rot_dim"]
    j = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    w = r["base"] ** (-2 * j / R)
    pos = positions.double()
    if axes == 3:
        axis = torch.repeat_interleave(torch.arange(3, device="cuda"),
                                       torch.tensor(r["sections"], device="cuda"))
        angle = (pos[axis] * w[:, None, None]).permute(1, 2, 0)
    else:
        angle = pos[..., None] * w
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if back:
        sin = -sin
    if r["layout"] == "half":
        a, b = y[..., :R // 2], y[..., R // 2:R]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., R:]], -1)
    a, b = y[..., 0:R:2], y[..., 1:R:2]
    z = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([z, y[..., R:]], -1)


def _plain_norm(s, c):
    outs, grads, of_weights = [], [], []
    for n in ("q", "k"):
        x, w = s[n].float(), s[n + "_weight"]
        f = 1.0 if w is None else w.float()
        inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        unit = x * inv
        outs.append(_turn(unit * f, s["rotary"], c["axes"], s["positions"]).to(s[n].dtype))
        if c["train"]:
            g = _turn(s[n + "_grad"].float(), s["rotary"], c["axes"], s["positions"], back=True)
            of_unit = g * f
            dx = inv * (of_unit - unit * (of_unit * unit).mean(-1, keepdim=True))
            grads.append(dx.to(s[n].dtype))
            if w is not None:
                of_weights.append((g * unit).sum((0, 1, 2)).to(w.dtype))
    return outs + grads + of_weights


# ---- the 4-bit cache ----

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _codes(x, scale):
    """Elements as codes 0 .. 15 at a scale: to nearest, ties to the even code.  The borders
    times the scale are exact in float32."""
    a = x.abs()
    n = ((a > 0.25 * scale).to(torch.uint8) + (a >= 0.75 * scale) + (a > 1.25 * scale)
         + (a >= 1.75 * scale) + (a > 2.5 * scale) + (a >= 3.5 * scale) + (a > 5.0 * scale))
    return n + (torch.signbit(x).to(torch.uint8) << 3)


def _key_scale(amax):
    """The smallest power of two s >= 2^LOWEST with amax <= 6 s."""
    f, x = torch.frexp(amax)
    e = torch.where(f <= 0.75, x - 3, x - 2)
    e = torch.where(amax == 0, torch.full_like(e, LOWEST), e).clamp(min=LOWEST)
    return torch.ldexp(torch.ones_like(amax), e)


def _value_scale(amax):
    """The smallest bfloat16 s >= 2^LOWEST with amax <= 6 s, in float32."""
    low = ((amax / 6.0).view(torch.int32) & -65536)
    s = low.view(torch.float32)
    s = torch.where(6.0 * s < amax, (low + 65536).view(torch.float32), s)
    return s.clamp(min=2.0 ** LOWEST)


def _put(s, name, at, x):
    """Whole pages x [n, Hkv, P, d] float32 into pages `at` of a table."""
    n, G, P, D = x.shape
    if name == "k":
        blocks = x.reshape(n, G, P, D // 32, 32)
        sc = _key_scale(blocks.abs().amax(-1, keepdim=True))
        q = _codes(blocks, sc).reshape(n, G, P, D // 2, 2)
        s["k"][at] = q[..., 0] | (q[..., 1] << 4)
        e = torch.frexp(sc[..., 0]).exponent + 126
        e = e.to(torch.uint8).reshape(n, G, P // 16, 4, 4, D // 32)          # n, u, r, c
        s["k_scale"][at] = e.permute(0, 1, 2, 4, 5, 3)
    else:
        sc = _value_scale(x.abs().amax(-1, keepdim=True))
        q = _codes(x, sc).reshape(n, G, P // 32, 16, 2, D).permute(0, 1, 2, 5, 3, 4)
        s["v"][at] = q[..., 0] | (q[..., 1] << 4)
        s["v_scale"][at] = sc[..., 0].to(torch.bfloat16)


def _get(s, name, at):
    """Pages `at` of a table: the codes [.., Hkv, P, d] and their scales, broadcast alike."""
    q = s[name][at]
    both = torch.stack([q & 15, q >> 4], -1)
    if name == "k":
        codes = both.flatten(-2)
        e = s["k_scale"][at].to(torch.int32) - 127
        e = e.movedim(-1, -3).flatten(-4, -2)                               # [.., P, d / 32]
        sc = torch.ldexp(torch.ones((), device="cuda"), e).repeat_interleave(32, -1)
    else:
        codes = both.flatten(-2).transpose(-1, -2).flatten(-3, -2)
        sc = s["v_scale"][at].float()[..., None]
    return codes, sc


def _values(codes, scale):
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device="cuda")
    return grid[codes.long()] * scale


def _plain_append(s, c):
    P, B, T, G, D = c["page"], c["batch"], c["tokens"], c["kv_heads"], c["head_dim"]
    start = s["start"].long()
    count = s["count"].long() if s["count"] is not None else torch.full_like(start, T)
    end = start + count
    blocks = (T + P - 2) // P + 1
    blk = (start // P)[:, None] + torch.arange(blocks, device="cuda")            # [B, blocks]
    tok = blk[:, :, None] * P + torch.arange(P, device="cuda")                   # [B, blocks, P]
    touched = (blk * P < end[:, None]) & (count > 0)[:, None]
    page = s["pages"].long()[torch.arange(B, device="cuda")[:, None],
                             blk.clamp(max=s["pages"].shape[1] - 1)]
    is_new = (tok >= start[:, None, None]) & (tok < end[:, None, None])
    src = (tok - start[:, None, None]).clamp(0, T - 1)
    if s["index"] is not None:
        src = s["index"].long()[torch.arange(B, device="cuda")[:, None, None], src]
    b, i = touched.nonzero(as_tuple=True)
    page, is_new, src = page[b, i], is_new[b, i][:, None, :, None], src[b, i]
    for name, new in (("k", s["new_k"]), ("v", s["new_v"])):
        fresh = new.permute(0, 2, 1, 3)[b[:, None], src].permute(0, 2, 1, 3).float()
        tables = {n: t[page] for n, t in s.items() if n in (name, name + "_scale")}
        _put(tables, name, slice(None), fresh)                     # every row of the pages anew
        if name == "k":
            old_k, old_s = s["k"][page], s["k_scale"][page]
            s["k"][page] = torch.where(is_new, tables["k"], old_k)
            keep = is_new.reshape(-1, 1, P // 16, 4, 4, 1).permute(0, 1, 2, 4, 5, 3)
            s["k_scale"][page] = torch.where(keep, tables["k_scale"], old_s)
        else:
            old_v, old_s = s["v"][page], s["v_scale"][page]
            half = is_new.reshape(-1, 1, P // 32, 1, 16, 2).to(torch.uint8)
            mask = half[..., 0] * 15 + half[..., 1] * 240
            s["v"][page] = (tables["v"] & mask) | (old_v & ~mask)
            s["v_scale"][page] = torch.where(is_new[..., 0], tables["v_scale"], old_s)
    # the new tokens, read back
    t = torch.arange(T, device="cuda")
    at = start[:, None] + t                                                      # [B, T]
    live = t < count[:, None]
    row_page = s["pages"].long()[torch.arange(B, device="cuda")[:, None],
                                 (at // P).clamp(max=s["pages"].shape[1] - 1)].clamp(min=0)
    out = []
    flat = torch.where(live, row_page, torch.zeros_like(row_page))
    used, where = torch.unique(flat, return_inverse=True)
    for name in ("k", "v"):
        x = _values(*_get(s, name, used))                                        # [., G, P, D]
        rows = x.transpose(1, 2)[where, at % P].transpose(1, 2)                  # [B, G, T, D]
        rows = torch.where(live[:, None, :, None], rows, torch.zeros_like(rows))
        out.append(rows.to(DTYPES[c["dtype"]]))
    return out


def _gathered(s, name, N):
    """[B, Hkv, N, d] of the cached tokens in float32 (rows behind a sequence: zeros)."""
    x = _values(*_get(s, name, s["pages"].long().clamp(min=0)))              # [B, n, G, P, D]
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :N]
    return torch.where((torch.arange(x.shape[2], device="cuda")
                        < s["lengths"][:, None])[:, None, :, None], x, torch.zeros_like(x))


def _plain_attend(s, c):
    B, H, G, T, D = c["batch"], c["heads"], c["kv_heads"], c["queries"], c["head_dim"]
    g = H // G
    k = _gathered(s, "k", max(c["len_max"], 1))
    N = k.shape[2]
    q = s["q"].float().reshape(B, G, g * T, D)
    logit = torch.matmul(q, k.transpose(2, 3).contiguous()) * (D ** -0.5)
    logit = logit.reshape(B, G, g, T, N)
    count = s["count"] if s["count"] is not None else torch.full_like(s["lengths"], T)
    t = torch.arange(T, device="cuda")
    limit = s["lengths"][:, None] - (count[:, None] - 1 - t)                      # [B, T]
    limit = torch.where(t < count[:, None], limit, torch.zeros_like(limit))
    seen = (torch.arange(N, device="cuda") < limit[:, :, None])[:, None, None]
    logit = torch.where(seen, logit, torch.full_like(logit, -math.inf))
    top = logit.amax(-1, keepdim=True)
    p = torch.exp(logit - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p.reshape(B, G, g * T, N), _gathered(s, "v", N)).reshape(B, H, T, D)
    valid = (t < count[:, None])[:, None, :, None]
    s["out"].copy_(torch.where(valid, o.to(s["out"].dtype), s["out"]))
    return s["out"]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["entry"] == "norm":
        return _exact_norm(s, c)
    if c["entry"] == "append":
        return _exact_append(s, c, _sizes(c))
    return _exact_attend(s, c, _sizes(c))


def _exact_norm(s, c):
    """The definition, a pair at a time as a product of complex numbers; gradients by
    torch's own differentiation of it."""
    r, R = s["rotary"], c["rot_dim"]
    leaves, outs, given = [], [], []
    with torch.enable_grad():
        weights = []
        for n in ("q", "k"):
            x = s[n].detach().double().requires_grad_(c["train"])
            w = s[n + "_weight"]
            w = None if w is None else w.detach().double().requires_grad_(c["train"])
            leaves.append(x)
            weights += [] if w is None else [w]
            y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
            y = y if w is None else y * w
            cols = list(y.unbind(-1))
            for j in range(R // 2):
                f = math.exp(-2.0 * j / R * math.log(r["base"]))
                pos = s["positions"]
                if c["axes"] == 3:
                    a0, a1 = r["sections"][0], r["sections"][0] + r["sections"][1]
                    pos = pos[(j >= a0) + (j >= a1)]
                a = (pos.double() * f)[:, None]
                i0, i1 = (j, j + R // 2) if r["layout"] == "half" else (2 * j, 2 * j + 1)
                z = torch.complex(y[..., i0], y[..., i1]) * torch.polar(torch.ones_like(a), a)
                cols[i0], cols[i1] = z.real, z.imag
            outs.append(torch.stack(cols, -1))
        if not c["train"]:
            return outs
        given = [s["q_grad"].double(), s["k_grad"].double()]
        grads = torch.autograd.grad(outs, leaves + weights, given)
    return [o.detach() for o in outs] + list(grads)


def _exact_codes(y):
    """Nearest of the 4-bit values, ties to the even code: multiples of a step that doubles
    from 2 on and from 4 on."""
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.round(y / step) * step


def _exact_append(s, c, z):
    B, T, D, G = c["batch"], c["tokens"], c["head_dim"], c["kv_heads"]
    out = [torch.zeros((B, G, T, D), dtype=torch.float64, device="cuda") for _ in range(2)]
    for b, n in enumerate(z["count"]):
        if n == 0:
            continue
        k, v = (x[b].double() if s["index"] is None else x[b][:, s["index"][b].long()].double()
                for x in (s["new_k"], s["new_v"]))
        k = k[:, :n].reshape(G, n, D // 32, 32)
        m = k.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(m > 0, m, torch.ones_like(m)) / 6.0))
        e = torch.where(6.0 * torch.exp2(e - 1) >= m, e - 1, e)
        e = torch.where(6.0 * torch.exp2(e) < m, e + 1, e)
        sc = torch.exp2(torch.where(m > 0, e, torch.full_like(e, LOWEST)).clamp(min=LOWEST))
        out[0][b, :, :n] = (_exact_codes(k / sc) * sc).reshape(G, n, D)
        v = v[:, :n]
        m = v.abs().amax(-1, keepdim=True)
        f, x = torch.frexp(m / 6.0)
        f, unit = torch.ceil(f * 256.0), torch.exp2(x.double() - 8)
        f = torch.where(6.0 * (f - 1) * unit >= m, f - 1, f)
        sc = (f * unit).clamp(min=2.0 ** LOWEST)
        out[1][b, :, :n] = _exact_codes(v / sc) * sc
    return out


def _exact_attend(s, c, z):
    D, G, P = c["head_dim"], c["kv_heads"], c["page"]
    g = c["heads"] // G
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device="cuda")
    for b, (n, count) in enumerate(zip(z["length"], z["count"])):
        if n == 0:
            continue
        i = torch.arange(n, device="cuda")
        page, row = s["pages"][b].long()[i // P], i % P
        d = torch.arange(D, device="cuda")
        for h in range(G):
            byte = s["k"][page, h, row][:, d // 2].long()
            e = s["k_scale"][page, h, row // 16, row % 4][i, :, row % 16 // 4][:, d // 32].double()
            k = grid[(byte >> (4 * (d % 2))) & 15] * torch.exp2(e - 127)
            byte = s["v"][page, h, row // 32, :, row % 32 // 2].long()
            v = grid[(byte >> (4 * (row % 2))[:, None]) & 15]
            v = v * s["v_scale"][page, h, row].double()[:, None]
            q = s["q"][b, h * g:(h + 1) * g, :count].double()
            a = torch.matmul(q, k.t().contiguous()) / math.sqrt(D)
            back = count - 1 - torch.arange(count, device="cuda")
            a = a.masked_fill((i[None] + back[:, None] >= n)[None], -math.inf)
            p = torch.nan_to_num(torch.softmax(a, -1), nan=0.0)
            out[b, h * g:(h + 1) * g, :count] = torch.matmul(p, v)
    return out
