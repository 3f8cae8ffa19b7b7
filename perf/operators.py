"""Measured cases of the paged cache: append with position rotation, DeQuant of pages, attention by page tables, and attention of
batches that share a prefix.

A case is a dict of plain values; ``prepare`` makes from it and a seed what a serving program holds before the call, ``run`` makes
one call.  With ``own`` false ``run`` computes the same from elementary torch operations (codes in 64 bits, the rest in 32).

Pages are tiles of 64 tokens: codes int8 [Hkv, pages, 2944], radii binary16 [Hkv, pages, 512], in the layout that the library
specifies at the top of csrc/pq_layout.h, restated at ``_key_strings`` and ``_value_strings`` below.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
PAGE = 64
CODE_DWORDS = 736  # 2944 bytes

#: Lloyd-Max centroids of the angle densities of levels 2, 3, 4 (level 1: sixteen equal cells)
CENTROIDS = {
    2: (0.3097561169824672, 0.6339802399913396, 0.9368160868035565, 1.2610402098124294),
    3: (0.4262496930707343, 0.6743849977574453, 0.8964113290374507, 1.1445466337241617),
    4: (0.5242140911034451, 0.7059094056614837, 0.8648869211334125, 1.0465822356914518),
}
#: share of the angles of levels 2, 3, 4 in the outer cells (each of two)
OUTER = {2: 0.2066, 3: 0.1835, 4: 0.1728}

_kept = {}


def _rotation():
    """The preconditioner S: the orthogonal factor of a fixed Gaussian matrix, 64 bits, host."""
    if "S" not in _kept:
        _kept["S"] = np.ascontiguousarray(np.linalg.qr(np.random.RandomState(2502).standard_normal((D, D)))[0])
    return _kept["S"]


def _context():
    """The framework's context for that S: a program makes one and keeps it."""
    if "ctx" not in _kept:
        from paper_2502_02617_amd import Context

        _kept["ctx"] = Context(S=_rotation())
    return _kept["ctx"]


# ---------------------------------------------------------------- cases


def listed():
    return [
        # a decode step's new tokens, one per sequence of a small batch: latency alone
        {"name": "append 16 x 1", "op": "append", "B": 16, "Hq": 32, "Hkv": 8, "lo": 100, "hi": 4000, "new_lo": 1, "new_hi": 1, "pad": 0,
         "dtype": "bf16", "rot": 128, "inter": False},
        # one chunk of a prompt, beginning inside a page
        {"name": "append 8191", "op": "append", "B": 1, "Hq": 32, "Hkv": 8, "lo": 4130, "hi": 4130, "new_lo": 8191, "new_hi": 8191, "pad": 1,
         "dtype": "bf16", "rot": 128, "inter": False},
        # prompts of many users in one call, fp32 activations, rotation of half the head in neighbouring pairs
        {"name": "append ragged fp32", "op": "append", "B": 48, "Hq": 14, "Hkv": 2, "lo": 1, "hi": 900, "new_lo": 1, "new_hi": 700, "pad": 5,
         "dtype": "fp32", "rot": 64, "inter": True},
        # a cached prompt back to bf16 for the dense attention of its next chunk
        {"name": "read 8000", "op": "read", "B": 1, "Hq": 32, "Hkv": 8, "lo": 8000, "hi": 8000, "dtype": "bf16"},
        # caches of several sequences to fp32 (moving them to another format)
        {"name": "read ragged fp32", "op": "read", "B": 24, "Hq": 8, "Hkv": 8, "lo": 20, "hi": 6000, "dtype": "fp32"},
        # one user, short context
        {"name": "attend 1 x 1000", "op": "attend", "B": 1, "Hq": 32, "Hkv": 8, "lo": 1000, "hi": 1000, "M": 1, "rot": 128, "inter": False},
        # the decode batch that the contiguous cache is benchmarked on
        {"name": "attend 16 x 32768", "op": "attend", "B": 16, "Hq": 32, "Hkv": 8, "lo": 32768, "hi": 32768, "M": 1, "rot": 128, "inter": False},
        # serving: many sequences of mixed lengths
        {"name": "attend ragged 64", "op": "attend", "B": 64, "Hq": 32, "Hkv": 8, "lo": 200, "hi": 8000, "M": 1, "rot": 128, "inter": False},
        # four draft tokens per sequence
        {"name": "attend drafts", "op": "attend", "B": 16, "Hq": 32, "Hkv": 8, "lo": 6000, "hi": 12700, "M": 4, "rot": 128, "inter": False},
        # a few users of one system prompt
        {"name": "prefix 4 x 1000", "op": "prefix", "B": 4, "Hq": 32, "Hkv": 8, "groups": 1, "plo": 1000, "phi": 1000, "lo": 1, "hi": 60, "M": 1,
         "rot": 128, "inter": False},
        # many users of one long document
        {"name": "prefix 64 x 16384", "op": "prefix", "B": 64, "Hq": 32, "Hkv": 8, "groups": 1, "plo": 16384, "phi": 16384, "lo": 64, "hi": 1000,
         "M": 1, "rot": 128, "inter": False},
        # several documents, two draft tokens, lengths that end inside pages
        {"name": "prefix 6 groups", "op": "prefix", "B": 50, "Hq": 28, "Hkv": 4, "groups": 6, "plo": 700, "phi": 9000, "lo": 1, "hi": 500, "M": 2,
         "rot": 64, "inter": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "attend", "attend", "prefix", "prefix"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 4, 7, 8])
    c = {"op": op, "Hq": Hkv * G, "Hkv": Hkv}
    rot = {"rot": rng.choice([128, 128, 64, 32]), "inter": rng.random() < 0.4}
    if op == "append":
        B = _log_int(rng, 1, 128)
        top = _log_int(rng, 1, max(1, 8192 // B))
        hi = _log_int(rng, 1, 4096)
        c.update(B=B, lo=rng.choice([1, max(1, hi // 2)]), hi=hi, new_lo=rng.choice([1, top]), new_hi=top, pad=rng.choice([0, 0, 7]),
                 dtype=rng.choice(["bf16", "bf16", "fp32"]), **rot)
    elif op == "read":
        B = _log_int(rng, 1, 32)
        top = _log_int(rng, 1, max(64, 32768 // B))
        c.update(B=B, lo=max(1, top // rng.choice([1, 4, 50])), hi=top, dtype=rng.choice(["bf16", "fp32"]))
    elif op == "attend":
        B = _log_int(rng, 1, 128)
        top = _log_int(rng, 1, 200_000 // B)
        c.update(B=B, lo=max(1, top // rng.choice([1, 3, 40])), hi=top, M=rng.choice([1, 1, 1, 2, max(1, 16 // G)]), **rot)
    else:
        B = _log_int(rng, 2, 96)
        top = _log_int(rng, 64, min(16384, 600_000 // B))
        c.update(B=B, groups=rng.randint(1, max(1, B // 4)), plo=max(1, top // rng.choice([1, 4])), phi=top, lo=1, hi=_log_int(rng, 1, 1000),
                 M=rng.choice([1, 1, 2]), **rot)
    return c


def _lengths(case, what, n, lo, hi):
    """n lengths between lo and hi, spread over their logarithm, the same for every seed of a case (the work is the case's)."""
    rng = random.Random("%s %d %d %d %d" % (what, case["B"], n, lo, hi))
    return [_log_int(rng, lo, hi) for _ in range(n)]


def _sizes(case):
    """Lengths of the case: tokens of each sequence in its own pages, new ones among them, prefix of each group."""
    B = case["B"]
    before = _lengths(case, "before", B, case["lo"], case["hi"])
    new = _lengths(case, "new", B, case["new_lo"], case["new_hi"]) if case["op"] == "append" else [0] * B
    own_len = [a + b for a, b in zip(before, new)]
    prefix = _lengths(case, "prefix", case["groups"], case["plo"], case["phi"]) if case["op"] == "prefix" else []
    return own_len, new, prefix


def _group_start(case):
    """First sequence of every group, and the end of the last: groups differ by one sequence at most."""
    return [(g * case["B"]) // case["groups"] for g in range(case["groups"] + 1)]


def work(case):
    own_len, new, prefix = _sizes(case)
    op, Hq, Hkv = case["op"], case["Hq"], case["Hkv"]
    size = 4 if case.get("dtype") == "fp32" else 2
    if op == "append":  # rows in, rotation table, packed vectors out, and their values back as bf16
        n = sum(new)
        return {"bytes": n * (2 * Hkv * (D * size + 62 + D * 2) + 4 * case["rot"]), "flops": n * 2 * Hkv * 4 * D * D}
    if op == "read":
        n = sum(own_len)
        return {"bytes": n * 2 * Hkv * (62 + D * size), "flops": n * 2 * Hkv * 2 * D * D}
    rows = case["B"] * case["M"] * Hq
    pairs = sum(own_len) * case["M"] * Hq
    if op == "prefix":
        start = _group_start(case)
        pairs += sum(p * (start[g + 1] - start[g]) * case["M"] * Hq for g, p in enumerate(prefix))
    cached = (sum(own_len) + sum(prefix)) * 2 * Hkv * 62
    return {"bytes": cached + rows * D * 4, "flops": pairs * 4 * D + rows * 4 * D * D}


# ---------------------------------------------------------------- inputs


def _join(fields, width, dwords):
    """Fields [..., n] of `width` bits one after another, as `dwords` dwords (int64 [..., dwords], below 2^32)."""
    out = torch.zeros(*fields.shape[:-1], dwords + 1, dtype=torch.int64, device=fields.device)
    for i in range(fields.shape[-1]):
        d, s = divmod(i * width, 32)
        f = fields[..., i]
        out[..., d] |= (f << s) & 0xFFFFFFFF
        out[..., d + 1] |= (f >> (32 - s)) & 0xFFFFFFFF
        if s + width > 64:
            out[..., d + 2] |= f >> (64 - s)
    return out[..., :dwords]


def _random_pages(gen, kind, Hkv, pages):
    """Codes and radii of `pages` pages as an encoded stream has them: level 1 uniform, levels 2 to 4 in the shares of their cells,
    radii of sixteen coordinates of about unit size, tokens of different sizes."""
    dev = gen.device
    shape = (Hkv, pages, PAGE, 8)

    def angle(level, *more):
        u = torch.rand(*shape, *more, device=dev, generator=gen)
        a = OUTER[level]
        return (u >= a).to(torch.int64) + (u >= 0.5) + (u >= 1 - a)

    c1 = torch.randint(0, 16, (*shape, 4, 2), device=dev, generator=gen)
    Q = c1[..., 0] | angle(2, 4) << 4 | c1[..., 1] << 6
    c3 = angle(3, 2)
    Bi = angle(4) << 4 | c3[..., 0] << 2 | c3[..., 1]
    del c1, c3
    token = torch.exp(0.2 * torch.randn(Hkv, pages, PAGE, 1, device=dev, generator=gen))
    R = ((4 + 0.7 * torch.randn(*shape, device=dev, generator=gen)).clamp_(min=0.3) * token).to(torch.float16)
    if kind == "key":
        block = Q[..., 0] | Q[..., 1] << 10 | Q[..., 2] << 20 | Q[..., 3] << 30 | Bi << 40
        w = _join(block, 46, 12)  # [Hkv, pages, 64, 12]
        last = w[..., 11].reshape(Hkv, pages, 32, 2)
        parts = [w[..., 0:4], w[..., 4:8], w[..., 8:11], last[..., 0] | last[..., 1] << 16]
        radii = R
    else:  # token 16 i + 4 g + e is slot 4 i + e of (g, block)
        def by_slot(x):
            x = x.reshape(Hkv, pages, 4, 4, 4, 8, -1)  # i, g, e, b
            return x.permute(0, 1, 3, 5, 6, 2, 4).reshape(Hkv, pages, 4, 8, x.shape[-1], 16)

        pair = torch.stack([Q[..., 0] | Q[..., 1] << 10, Q[..., 2] | Q[..., 3] << 10], -1)
        w = _join(by_slot(pair).reshape(Hkv, pages, PAGE, 16), 20, 10)
        vb = _join(by_slot(Bi[..., None]).reshape(Hkv, pages, 32, 16), 6, 3)
        parts = [w[..., 0:4], w[..., 4:8], w[..., 8:10], vb]
        radii = by_slot(R[..., None])
    t = torch.cat([p.reshape(Hkv, pages, -1) for p in parts], -1)
    t = torch.where(t >= 1 << 31, t - (1 << 32), t).to(torch.int32)
    return t.view(torch.uint8), radii.reshape(Hkv, pages, 512).contiguous().view(torch.int16)


def _cos_sin(positions, dim):
    """Rotation table of a program: fp32 [positions, dim], cosines then sines, angles in 64 bits."""
    freq = 500000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).to(torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dev, op, B, Hq, Hkv = "cuda", case["op"], case["B"], case["Hq"], case["Hkv"]
    own_len, new, prefix = _sizes(case)
    own_pages = [(n + PAGE - 1) // PAGE for n in own_len]
    pre_pages = [(n + PAGE - 1) // PAGE for n in prefix]
    total = sum(own_pages) + sum(pre_pages)
    pool = total + 3
    order = torch.randperm(pool, device=dev, generator=gen)[:total].to(torch.int32).split(own_pages + pre_pages)

    def table(rows):
        return torch.nn.utils.rnn.pad_sequence(list(rows), batch_first=True, padding_value=0).contiguous()

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    s = {"case": case, "pages": table(order[:B]), "ctx_len": ints(own_len), "max_ctx": max(own_len), "S": torch.from_numpy(_rotation()).to(dev)}
    if prefix:
        s.update(prefix_pages=table(order[B:]), prefix_len=ints(prefix), group_start=ints(_group_start(case)), max_prefix=max(prefix))
    s["k_codes"], s["k_radii"] = _random_pages(gen, "key", Hkv, pool)
    s["v_codes"], s["v_radii"] = _random_pages(gen, "value", Hkv, pool)
    if op in ("append", "read"):
        rows = new if op == "append" else own_len
        s["row_start"] = ints([0] + list(np.cumsum(rows)))
        n = sum(rows) + case.get("pad", 0)
        if op == "append":  # queries, keys and values of a token beside each other, as one projection leaves them
            qkv = torch.randn(n, Hq + 2 * Hkv, D, device=dev, generator=gen)
            channel = torch.rand(Hkv, D, device=dev, generator=gen).argsort(1) < 4  # four large channels of a head
            qkv[:, Hq : Hq + Hkv] *= torch.where(channel, torch.exp(2 + 0.5 * torch.randn(Hkv, D, device=dev, generator=gen)), 1.0)
            qkv = qkv.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
            s["xk"], s["xv"] = qkv[:, Hq : Hq + Hkv], qkv[:, Hq + Hkv :]
        ot = torch.float32 if op == "read" and case["dtype"] == "fp32" else torch.bfloat16
        s["out_k"], s["out_v"] = torch.zeros(n, Hkv, D, dtype=ot, device=dev), torch.zeros(n, Hkv, D, dtype=ot, device=dev)
    else:
        s["q"] = (1.5 * torch.randn(B, case["M"], Hq, D, device=dev, generator=gen)).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = 1.0 / math.sqrt(D)
    if "rot" in case:
        s["cos_sin"] = _cos_sin(max(own_len) + max(prefix or [0]), case["rot"])
    if own:
        from paper_2502_02617_amd import Context, Rotary

        s["ctx"] = _context()
        s["cache"] = (s["k_codes"], s["k_radii"], s["v_codes"], s["v_radii"])
        if "rot" in case:
            s["rotary"] = Rotary(s["cos_sin"], interleaved=case["inter"])
        if op == "attend":
            n = Context.attn_paged_workspace_bytes(B, case["M"], Hq, Hkv, s["max_ctx"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=dev)
        if op == "prefix":
            n = Context.attn_prefix_paged_workspace_bytes(B, case["M"], Hq, Hkv, s["max_ctx"], case["groups"], s["max_prefix"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------- the operators


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "prefix": _plain_prefix}[op](s)
    ctx, cache = s["ctx"], s["cache"]
    if op == "append":  # what the cache now holds comes back as the values that the codes stand for
        ctx.append_paged(s["xk"], s["xv"], s["row_start"], s["ctx_len"], *cache, s["pages"], rotary=s["rotary"])
        ctx.decode_paged(*cache, s["pages"], s["row_start"], s["ctx_len"], s["out_k"], s["out_v"])
        return s["out_k"], s["out_v"]
    if op == "read":
        ctx.decode_paged(*cache, s["pages"], s["row_start"], s["ctx_len"], s["out_k"], s["out_v"])
        return s["out_k"], s["out_v"]
    if op == "attend":
        ctx.attn_paged(s["q"], s["out"], *cache, s["pages"], s["ctx_len"], s["max_ctx"], s["scale"], s["workspace"], rotary=s["rotary"])
        return s["out"]
    ctx.attn_prefix_paged(s["q"], s["out"], *cache, s["pages"], s["ctx_len"], s["max_ctx"], s["prefix_pages"], s["prefix_len"],
                          s["group_start"], s["max_prefix"], s["scale"], s["workspace"], rotary=s["rotary"])
    return s["out"]


def _rotate(x, positions, cos_sin, inter):
    """Position rotation of the first `dim` coordinates of x [rows, heads, 128]: pairs (i, i + dim / 2), or neighbours."""
    dim = cos_sin.shape[1]
    c, s = cos_sin[positions].to(x.dtype)[:, None].chunk(2, -1)
    head, rest = x[..., :dim], x[..., dim:]
    if inter:
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat([torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2), rest], -1)
    a, b = head.chunk(2, -1)
    return torch.cat([a * c - b * s, a * s + b * c, rest], -1)


def _tables(dtype, dev):
    """cos and sin of the centroids by level."""
    t1 = (torch.arange(16, dtype=torch.float64, device=dev) + 0.5) * (math.pi / 8)
    t = {1: t1, **{l: torch.tensor(c, dtype=torch.float64, device=dev) for l, c in CENTROIDS.items()}}
    return {l: torch.stack([v.cos(), v.sin()], -1).to(dtype) for l, v in t.items()}


def _split(radius, codes, table):
    """One level down: the radius of each node times the cosine and the sine of its angle."""
    return (radius[..., None] * table[codes]).flatten(-2)


def _values(R, c4, c3, c2, c1):
    """DeQuant without the trailing S^T: block radii [..., 8] and the codes of the levels, in R's type."""
    t = _tables(R.dtype, R.device)
    return _split(_split(_split(_split(R, c4, t[4]), c3, t[3]), c2, t[2]), c1, t[1])


def _quantise(y):
    """Codes and block radii (rounded to binary16) of rotated vectors y [..., 128] in 64 bits."""
    u, v = y[..., 0::2], y[..., 1::2]
    psi = torch.atan2(v, u)
    c1 = torch.clamp(torch.floor(torch.where(psi < 0, psi + 2 * math.pi, psi) / (math.pi / 8)), 0, 15).long()
    r, codes = torch.hypot(u, v), [c1]
    for level in (2, 3, 4):
        c = CENTROIDS[level]
        u, v = r[..., 0::2], r[..., 1::2]
        psi = torch.atan2(v, u)
        codes.append((psi > (c[0] + c[1]) / 2).long() + (psi > (c[1] + c[2]) / 2) + (psi > (c[2] + c[3]) / 2))
        r = torch.hypot(u, v)
    return torch.clamp(r, max=65504.0).to(torch.float16), codes


def _row_tokens(s, rows):
    """Sequence and token of every row of `rows`, and whether a sequence has it."""
    start, row = s["row_start"].long(), torch.arange(rows, device=s["ctx_len"].device)
    b = torch.clamp(torch.searchsorted(start, row, right=True) - 1, 0, len(start) - 2)
    return b, s["ctx_len"].long()[b] - (start[b + 1] - row), row < start[-1]


def _plain_append(s):
    rows = s["xk"].shape[0]
    _, token, used = _row_tokens(s, rows)
    token = torch.clamp(token, 0, s["cos_sin"].shape[0] - 1)

    def values(x):
        R, (c1, c2, c3, c4) = _quantise(x @ s["S"])
        y = _values(R.double(), c4, c3, c2, c1) @ s["S"].T
        return torch.where(used[:, None, None], y, 0.0).to(torch.bfloat16)

    return values(_rotate(s["xk"].double(), token, s["cos_sin"], s["case"]["inter"])), values(s["xv"].double())


def _fields(dwords, bits, width):
    """Fields of `width` bits at the given bits of strings of dwords [..., n] (int64)."""
    at = torch.tensor(bits, device=dwords.device)
    d, sh = at >> 5, at & 31
    nxt = torch.clamp(d + 1, max=dwords.shape[-1] - 1)
    return (dwords[..., d] >> sh | dwords[..., nxt] << (32 - sh)) & ((1 << width) - 1)


def _key_strings(t):
    """Key pages [..., 736 dwords]: token tau owns a string of 368 bits, dwords 0-3, 4-7 and 8-10 in planes of their own and the last
    half in a plane of halves; block b from bit 46 b: four quarter indices of 10 bits, the block index of 6."""
    last = torch.stack([t[..., 704:] & 0xFFFF, t[..., 704:] >> 16], -1).flatten(-2)
    w = torch.cat([t[..., :256].unflatten(-1, (64, 4)), t[..., 256:512].unflatten(-1, (64, 4)), t[..., 512:704].unflatten(-1, (64, 3)),
                   last[..., None]], -1)
    Q = _fields(w, [46 * b + 10 * j for b in range(8) for j in range(4)], 10)
    return Q, _fields(w, [46 * b + 40 for b in range(8)], 6)


def _tokens_of_slots(x, *tail):
    """[..., g, b, ..., slot 4 i + e] -> [..., token 16 i + 4 g + e, ...]: x [..., 4, 8, k, 16] -> [..., 64, 8, k]"""
    x = x.unflatten(-1, (4, 4))  # ..., g, b, k, i, e
    n = x.dim()
    lead = list(range(n - 5))
    return x.permute(*lead, n - 2, n - 5, n - 1, n - 4, n - 3).flatten(n - 5, n - 3)


def _value_strings(t):
    """Value pages: the half-block n = 2 b + h of the tokens 16 i + 4 g + e is a string of 320 bits of 16 slots, planes of dwords 0-3, 4-7, 8-9;
    the block indices of (g, b) are strings of 96 bits."""
    w = torch.cat([t[..., :256].unflatten(-1, (64, 4)), t[..., 256:512].unflatten(-1, (64, 4)), t[..., 512:640].unflatten(-1, (64, 2))], -1)
    pair = _tokens_of_slots(_fields(w, [20 * s for s in range(16)], 20).unflatten(-2, (4, 8, 2)))  # [..., 64, 8, 2]
    Q = torch.stack([pair & 1023, pair >> 10], -1).flatten(-3)
    Bi = _fields(t[..., 640:].unflatten(-1, (32, 3)), [6 * s for s in range(16)], 6)
    return Q, _tokens_of_slots(Bi.unflatten(-2, (4, 8, 1))).squeeze(-1)


def _cached(codes, radii, kind, table):
    """Rotated-domain values fp32 [Hkv, *table, 64, 128] of the pages of `table`."""
    t = codes.view(torch.int32)[:, table.long()].long() & 0xFFFFFFFF
    Q, Bi = _key_strings(t) if kind == "key" else _value_strings(t)
    R = radii.view(torch.float16)[:, table.long()]
    R = R.unflatten(-1, (64, 8)) if kind == "key" else _tokens_of_slots(R.unflatten(-1, (4, 8, 1, 16))).squeeze(-1)
    c1 = torch.stack([Q & 15, Q >> 6], -1).flatten(-2)
    c3 = torch.stack([Bi >> 2 & 3, Bi & 3], -1).flatten(-2)
    return _values(R.float(), Bi >> 4, c3, Q >> 4 & 3, c1)


def _plain_read(s):
    b, token, _ = _row_tokens(s, s["out_k"].shape[0])

    def values(kind, codes, radii):
        y = _cached(codes, radii, kind, s["pages"]).flatten(2, 3)[:, b, token]  # [Hkv, rows, 128]
        return (y @ s["S"].float().T).transpose(0, 1).contiguous().to(s["out_k"].dtype)

    return values("key", s["k_codes"], s["k_radii"]), values("value", s["v_codes"], s["v_radii"])


def _attention(s, table, seen, positions):
    """Attention of q [B, M, Hq, 128] over the pages of `table` [B, P]; seen [B, M, 64 P]: the tokens that take part."""
    q, S = s["q"], s["S"].float()
    B, M, Hq, _ = q.shape
    Hkv = s["k_codes"].shape[0]
    K = _cached(s["k_codes"], s["k_radii"], "key", table).flatten(2, 3)  # [Hkv, B, tokens, 128]
    V = _cached(s["v_codes"], s["v_radii"], "value", table).flatten(2, 3)
    x = _rotate(q.float().flatten(0, 1), positions.flatten(), s["cos_sin"], s["case"]["inter"]) @ S
    x = x.reshape(B, M, Hkv, Hq // Hkv, D).permute(2, 0, 1, 3, 4).flatten(2, 3)  # [Hkv, B, M G, 128]
    score = torch.matmul(x, K.transpose(-1, -2)) * s["scale"]
    score = torch.where(seen.repeat_interleave(Hq // Hkv, 1), score, -math.inf)
    top = torch.clamp(score.amax(-1, keepdim=True), min=-3e38)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    V = torch.where(seen.any(1)[..., None], V, 0.0)
    o = torch.matmul(p, V) / torch.where(total > 0, total, 1.0)
    o = (o @ S.T).unflatten(2, (M, Hq // Hkv)).permute(1, 2, 0, 3, 4)
    return o.reshape(B, M, Hq, D).to(torch.bfloat16)


def _causal(length, M, tokens):
    """[B, M, tokens]: query m, the (M - 1 - m)-th newest token, sees the tokens up to its own."""
    m = torch.arange(M, device=length.device)
    return torch.arange(tokens, device=length.device) < (length[:, None] - (M - 1 - m))[..., None]


def _plain_attend(s):
    M, length = s["case"]["M"], s["ctx_len"].long()
    positions = torch.clamp(length[:, None] - M + torch.arange(M, device=length.device), min=0)
    return _attention(s, s["pages"], _causal(length, M, PAGE * s["pages"].shape[1]), positions)


def _plain_prefix(s):
    M, B, length = s["case"]["M"], s["case"]["B"], s["ctx_len"].long()
    group = torch.searchsorted(s["group_start"].long(), torch.arange(B, device=length.device), right=True) - 1
    prefix = s["prefix_len"].long()[group]
    table = torch.cat([s["prefix_pages"][group], s["pages"]], 1)
    shared = torch.arange(PAGE * s["prefix_pages"].shape[1], device=length.device) < prefix[:, None]
    seen = torch.cat([shared[:, None].expand(-1, M, -1), _causal(length, M, PAGE * s["pages"].shape[1])], -1)
    positions = torch.clamp((prefix + length)[:, None] - M + torch.arange(M, device=length.device), min=0)
    return _attention(s, table, seen, positions)


# ---------------------------------------------------------------- 64 bits, by the definitions


def _bit_places(kind):
    """Where in a page's 23552 code bits the 46 bits of block b of token tau lie: int64 [64, 8, 46], from the planes' byte positions."""
    if kind not in _kept:
        at = np.zeros((64, 8, 46), dtype=np.int64)
        for tau in range(64):
            i, g, e = tau >> 4, tau >> 2 & 3, tau & 3
            slot = 4 * i + e
            for b in range(8):
                for p in range(46):
                    if kind == "key":
                        byte, bit = divmod(46 * b + p, 8)
                        place = 16 * tau + byte if byte < 16 else 1024 + 16 * tau + byte - 16 if byte < 32 else \
                            2048 + 12 * tau + byte - 32 if byte < 44 else 2816 + 2 * tau + byte - 44
                    elif p < 40:
                        lane = 16 * g + 2 * b + p // 20
                        byte, bit = divmod(20 * slot + p % 20, 8)
                        place = 16 * lane + byte if byte < 16 else 1024 + 16 * lane + byte - 16 if byte < 32 else 2048 + 8 * lane + byte - 32
                    else:
                        byte, bit = divmod(6 * slot + p - 40, 8)
                        place = 2560 + 12 * (8 * g + b) + byte
                    at[tau, b, p] = 8 * place + bit
        _kept[kind] = at
    return _kept[kind]


def _centroid(level, dev):
    return torch.tensor([(k + 0.5) * math.pi / 8 for k in range(16)] if level == 1 else CENTROIDS[level], dtype=torch.float64, device=dev)


def _exact_rebuild(radius, angles, S):
    """Vectors from block radii [n, 8] and the angles of levels 1 to 4 ([n, 64], [n, 32], [n, 16], [n, 8]): coordinate k is its block's
    radius times, for each level, the cosine or the sine of the angle above it."""
    k = torch.arange(D, device=radius.device)
    y = radius[:, k >> 4]
    for level, a in enumerate(angles, 1):
        node = a[:, k >> level]
        y = y * torch.where((k >> (level - 1)) % 2 == 0, node.cos(), node.sin())
    return y @ S.T


def _exact_pages(s, kind, pages, head):
    """Vectors [64 len(pages), 128] that the pages of one head hold, in 64 bits."""
    dev = s["S"].device
    name = kind[0]
    raw = s[name + "_codes"][head, pages.long()]
    bits = (raw[..., None] >> torch.arange(8, device=dev, dtype=torch.uint8) & 1).flatten(1)
    block = bits[:, torch.from_numpy(_bit_places(kind)).to(dev)].flatten(0, 1).double()  # [tokens, 8, 46]

    def number(lo, n):
        return (block[..., lo : lo + n] * 2.0 ** torch.arange(n, device=dev)).sum(-1).long()

    c1 = torch.stack([number(10 * (j // 2) + (6 if j & 1 else 0), 4) for j in range(8)], -1).flatten(1)
    c2 = torch.stack([number(10 * j + 4, 2) for j in range(4)], -1).flatten(1)
    c3 = torch.stack([number(42, 2), number(40, 2)], -1).flatten(1)
    c4 = number(44, 2)
    half = s[name + "_radii"].view(torch.float16)[head, pages.long()].double()
    if kind == "key":
        radius = half.reshape(-1, 8)
    else:
        tau = torch.arange(64, device=dev)
        slot = 4 * (tau >> 4) + (tau & 3)
        radius = half[:, (16 * (8 * (tau >> 2 & 3)[:, None] + torch.arange(8, device=dev)) + slot[:, None])].flatten(0, 1)
    return _exact_rebuild(radius, [_centroid(l, dev)[c] for l, c in ((1, c1), (2, c2), (3, c3), (4, c4))], s["S"])


def _exact_turn(x, positions, cos_sin, inter):
    """Position rotation as a product with a complex number per pair."""
    dim = cos_sin.shape[1]
    t = cos_sin[positions].double()
    w = torch.complex(t[:, : dim // 2], t[:, dim // 2 :])[:, None]
    x = x.clone()
    first, second = (slice(0, dim, 2), slice(1, dim, 2)) if inter else (slice(0, dim // 2), slice(dim // 2, dim))
    z = torch.complex(x[..., first], x[..., second]) * w
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_coded(x, S):
    """What a vector becomes in the cache: Polar, the nearest centroid of every angle, the radius as binary16, DeQuant."""
    r = x @ S
    chosen = []
    for level in (1, 2, 3, 4):
        u, v = r[:, 0::2], r[:, 1::2]
        psi = torch.atan2(v, u)
        psi = torch.where(psi < 0, psi + 2 * math.pi, psi)
        c = _centroid(level, x.device)
        chosen.append(c[(psi[..., None] - c).abs().argmin(-1)])
        r = (u * u + v * v).sqrt()
    return _exact_rebuild(torch.clamp(r, max=65504.0).half().double(), chosen, S)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    own_len, new, prefix = _sizes(case)
    B, Hq, Hkv, op = case["B"], case["Hq"], case["Hkv"], case["op"]
    if op in ("append", "read"):
        out = [torch.zeros(s["out_k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        row = 0
        for b in range(B):
            n = new[b] if op == "append" else own_len[b]
            first = own_len[b] - n
            for h in range(Hkv):
                if op == "append":
                    at = torch.arange(first, first + n, device="cuda")
                    k = _exact_turn(s["xk"][row : row + n, h : h + 1].double(), at, s["cos_sin"], case["inter"])[:, 0]
                    out[0][row : row + n, h] = _exact_coded(k, s["S"])
                    out[1][row : row + n, h] = _exact_coded(s["xv"][row : row + n, h].double(), s["S"])
                else:
                    pages = s["pages"][b, : (n + PAGE - 1) // PAGE]
                    out[0][row : row + n, h] = _exact_pages(s, "key", pages, h)[:n]
                    out[1][row : row + n, h] = _exact_pages(s, "value", pages, h)[:n]
            row += n
        return tuple(out)
    M, G = case["M"], Hq // Hkv
    if B * Hkv * (max(own_len) + max(prefix or [0])) > 30_000_000:
        return None
    out = torch.zeros(B, M, Hq, D, dtype=torch.float64, device="cuda")
    start = _group_start(case) if prefix else [0, B]
    for g in range(len(start) - 1):
        P = prefix[g] if prefix else 0
        for h in range(Hkv):
            shared = [_exact_pages(s, kind, s["prefix_pages"][g, : (P + PAGE - 1) // PAGE], h)[:P] for kind in ("key", "value")] if P else None
            for b in range(start[g], start[g + 1]):
                n = own_len[b]
                K, V = (_exact_pages(s, kind, s["pages"][b, : (n + PAGE - 1) // PAGE], h)[:n] for kind in ("key", "value"))
                if P:
                    K, V = torch.cat([shared[0], K]), torch.cat([shared[1], V])
                at = torch.clamp(torch.arange(P + n - M, P + n, device="cuda"), min=0)
                q = _exact_turn(s["q"][b, :, h * G : (h + 1) * G].double(), at, s["cos_sin"], case["inter"])
                for m in range(M):
                    seen = P + max(0, n - (M - 1 - m))
                    if seen > 0:
                        p = torch.softmax((q[m] @ K[:seen].T) * s["scale"], -1)
                        out[b, m, h * G : (h + 1) * G] = p @ V[:seen]
    return out
