"""GPU tests of the paged cache: append with position rotation, DeQuant of pages and attention by page tables against the oracle (64 bits,
CPU) and plain counterparts of tables and rotation (paged_ref).

Codes have to be equal, all of them but those of angles that lie on a border: they are settled in 64 bits.  Radii: one binary16 rounding of an exact number, which the kernels
have to 1e-6 (helpers.check_radii).  DeQuant to fp32: products of four table entries, a radius and S in fp32, sums of 128: 1e-6 of a vector's norm
leaves room for four times the 2.2e-7 that such sums have; to bf16 half a step, 2^-8, of an element on top.  Attention: 2e-3 as for the other calls
on this cache (binary16 operands, five roundings of 2^-11 each)."""
import sys

import numpy as np
import pytest
import torch

import oracle
from paper_2502_02617_amd import Context, PolarQuantError, Rotary
from tests import helpers, layout_ref, paged_ref
from tests.paged_ref import KEY, VALUE

pytestmark = pytest.mark.gpu
DEV = "cuda"

_formats = {}


def fmt(name):
    if name not in _formats:
        bits = None
        if name == "general":
            ctx = Context(seed=3)
        elif name == "hadamard":
            ctx = Context(seed=4, hadamard=True)
        elif name == "identity":
            ctx = Context(S=np.eye(128))
        elif name == "books":
            ctx = Context(seed=5)
            cb = np.concatenate([ctx.codebook(l)[0] for l in (1, 2, 3, 4)])
            cb[:16] += 0.07 * np.sin(1.0 + 3.0 * np.arange(16))
            cb[16:] *= 0.96
            ctx.set_codebooks(cb)
        else:
            bits = (3, 1, 2) if name == "deep" else (2, 2, 2)
            ctx = Context(seed=6, hadamard=name == "deep hadamard")
            ctx.set_recursion_depth(7, bits)
        _formats[name] = paged_ref.Format(ctx, bits)
    return _formats[name]


FORMATS = ["general", "hadamard", "identity", "books", "deep", "deep hadamard"]


def say(msg):
    print(f"[gpu-test] {msg}", flush=True)
    sys.stdout.flush()


def dev32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=DEV)


def rows(rng, n, heads, dtype, extra=0):
    """[n, heads, 128] keys and values as views of one wider tensor"""
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    wide = torch.randn(n, 2 * heads + extra, 128, generator=g)
    wide[:, extra] *= torch.exp(1.5 * torch.randn(128, generator=g))
    wide = wide.to(dtype).to(DEV)
    return wide[:, extra : extra + heads], wide[:, extra + heads :]


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def near_rounding(got, want, exact_r):
    """The number of radii that differ: each by one binary16 step, and its exact value next to the border between the two."""
    bad = got != want
    if bad.any():
        lo = np.minimum(got[bad], want[bad])
        assert np.all(np.maximum(got[bad], want[bad]) - lo == 1)
        mid = 0.5 * (lo.view(np.float16).astype(np.float64) + (lo + np.uint16(1)).view(np.float16).astype(np.float64))
        assert np.all(np.abs(exact_r[bad] - mid) <= helpers.RADIUS_REL_TOL * mid)
    return int(bad.sum())


def check_exact_codes(f, got, want, psi):
    """Equal, but for angles on a border itself (S of signs makes coordinates of bf16 vectors that are exactly zero or equal): y's sums of 128 products
    are off by up to 128 * 2^-53 of the vector's norm in any order, 1.6e-13 of a typical pair, whose length is an eighth of the norm; 1e-12 leaves room
    for pairs six times shorter."""
    if np.array_equal(f.code_bytes(got), f.code_bytes(want)):
        return
    Jg = layout_ref.unpack_canonical_deep(got, f.bits)[0] if f.bits else layout_ref.unpack_canonical(got)[0]
    Jo = oracle.unpack_deep(want, f.bits)[0] if f.bits else oracle.unpack(want)[0]
    bad = Jg != Jo
    assert not bad[:, 120:].any()
    dist = helpers.boundary_distance(psi[:, :120], f.cb if f is _formats.get("books") else None)
    assert dist[bad[:, :120]].max() <= 1e-12, dist[bad[:, :120]].max()


def check_appended(f, cache, pages, lens, new, xk, xv, positions, table, interleaved):
    row = off = count = 0
    held = cache.read()
    for b, (n, m) in enumerate(zip(lens, new)):
        for kind, x in ((KEY, xk), (VALUE, xv)):
            v = f64(x[row : row + m])
            if kind == KEY and table is not None:
                v = paged_ref.rotate(v, positions[row : row + m], table, interleaved)
            v = np.ascontiguousarray(v.transpose(1, 0, 2)).reshape(-1, 128)
            if not len(v):
                continue
            want, psi, y = f.encode(v, want_psi=True, want_y=True)
            got = paged_ref.tokens(held[kind], pages[b], n - m, n).reshape(-1, f.record)
            check_exact_codes(f, got, want, psi)
            # a few vectors at a time: the rate over them all is checked below (one radius of 32 is over any rate)
            exact_r = np.linalg.norm(y, axis=1, keepdims=True) if f.bits else np.linalg.norm(y.reshape(-1, 8, 16), axis=2)
            off, count = off + near_rounding(f.radii(got), f.radii(want), exact_r), count + exact_r.size
        row += m
    assert off <= max(2, helpers.RADIUS_MISMATCH_RATE * count), (off, count)


# before, new: tokens cached and appended per sequence
BATCHES = [
    ([0], [1]),
    ([63, 64, 0, 5], [1, 1, 1, 1]),
    ([0, 10, 64, 130], [64, 0, 200, 3]),
    ([1, 0, 0, 60, 127, 7], [0, 0, 130, 5, 1, 70]),
    ([(11 * i) % 70 for i in range(70)], [1 + (7 * i) % 3 for i in range(70)]),
    ([37], [700]),
    ([5, 0, 63, 200, 64], [300, 64, 1, 129, 190]),      # whole tiles of several sequences
    ([0, 7, 130, 1], [400, 1, 133, 0]),
]


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_append(name, batch):
    before, new = BATCHES[batch]
    f, rng = fmt(name), np.random.default_rng(batch)
    # S = I leaves bf16 coordinates as they are, and two equal ones lie on a cell border exactly
    dtype = torch.float32 if (batch + len(name)) % 2 or name == "identity" else torch.bfloat16
    heads, dim, inter = (3, 64, True) if batch % 2 else (2, 128, False)
    lens = [a + b for a, b in zip(before, new)]
    pages = paged_ref.page_table(rng, 4 + sum((n + 63) // 64 for n in lens), lens)
    pad = 2 if batch % 3 == 0 else 0
    say(f"append {name} batch {batch} {dtype}")
    cache = paged_ref.Cache(f, heads, 4 + sum((n + 63) // 64 for n in lens), fill=0x5A)
    xk, xv = rows(rng, sum(new) + pad, heads, dtype, extra=2)
    table = paged_ref.cos_sin(max(lens) - 1 if max(lens) > 1 else 1, dim)
    was = [t.clone() for t in cache.all]
    f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + new)), dev32(lens), *cache.all, dev32(pages), rotary=Rotary(torch.from_numpy(table).to(DEV), inter))
    torch.cuda.synchronize()
    positions = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)] or [np.zeros(0, int)])
    check_appended(f, cache, pages, lens, new, xk, xv, positions, table, inter)
    # the slots that the call does not name keep their contents: earlier tokens, the rest of last pages, pages of nobody
    untouched = np.ones((cache.kc.shape[1], 64), bool)
    for b, (n, m) in enumerate(zip(lens, new)):
        t = np.arange(n - m, n)
        untouched[pages[b][t >> 6], t & 63] = False
    held = cache.read()
    for t, w in zip(cache.all, was):
        t.copy_(w)
    for now, before_it in zip(held, cache.read()):
        assert np.array_equal(now[:, untouched], before_it[:, untouched])


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_in_chunks_and_one_by_one(name, dtype):
    """Codes do not depend on the batch a vector comes in: 20000 tokens of two sequences as chunks and as 20000 rows of their own.  Radii may differ by a
    rounding, as everywhere, one in a thousand of them at most."""
    f, rng = fmt(name), np.random.default_rng(3)
    n, heads = 20000, 2
    lens, new = [n // 2 + 37, n // 2 + 5], [n // 2, n // 2]
    n_pages = sum((m + 63) // 64 for m in lens)
    pages = paged_ref.page_table(rng, n_pages, lens)
    xk, xv = rows(rng, n, heads, dtype)
    if name == "identity":      # coordinates that differ, so that none lies on a cell border
        xk, xv = (xk.float() + torch.rand(xk.shape, device=DEV) * 1e-3 for _ in range(2)) if dtype == torch.float32 else (xk, xv)
    rot = Rotary(torch.from_numpy(paged_ref.cos_sin(n, 128)).to(DEV))
    caches = [paged_ref.Cache(f, heads, n_pages, fill=0) for _ in range(2)]
    f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + new)), dev32(lens), *caches[0].all, dev32(pages), rotary=rot)
    token = np.concatenate([np.arange(m - k, m) for m, k in zip(lens, new)])
    each = np.repeat(pages, new, axis=0)
    f.ctx.append_paged(xk, xv, dev32(np.arange(n + 1)), dev32(token + 1), *caches[1].all, dev32(each), rotary=rot)
    torch.cuda.synchronize()
    a, b = caches
    assert torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)
    for x, y in ((a.kr, b.kr), (a.vr, b.vr)):
        if f.bits:      # words of a radius and codes
            x, y = x.view(torch.int32), y.view(torch.int32)
            assert torch.equal(x & 0xFFFF, y & 0xFFFF)
            x, y = x >> 16, y >> 16
        step = (x.int() - y.int()).abs()
        assert int(step.max()) <= 1 and float((step > 0).float().mean()) <= 1e-3


def appended_both_ways(f, xk, xv, lens, new, heads, n_pages):
    """Caches of the same rows appended in chunks, and as rows of their own."""
    pages = paged_ref.page_table(np.random.default_rng(3), n_pages, lens)
    caches = [paged_ref.Cache(f, heads, n_pages, fill=0) for _ in range(2)]
    f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + new)), dev32(lens), *caches[0].all, dev32(pages))
    token = np.concatenate([np.arange(m - k, m) for m, k in zip(lens, new)])
    f.ctx.append_paged(xk, xv, dev32(np.arange(len(token) + 1)), dev32(token + 1), *caches[1].all, dev32(np.repeat(pages, new, axis=0)))
    torch.cuda.synchronize()
    return caches


def test_append_of_vectors_that_all_lie_on_borders():
    """S = I and pairs of equal coordinates: an angle of pi/4, a border of the first level's four cells, in every vector; all of them go through the
    64-bit step, more than 256 of a workgroup."""
    f, heads, n = fmt("identity"), 8, 10240
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, 2 * heads, 128, generator=g).to(torch.bfloat16)
    x[:, :, 1] = x[:, :, 0]
    x[:, :, 77] = -x[:, :, 76]
    x = x.to(DEV)
    a, b = appended_both_ways(f, x[:, :heads], x[:, heads:], [n + 5], [n], heads, 161)
    assert torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)


@pytest.mark.parametrize("heads,n", [(1, 1031), (3, 683), (1, 4099)])
def test_append_of_single_rows_in_several_rounds(heads, n):
    """More rows of their own than one round of the workgroups takes, and a last round in part."""
    f = fmt("general")
    xk, xv = rows(np.random.default_rng(n), n, heads, torch.bfloat16)
    a, b = appended_both_ways(f, xk, xv, [n + 5], [n], heads, (n + 68) // 64)
    assert torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc) and bool((a.vc != 0).any())


@pytest.mark.parametrize("name", ["general", "hadamard", "deep"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_very_small_and_very_large_vectors(name, dtype):
    """Codes do not depend on a vector's length, from 1e-30 to 1e30; vectors of zeros, infinities and NaN leave their neighbours alone."""
    f, heads, n = fmt(name), 2, 640
    g = torch.Generator().manual_seed(5)
    x = torch.randn(n, 2 * heads, 128, generator=g)
    x[1::2] *= torch.exp2(torch.randint(-100, 101, (n // 2, 1, 1), generator=g).float())
    x = x.to(dtype)
    odd = {100: 0.0, 201: float("inf"), 302: float("nan"), 303: -float("inf")}
    for row, value in odd.items():
        x[row] = value
    x = x.to(DEV)
    for cache in appended_both_ways(f, x[:, :heads], x[:, heads:], [n + 5], [n], heads, 11):
        held, pages = cache.read(), paged_ref.page_table(np.random.default_rng(3), 11, [n + 5])
        sound = np.array([r for r in range(n) if r not in odd])
        for kind, part in ((KEY, x[:, :heads]), (VALUE, x[:, heads:])):
            got = paged_ref.tokens(held[kind], pages[0], 5, n + 5).reshape(heads, n, f.record)
            for h in range(heads):
                want, psi, _ = f.encode(f64(part[sound, h]), want_psi=True, want_y=True)
                check_exact_codes(f, np.ascontiguousarray(got[h][sound]), want, psi)
                assert np.array_equal(f.radii(got[h][100:101]), f.radii(f.encode(np.zeros((1, 128)))))


def test_append_with_more_tile_numbers_than_the_workgroups_take():
    """300 sequences of 14 rows and 64 heads: more than 65536 (tile, head, keys or values) numbers."""
    f, heads, B = fmt("general"), 64, 300
    lens, new = [(3 * i) % 100 + 14 for i in range(B)], [14] * B
    n_pages = sum((n + 63) // 64 for n in lens)
    xk, xv = rows(np.random.default_rng(2), 14 * B, heads, torch.bfloat16)
    a, b = appended_both_ways(f, xk, xv, lens, new, heads, n_pages)
    assert torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)
    assert bool((a.kc != 0).any())


@pytest.mark.parametrize("name", ["general", "deep"])
def test_append_positions_without_table_and_rows_of_nobody(name):
    """Given positions; no rotation; tokens without a page, negative tokens and rows behind the last sequence write nothing."""
    f, rng = fmt(name), np.random.default_rng(5)
    lens, new = [100, 3, 70], [40, 5, 70]          # sequence 1 has fewer tokens than rows: two rows belong to no token
    pages = paged_ref.page_table(rng, 9, lens)
    pages[2, 0] = 9                                # not in the pool
    cache = paged_ref.Cache(f, 2, 9)
    xk, xv = rows(rng, 120, 2, torch.bfloat16)
    table = paged_ref.cos_sin(500, 32)
    positions = rng.integers(-5, 600, size=120)
    start = [0, 40, 45, 115]
    f.ctx.append_paged(xk, xv, dev32(start), dev32(lens), *cache.all, dev32(pages), rotary=Rotary(torch.from_numpy(table).to(DEV)),
                       positions=dev32(positions))
    torch.cuda.synchronize()
    check_appended(f, cache, pages, lens[:1], new[:1], xk, xv, positions, table, False)
    check_appended(f, cache, pages[1:], [3], [3], xk[42:], xv[42:], positions[42:], table, False)
    check_appended(f, cache, pages[2:, 1:], [6], [6], xk[109:], xv[109:], positions[109:], table, False)
    used = pages[(pages >= 0) & (pages < 9)]
    for t in cache.all:
        left = t.view(torch.uint8)[:, np.setdiff1d(np.arange(9), used)]
        assert bool((left == 0xFF).all())
    f.ctx.append_paged(xk, xv, dev32(start), dev32(lens), *cache.all, dev32(pages))
    torch.cuda.synchronize()
    check_appended(f, cache, pages, lens[:1], new[:1], xk, xv, None, None, False)


def filled(f, rng, lens, heads, n_pages, ld=None):
    """A cache of random vectors encoded by the oracle -> (cache, pages, vectors per sequence: [heads][n, 128] keys, values)"""
    pages = paged_ref.page_table(rng, n_pages, lens, ld)
    cache = paged_ref.Cache(f, heads, n_pages)
    vectors = []
    for b, n in enumerate(lens):
        kv = []
        for kind in (KEY, VALUE):
            x = rng.standard_normal((heads, n, 128)) * np.exp(0.3 * rng.standard_normal((heads, n, 1)))
            rec = f.encode(x.reshape(-1, 128)).reshape(heads, n, f.record) if n else np.zeros((heads, 0, f.record), np.uint8)
            cache.put(kind, rec, pages[b])
            kv.append([f.decode(rec[h]) if n else np.zeros((0, 128)) for h in range(heads)])
        vectors.append(kv)
    return cache, pages, vectors


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("lens,take", [([1], [1]), ([130, 0, 64, 63], [130, 0, 64, 63]), ([100, 200, 65, 5], [1, 137, 2, 5]),
                                       (list(range(1, 70)), [1 + i % 2 for i in range(69)]), ([1500], [1411])])
def test_decode(name, lens, take):
    take = [min(a, b) for a, b in zip(take, lens)]
    f, rng = fmt(name), np.random.default_rng(len(lens))
    heads = 3
    say(f"decode_paged {name} {len(lens)} sequences")
    cache, pages, vectors = filled(f, rng, lens, heads, 3 + sum((n + 63) // 64 for n in lens))
    start = np.cumsum([0] + take)
    want = [np.concatenate([np.stack(kv[kind], 1)[n - t :] for kv, n, t in zip(vectors, lens, take)]) for kind in (KEY, VALUE)]
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.full((2, int(start[-1]) + 2, heads + 1, 128), 7.0, dtype=dtype, device=DEV)
        out = [wide[0, :, :heads], wide[1, :, :heads]]
        f.ctx.decode_paged(*cache.all, dev32(pages), dev32(start), dev32(lens), out[0], out[1])
        torch.cuda.synchronize()
        for o, w in zip(out, want):
            got = f64(o)[: start[-1]]
            norm = np.linalg.norm(w, axis=-1, keepdims=True)
            half_step = 0 if dtype == torch.float32 else 2.0**-8 * np.abs(w)
            assert np.all(np.abs(got - w) <= half_step + 1e-6 * norm)
        assert bool((wide[:, :, heads] == 7).all()) and bool((wide[:, start[-1] :] == 7).all())
        only = torch.zeros_like(wide[1, :, :heads])
        f.ctx.decode_paged(*cache.all, dev32(pages), dev32(start), dev32(lens), None, only)
        assert torch.equal(only[: start[-1]], out[1][: start[-1]])


def test_decode_of_missing_pages_and_of_nobody():
    f, rng = fmt("general"), np.random.default_rng(8)
    cache, pages, vectors = filled(f, rng, [200, 3], 2, 8)
    pages[0, 1], pages[0, 3] = -1, 8
    start = [0, 200, 205]                                # sequence 1: two rows more than it has tokens
    out = [torch.full((206, 2, 128), 7.0, device=DEV) for _ in range(2)]
    f.ctx.decode_paged(*cache.all, dev32(pages), dev32(start), dev32([200, 3]), *out)
    torch.cuda.synchronize()
    for kind, o in enumerate(out):
        got, w = f64(o), np.stack(vectors[0][kind], 1)
        w[64:128] = 0
        w[192:] = 0
        assert np.all(got[64:128] == 0) and np.all(got[192:200] == 0)
        assert np.abs(got[:200] - w).max() <= 1e-6 * np.linalg.norm(w, axis=-1).max()
        assert np.all(got[200:202] == 7) and np.all(got[205] == 7)
        assert np.abs(got[202:205] - np.stack(vectors[1][kind], 1)).max() <= 1e-4


def reference(vectors, q, lens, M, scale, table=None, interleaved=False, positions=None, missing=()):
    """q [B, M, Hq, 128] -> attention in 64 bits; missing: (sequence, page) pairs without a page"""
    out = np.zeros(q.shape)
    for b, n in enumerate(lens):
        qb = q[b]
        if table is not None:
            at = positions[b] if positions is not None else np.arange(n - M, n)
            qb = paged_ref.rotate(qb, at, table, interleaved)
        gone = np.zeros(n, bool)
        for s, p in missing:
            if s == b:
                gone[64 * p : 64 * p + 64] = True

        def part(x):
            return lambda m: x[: max(0, n - (M - 1 - m))][~gone[: max(0, n - (M - 1 - m))]]

        out[b] = paged_ref.attention(qb, [part(k) for k in vectors[b][0]], [part(v) for v in vectors[b][1]], scale, M)
    return out


def attend(f, cache, pages, lens, q, out_dtype=torch.float32, max_ctx=None, **kw):
    B, M, Hq, _ = q.shape
    max_ctx = max_ctx or max(1, max(lens))
    out = torch.full(q.shape, float("nan"), dtype=out_dtype, device=DEV)
    ws = torch.full((Context.attn_paged_workspace_bytes(B, M, Hq, cache.heads, max_ctx),), 0xFF, dtype=torch.uint8, device=DEV)
    f.ctx.attn_paged(q, out, *cache.all, dev32(pages), dev32(lens), max_ctx, helpers.softmax_scale(), ws, **kw)
    torch.cuda.synchronize()
    return out


def check_rows(got, ref, lens):
    assert np.all(np.isfinite(got))
    for b in range(len(lens)):
        if lens[b] == 0:
            assert np.all(got[b] == 0)
    assert helpers.rel_l2(got, ref) <= 2e-3
    worst = max([helpers.rel_l2(got[b], ref[b]) for b in range(len(lens)) if np.any(ref[b])], default=0.0)
    say(f"  rel L2 {helpers.rel_l2(got, ref):.2e}, worst sequence {worst:.2e}")
    assert worst <= 4e-3


@pytest.mark.parametrize("name", ["general", "hadamard", "books", "deep"])
@pytest.mark.parametrize("Hq,Hkv,M", [(8, 2, 1), (7, 1, 1), (16, 1, 1), (4, 4, 3), (14, 2, 2), (5, 1, 3), (32, 8, 4)])
def test_attention(name, Hq, Hkv, M):
    f, rng = fmt(name), np.random.default_rng(Hq + M)
    lens = [1, 0, 64, 700, 65, 128, 3, 31]
    say(f"attn_paged {name} Hq={Hq} Hkv={Hkv} M={M}")
    cache, pages, vectors = filled(f, rng, lens, Hkv, 30)
    q = torch.randn(len(lens), M, Hq, 128, generator=torch.Generator().manual_seed(Hq)).to(torch.bfloat16).to(DEV)
    table, inter = paged_ref.cos_sin(650, 64 if M > 1 else 128), M == 2
    got = attend(f, cache, pages, lens, q, rotary=Rotary(torch.from_numpy(table).to(DEV), inter))
    check_rows(f64(got), reference(vectors, f64(q), lens, M, helpers.softmax_scale(), table, inter), lens)
    plain = attend(f, cache, pages, lens, q)
    check_rows(f64(plain), reference(vectors, f64(q), lens, M, helpers.softmax_scale()), lens)
    assert torch.equal(attend(f, cache, pages, lens, q, torch.bfloat16), plain.to(torch.bfloat16))


@pytest.mark.parametrize("M", [1, 3])
def test_paged_attention_equals_that_of_a_contiguous_cache(M):
    """Pages in order are a contiguous cache: the same kernels, the same bits."""
    f, rng = fmt("general"), np.random.default_rng(3)
    lens, Hkv, Hq = [1000, 64, 3000], 2, 8
    cache, _, _ = filled(f, rng, [64 * 64], Hkv, 64)
    ids = np.arange(64)
    cache2 = paged_ref.Cache(f, Hkv, 64)
    order = rng.permutation(64)
    for a, b in zip(cache2.all, cache.all):
        a[:, order] = b[:, ids]
    starts = [0, 1024, 1088]
    pages = np.full((3, 50), -7)
    for b, n in enumerate(lens):
        k = (n + 63) // 64
        pages[b, :k] = order[starts[b] // 64 : starts[b] // 64 + k]
    q = torch.randn(3, M, Hq, 128, device=DEV).to(torch.bfloat16)
    out = torch.empty(q.shape, device=DEV)
    ws = torch.empty(Context.attn_mq_workspace_bytes(3, M, Hq, Hkv, 3000), dtype=torch.uint8, device=DEV)
    f.ctx.attn_decode_polar_mq(q, out, *cache.all, torch.tensor(starts, device=DEV), dev32(lens), 3000, helpers.softmax_scale(), ws)
    torch.cuda.synchronize()
    assert torch.equal(attend(f, cache2, pages, lens, q, max_ctx=3000), out)


@pytest.mark.parametrize("Hq,M", [(2, 1), (8, 1), (8, 2)])
def test_attention_passes_over_missing_pages(Hq, M):
    f, rng = fmt("general"), np.random.default_rng(11)
    lens = [64 * 70 + 5, 200, 64, 130]
    cache, pages, vectors = filled(f, rng, lens, 1, 90)
    missing = [(0, p) for p in range(0, 65)] + [(0, 70), (1, 3), (2, 0), (3, 1)]
    for b, p in missing:
        pages[b, p] = -1 if p % 2 else 90
    q = torch.randn(4, M, Hq, 128, device=DEV).to(torch.bfloat16)
    got = f64(attend(f, cache, pages, lens, q))
    assert np.all(got[2] == 0)
    check_rows(got, reference(vectors, f64(q), lens, M, helpers.softmax_scale(), missing=missing), lens)


@pytest.mark.parametrize("name", ["general", "deep"])
@pytest.mark.parametrize("Hq,M", [(16, 1), (64, 1), (40, 3)])
def test_attention_under_a_large_largest_context(name, Hq, M):
    """The kernels' variants for many tiles are chosen by the largest context: four, eight and fifteen pairs per kv head."""
    f, rng = fmt(name), np.random.default_rng(15)
    lens = [300, 0, 1, 64, 129, 700, 65, 3]
    cache, pages, vectors = filled(f, rng, lens, 8, 40, ld=1000)
    pages[5, 4] = -1
    q = torch.randn(8, M, Hq, 128, device=DEV).to(torch.bfloat16)
    got = f64(attend(f, cache, pages, lens, q, max_ctx=64000))
    check_rows(got, reference(vectors, f64(q), lens, M, helpers.softmax_scale(), missing=[(5, 4)]), lens)


def test_attention_of_many_sequences_and_given_positions():
    """More sequences than the kernels keep lengths of in LDS, and more than one round of the row search."""
    f, rng = fmt("general"), np.random.default_rng(12)
    lens = [int(n) for n in rng.integers(0, 150, size=150)]
    cache, pages, vectors = filled(f, rng, lens, 1, 400, ld=6)
    q = torch.randn(150, 2, 4, 128, device=DEV).to(torch.bfloat16)
    table, positions = paged_ref.cos_sin(300, 128), rng.integers(-3, 310, size=(150, 2))
    got = f64(attend(f, cache, pages, lens, q, max_ctx=380, rotary=Rotary(torch.from_numpy(table).to(DEV)), positions=dev32(positions)))
    check_rows(got, reference(vectors, f64(q), lens, 2, helpers.softmax_scale(), table, False, positions), lens)


def test_a_serving_run():
    """Prompts in chunks, then steps of one token, every call on a side stream; the attention sees exactly what was appended."""
    f, rng = fmt("general"), np.random.default_rng(13)
    Hq, Hkv, B = 8, 2, 3
    table = paged_ref.cos_sin(400, 128)
    rotary = Rotary(torch.from_numpy(table).to(DEV))
    final = [130, 64, 200]
    pages = paged_ref.page_table(rng, 20, final)
    cache = paged_ref.Cache(f, Hkv, 20)
    lens, chunks, seen = [0] * B, [[100, 60, 1], [27, 1, 190], [1, 1, 1], [1, 1, 1], [1, 1, 1]], [[[], []] for _ in range(B)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for new in chunks:
        lens = [a + b for a, b in zip(lens, new)]
        xk, xv = rows(rng, sum(new), Hkv, torch.bfloat16, extra=Hq)
        at = 0
        for b, m in enumerate(new):
            k = paged_ref.rotate(f64(xk[at : at + m]), np.arange(lens[b] - m, lens[b]), table, False)
            seen[b][0].append(k)
            seen[b][1].append(f64(xv[at : at + m]))
            at += m
        q = torch.randn(B, 1, Hq, 128, device=DEV).to(torch.bfloat16)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + new)), dev32(lens), *cache.all, dev32(pages), rotary=rotary)
            got = attend(f, cache, pages, lens, q, max_ctx=200, rotary=rotary)
        vectors = [[[f.decode(f.encode(np.concatenate(s)[:, h])) for h in range(Hkv)] for s in kv] for kv in seen]
        check_rows(f64(got), reference(vectors, f64(q), lens, 1, helpers.softmax_scale(), table), lens)
    total = sum(lens)
    out = [torch.empty(total, Hkv, 128, device=DEV) for _ in range(2)]
    f.ctx.decode_paged(*cache.all, dev32(pages), dev32(np.cumsum([0] + lens)), dev32(lens), *out)
    for kind in (KEY, VALUE):
        want = np.concatenate([np.stack(kv[kind], 1) for kv in vectors])
        assert helpers.rel_l2(f64(out[kind]), want) <= 1e-3   # a radius may differ by one rounding
    assert all(len(np.concatenate(s[0])) == n for s, n in zip(seen, lens)) and lens == [130, 64, 194]


def test_captured_steps_follow_the_lengths_on_the_device():
    """Append and attention captured once, replayed while lengths and rows change in place."""
    f, rng = fmt("general"), np.random.default_rng(14)
    Hq, Hkv, B = 8, 2, 4
    start = [60, 0, 127, 190]
    cache, pages, vectors = filled(f, rng, start, Hkv, 24, ld=5)
    spare = iter(np.setdiff1d(np.arange(24), pages[pages >= 0]))
    for b in range(B):
        for j in range(5):
            if pages[b, j] < 0:
                pages[b, j] = next(spare)
    table = dev32(pages)
    ctx_len, row_start = dev32(start), dev32(np.arange(B + 1))
    xk = torch.zeros(B, Hkv, 128, dtype=torch.bfloat16, device=DEV)
    xv, q = torch.zeros_like(xk), torch.zeros(B, 1, Hq, 128, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(B, 1, Hq, 128, device=DEV)
    ws = torch.empty(Context.attn_paged_workspace_bytes(B, 1, Hq, Hkv, 320), dtype=torch.uint8, device=DEV)

    def step(o):
        f.ctx.append_paged(xk, xv, row_start, ctx_len, *cache.all, table)
        f.ctx.attn_paged(q, o, *cache.all, table, ctx_len, 320, helpers.softmax_scale(), ws)

    f.ctx.prepare_device()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    lens, eager = list(start), torch.zeros_like(out)
    for i in range(5):
        ctx_len += 1
        lens = [n + 1 for n in lens]
        for t in (xk, xv, q):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(31 * i + t.shape[1])).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            for kind, x in ((0, xk), (1, xv)):
                for h in range(Hkv):
                    new = f.decode(f.encode(f64(x[b, h : h + 1])))
                    vectors[b][kind][h] = np.concatenate([vectors[b][kind][h], new])
        check_rows(f64(out), reference(vectors, f64(q), lens, 1, helpers.softmax_scale()), lens)
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, out)


def test_refused_calls_leave_the_outputs_alone():
    f = fmt("general")
    cache = paged_ref.Cache(f, 2, 4)
    q = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16, device=DEV)
    out = torch.full(q.shape, 7.0, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    pages = dev32([[0, 1], [2, 3]])
    with pytest.raises(PolarQuantError, match="EINVAL"):
        f.ctx.attn_paged(q, out, *cache.all, pages, dev32([1, 1]), 129, 0.1, ws)   # the table is too short for max_ctx
    with pytest.raises(PolarQuantError, match="int32"):
        f.ctx.attn_paged(q, out, *cache.all, pages.long(), dev32([1, 1]), 128, 0.1, ws)
    with pytest.raises(PolarQuantError):
        f.ctx.attn_paged(q.float(), out, *cache.all, pages, dev32([1, 1]), 128, 0.1, ws)
    assert bool((out == 7).all())
