"""GPU tests of attention with common prefixes (pq_attn_prefix_paged) against attention in 64 bits over prefix and own tokens.
Tolerance: 2e-3 as for the other calls; keys and values are rebuilt by binary16 products, two more roundings of 2^-11 of an element."""
import numpy as np
import pytest
import torch

from paper_2502_02617_amd import Context, Rotary
from tests import helpers, paged_ref
from tests.test_gpu_paged import DEV, check_rows, dev32, f64, filled, fmt, rows, say

pytestmark = pytest.mark.gpu


class Batch:
    """Groups of sequences; sizes: sequences of every group, prefix: its length, own: lengths of all sequences (ungrouped ones `ahead` and
    `behind` the groups among them)."""

    def __init__(self, f, seed, sizes, prefix, own, Hkv, ahead=0, missing=()):
        self.f, self.Hkv, self.own, self.prefix = f, Hkv, own, prefix
        self.start = list(np.cumsum([ahead] + list(sizes)))
        self.group = [-1] * ahead + [g for g, n in enumerate(sizes) for _ in range(n)] + [-1] * (len(own) - self.start[-1])
        rng = np.random.default_rng(seed)
        lens = list(prefix) + list(own)
        self.cache, pages, vectors = filled(f, rng, lens, Hkv, 2 + sum((n + 63) // 64 for n in lens))
        n = len(prefix)
        self.pre_pages, self.pages, self.pre_vectors, self.vectors = pages[:n].copy(), pages[n:].copy(), vectors[:n], vectors[n:]
        self.missing = missing
        for g, p in missing:
            self.pre_pages[g, p] = -1 if p % 2 else self.cache.kc.shape[1]

    def run(self, q, out_dtype=torch.float32, max_prefix=None, max_ctx=None, **kw):
        B, M, Hq, _ = q.shape
        max_prefix, max_ctx = max_prefix or max(self.prefix), max_ctx if max_ctx is not None else max(self.own)
        out = torch.full(q.shape, float("nan"), dtype=out_dtype, device=DEV)
        n = Context.attn_prefix_paged_workspace_bytes(B, M, Hq, self.Hkv, max_ctx, len(self.prefix), max_prefix)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
        self.f.ctx.attn_prefix_paged(q, out, *self.cache.all, dev32(self.pages), dev32(self.own), max_ctx, dev32(self.pre_pages),
                                     dev32(self.prefix), dev32(self.start), max_prefix, helpers.softmax_scale(), ws, **kw)
        torch.cuda.synchronize()
        return out

    def want(self, q, table=None, interleaved=False, positions=None):
        M, out = q.shape[1], np.zeros(q.shape)
        for b, n in enumerate(self.own):
            g = self.group[b]
            P = self.prefix[g] if g >= 0 else 0
            keep = np.ones(P, bool)
            for h, p in self.missing:
                if h == g:
                    keep[64 * p : 64 * p + 64] = False
            qb = q[b]
            if table is not None:
                qb = paged_ref.rotate(qb, positions[b] if positions is not None else np.arange(P + n - M, P + n), table, interleaved)

            def part(kind, h):
                before = self.pre_vectors[g][kind][h][keep] if g >= 0 else np.zeros((0, 128))
                return lambda m: np.concatenate([before, self.vectors[b][kind][h][: max(0, n - (M - 1 - m))]])

            out[b] = paged_ref.attention(qb, [part(0, h) for h in range(self.Hkv)], [part(1, h) for h in range(self.Hkv)], helpers.softmax_scale(), M)
        return out

    def total(self):
        return [n + (self.prefix[g] if g >= 0 else 0) for n, g in zip(self.own, self.group)]


def queries(B, M, Hq, seed):
    return torch.randn(B, M, Hq, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


SHAPES = [  # sizes, prefix, own, Hq, Hkv, M, ahead
    ([3], [200], [1, 70, 0], 8, 2, 1, 0),
    ([2], [1], [5, 64], 4, 4, 1, 0),                                            # one token
    ([1, 0, 4, 2], [130, 64, 0, 33], [3, 0, 1, 100, 65, 2, 64], 7, 1, 2, 0),     # an empty group, an empty prefix, half a tile
    ([5, 6], [1000, 777], [0, 9, 300, 1, 1, 20, 0, 64, 128, 7, 2, 40, 50], 14, 2, 1, 1),   # sequences ahead of the groups and behind
    ([40], [300], [(7 * i) % 90 for i in range(40)], 4, 1, 1, 0),                # rows of two blocks
    ([9, 35], [150, 450], [(5 * i) % 70 for i in range(44)], 16, 1, 1, 0),       # 144 and 560 rows
    ([12], [260], [3 + (5 * i) % 70 for i in range(12)], 8, 1, 2, 0),
]


@pytest.mark.parametrize("name", ["general", "hadamard", "books", "deep"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_attention(name, shape):
    sizes, prefix, own, Hq, Hkv, M, ahead = SHAPES[shape]
    batch = Batch(fmt(name), shape, sizes, prefix, own, Hkv, ahead)
    B = len(own)
    say(f"attn_prefix_paged {name} {sizes} {prefix}")
    q = queries(B, M, Hq, shape)
    table, inter = paged_ref.cos_sin(900, 64 if shape % 2 else 128), shape % 2 == 1
    got = batch.run(q, rotary=Rotary(torch.from_numpy(table).to(DEV), inter))
    check_rows(f64(got), batch.want(f64(q), table, inter), batch.total())
    plain = batch.run(q)
    check_rows(f64(plain), batch.want(f64(q)), batch.total())
    assert torch.equal(batch.run(q, torch.bfloat16), plain.to(torch.bfloat16))
    assert torch.equal(batch.run(q), plain)      # equal calls give equal bits


def test_long_prefix_in_many_pieces_with_missing_pages():
    """4170 tokens of one kv head over all workgroups, a page missing in the middle, the first and the last tile."""
    batch = Batch(fmt("general"), 5, [33], [64 * 65 + 10], [i for i in range(33)], 1, 0, missing=[(0, 0), (0, 30), (0, 65)])
    q = queries(33, 1, 8, 5)
    check_rows(f64(batch.run(q)), batch.want(f64(q)), batch.total())


def test_a_prefix_without_any_page_and_no_tokens():
    batch = Batch(fmt("general"), 6, [2, 2], [100, 128], [0, 0, 0, 5], 2, 0, missing=[(0, 0), (0, 1)])
    q = queries(4, 1, 4, 6)
    got = f64(batch.run(q, max_ctx=64))
    assert np.all(got[:2] == 0)
    check_rows(got, batch.want(f64(q)), [0, 0, 128, 133])


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_small_and_large_keys(size):
    """Scores of a thousandth and of thirty times the usual size.  Roundings to binary16 have an rms of 2e-4: four of them in each of a score's 128 products
    (query, the key's two products and its table's entry) leave 4e-4 of its rms: nothing at a thousandth, 1.2 % of the weights' exponent at 30 (scores of
    rms 30), below 2e-2."""
    f = fmt("general")
    batch = Batch(f, 7, [20], [500], [10] * 20, 1)
    q = (queries(20, 1, 8, 7).float() * size).to(torch.bfloat16)
    ref, got = batch.want(f64(q)), f64(batch.run(q))
    assert helpers.rel_l2(got, ref) <= (2e-3 if size < 1 else 2e-2)


def test_prefix_equals_joined_tables():
    """The same tokens as one sequence: attn_paged on the joined page tables."""
    f = fmt("general")
    batch = Batch(f, 8, [6, 5], [320, 64], [1, 64, 100, 7, 65, 30, 2, 3, 200, 9, 128], 2)
    q = queries(11, 1, 8, 8)
    table = Rotary(torch.from_numpy(paged_ref.cos_sin(600, 128)).to(DEV))
    joined = np.full((11, 12), -1)
    for b, g in enumerate(batch.group):
        k, own = batch.prefix[g] // 64, (batch.own[b] + 63) // 64
        joined[b, :k] = batch.pre_pages[g, :k]
        joined[b, k : k + own] = batch.pages[b, :own]
    lens = batch.total()
    out = torch.empty(q.shape, device=DEV)
    ws = torch.empty(Context.attn_paged_workspace_bytes(11, 1, 8, 2, 500), dtype=torch.uint8, device=DEV)
    f.ctx.attn_paged(q, out, *batch.cache.all, dev32(joined), dev32(lens), 500, helpers.softmax_scale(), ws, rotary=table)
    torch.cuda.synchronize()
    assert helpers.rel_l2(f64(batch.run(q, rotary=table)), f64(out)) <= 2e-3
    positions = dev32([[n - 1] for n in lens])
    assert torch.equal(batch.run(q, rotary=table, positions=positions), batch.run(q, rotary=table))


def test_no_groups_is_attn_paged():
    f = fmt("general")
    batch = Batch(f, 9, [], [], [1, 64, 100], 2)
    q = queries(3, 1, 8, 9)
    out = torch.full(q.shape, float("nan"), device=DEV)
    ws = torch.empty(Context.attn_prefix_paged_workspace_bytes(3, 1, 8, 2, 100, 0, 0), dtype=torch.uint8, device=DEV)
    none = torch.zeros(0, 1, dtype=torch.int32, device=DEV)
    f.ctx.attn_prefix_paged(q, out, *batch.cache.all, dev32(batch.pages), dev32(batch.own), 100, none, none[:, 0], dev32([0]), 0,
                            helpers.softmax_scale(), ws)
    torch.cuda.synchronize()
    check_rows(f64(out), batch.want(f64(q)), batch.own)


def test_captured_with_lengths_that_grow():
    f = fmt("general")
    batch = Batch(f, 10, [3, 4], [190, 70], [30, 60, 1, 64, 10, 20, 90], 2)
    q, M = torch.zeros(7, 1, 8, 128, dtype=torch.bfloat16, device=DEV), 1
    out, eager = torch.zeros(q.shape, device=DEV), torch.zeros(q.shape, device=DEV)
    ws = torch.empty(Context.attn_prefix_paged_workspace_bytes(7, M, 8, 2, 90, 2, 190), dtype=torch.uint8, device=DEV)
    own, prefix = dev32([0] * 7), dev32([0, 0])
    args = dev32(batch.pages), dev32(batch.pre_pages), dev32(batch.start)
    f.ctx.prepare_device()

    def call(o):
        f.ctx.attn_prefix_paged(q, o, *batch.cache.all, args[0], own, 90, args[1], prefix, args[2], 190, helpers.softmax_scale(), ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    full_own, full_prefix = list(batch.own), list(batch.prefix)
    for i in range(4):
        batch.own = [max(0, n - 10 * (3 - i)) for n in full_own]
        batch.prefix = [max(0, n - 50 * (3 - i)) for n in full_prefix]
        own.copy_(dev32(batch.own))
        prefix.copy_(dev32(batch.prefix))
        q.copy_(queries(7, 1, 8, 100 + i))
        graph.replay()
        torch.cuda.synchronize()
        short = Batch.__new__(Batch)
        short.__dict__.update(batch.__dict__)
        short.vectors = [[[x[:n] for x in kind] for kind in v] for v, n in zip(batch.vectors, batch.own)]
        short.pre_vectors = [[[x[:n] for x in kind] for kind in v] for v, n in zip(batch.pre_vectors, batch.prefix)]
        check_rows(f64(out), short.want(f64(q)), short.total())
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, out)


@pytest.mark.parametrize("shape", [(80, 2, 8, 4, 140), (70, 9, 64, 4, 70)])
def test_more_row_blocks_than_lanes_and_more_streams_than_workgroups(shape):
    """Groups x kv heads above 256: a workgroup goes on from one stream into the next; blocks of 128 rows, and of 256."""
    groups, each, Hq, Hkv, longest = shape
    f, rng = fmt("general"), np.random.default_rng(21)
    prefix = [int(n) for n in rng.integers(0, longest, size=groups)]
    sizes = [int(n) for n in rng.integers(0, each + 1, size=groups)] if each < 3 else [each] * groups
    own = [int(n) for n in rng.integers(0, 20, size=sum(sizes) + 2)]
    batch = Batch(f, 21, sizes, prefix, own, Hkv, ahead=1)
    q = queries(len(own), 1, Hq, 21)
    check_rows(f64(batch.run(q)), batch.want(f64(q)), batch.total())


def test_two_calls_at_once():
    """Two streams, two workspaces: the results of calls one after the other."""
    f = fmt("general")
    batches = [Batch(f, 30 + i, [20], [3000 + 500 * i], [40] * 20, 2) for i in range(2)]
    q = [queries(20, 1, 8, 30 + i) for i in range(2)]
    one_by_one = [b.run(x) for b, x in zip(batches, q)]
    n = Context.attn_prefix_paged_workspace_bytes(20, 1, 8, 2, 40, 1, 3500)
    outs, streams = [torch.empty(q[0].shape, device=DEV) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    args = [(dev32(b.pages), dev32(b.own), dev32(b.pre_pages), dev32(b.prefix), dev32(b.start), torch.empty(n, dtype=torch.uint8, device=DEV))
            for b in batches]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, x, o, s, (pages, own, pre, length, start, ws) in zip(batches, q, outs, streams, args):
            with torch.cuda.stream(s):
                f.ctx.attn_prefix_paged(x, o, *b.cache.all, pages, own, 40, pre, length, start, b.prefix[0], helpers.softmax_scale(), ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one_by_one, outs))


def test_a_serving_run_with_a_common_prompt():
    """A prompt appended once in two chunks, questions of three sequences behind it, single tokens: append, attention with the prefix, DeQuant."""
    f, rng = fmt("general"), np.random.default_rng(17)
    Hq, Hkv, B, P = 8, 2, 3, 150
    table = paged_ref.cos_sin(400, 128)
    rotary = Rotary(torch.from_numpy(table).to(DEV))
    pages = paged_ref.page_table(rng, 14, [P] + [120] * B)
    cache = paged_ref.Cache(f, Hkv, 14)
    prompt, lens, seen = [], 0, [[[], []] for _ in range(B)]
    for m in (100, 50):
        lens += m
        xk, xv = rows(rng, m, Hkv, torch.bfloat16)
        f.ctx.append_paged(xk, xv, dev32([0, m]), dev32([lens]), *cache.all, dev32(pages[:1]), rotary=rotary)
        prompt.append((paged_ref.rotate(f64(xk), np.arange(lens - m, lens), table, False), f64(xv)))
    held = [f.decode(f.encode(np.concatenate([c[kind] for c in prompt])[:, h])) for kind in (0, 1) for h in range(Hkv)]
    out = [torch.empty(P, Hkv, 128, device=DEV) for _ in range(2)]
    f.ctx.decode_paged(*cache.all, dev32(pages[:1]), dev32([0, P]), dev32([P]), *out)
    assert all(helpers.rel_l2(f64(out[kind][:, h]), held[kind * Hkv + h]) <= 1e-3 for kind in (0, 1) for h in range(Hkv))
    own = [0] * B
    for new in ([30, 1, 64], [1, 1, 1], [1, 1, 1]):
        own = [a + b for a, b in zip(own, new)]
        xk, xv = rows(rng, sum(new), Hkv, torch.bfloat16, extra=Hq)
        at = np.concatenate([np.arange(P + n - m, P + n) for n, m in zip(own, new)])
        f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + new)), dev32(own), *cache.all, dev32(pages[1:]), rotary=rotary, positions=dev32(at))
        k, v, row = paged_ref.rotate(f64(xk), at, table, False), f64(xv), 0
        for b, m in enumerate(new):
            seen[b][0].append(k[row : row + m])
            seen[b][1].append(v[row : row + m])
            row += m
        q = queries(B, 1, Hq, own[0])
        got = torch.empty(q.shape, device=DEV)
        ws = torch.empty(Context.attn_prefix_paged_workspace_bytes(B, 1, Hq, Hkv, 120, 1, P), dtype=torch.uint8, device=DEV)
        f.ctx.attn_prefix_paged(q, got, *cache.all, dev32(pages[1:]), dev32(own), 120, dev32(pages[:1]), dev32([P]), dev32([0, B]), P,
                                helpers.softmax_scale(), ws, rotary=rotary)
        torch.cuda.synchronize()
        want = np.zeros(q.shape)
        for b in range(B):
            mine = [f.decode(f.encode(np.concatenate(seen[b][kind])[:, h])) for kind in (0, 1) for h in range(Hkv)]
            keys, values = ([(lambda m, x=np.concatenate([held[kind * Hkv + h], mine[kind * Hkv + h]]): x) for h in range(Hkv)] for kind in (0, 1))
            qb = paged_ref.rotate(f64(q)[b], np.array([P + own[b] - 1]), table, False)
            want[b] = paged_ref.attention(qb, keys, values, helpers.softmax_scale(), 1)
        check_rows(f64(got), want, [P + n for n in own])


def test_pages_whose_bytes_lie_beyond_32_bits():
    """A head plane of 4.4 GB: the same calls on pages at its ends and on a pool of eight pages give the same bits."""
    f, rng = fmt("general"), np.random.default_rng(23)
    n_pages, Hq, lens = 1_500_000, 4, [190, 64, 130]
    small = paged_ref.page_table(rng, 8, lens)
    names = np.array([n_pages - 1, 0, 1_458_889, 7, n_pages - 2, 1_458_888, 1_459_000, 1])  # 1458888 * 2944 is just below 2^32
    large = np.where(small >= 0, names[small], -1)
    xk, xv = rows(rng, sum(lens), 1, torch.bfloat16)
    q = queries(2, 1, Hq, 23)
    results = []
    for table, pool in ((small, 8), (large, n_pages)):
        cache = paged_ref.Cache(f, 1, pool)
        f.ctx.append_paged(xk, xv, dev32(np.cumsum([0] + lens)), dev32(lens), *cache.all, dev32(table))
        f.ctx.append_paged(xk[:3], xv[:3], dev32([0, 1, 2, 3]), dev32([n - 5 for n in lens]), *cache.all, dev32(table))
        out = [torch.zeros(sum(lens), 1, 128, device=DEV) for _ in range(2)]
        f.ctx.decode_paged(*cache.all, dev32(table), dev32(np.cumsum([0] + lens)), dev32(lens), *out)
        plain, shared = torch.zeros(q.shape, device=DEV), torch.zeros(q.shape, device=DEV)
        ws = torch.empty(Context.attn_prefix_paged_workspace_bytes(2, 1, Hq, 1, 190, 1, 130), dtype=torch.uint8, device=DEV)
        f.ctx.attn_paged(q, plain, *cache.all, dev32(table[:2]), dev32(lens[:2]), 190, helpers.softmax_scale(), ws)
        f.ctx.attn_prefix_paged(q, shared, *cache.all, dev32(table[:2]), dev32(lens[:2]), 190, dev32(table[2:]), dev32(lens[2:]), dev32([0, 2]), 130,
                                helpers.softmax_scale(), ws)
        torch.cuda.synchronize()
        results.append(out + [plain, shared])
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*results)) and all(bool(torch.isfinite(a).all()) and bool(a.any()) for a in results[0])
