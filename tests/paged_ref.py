"""Plain 64-bit counterparts of the paged calls, for their tests: page tables, ragged rows, position rotation, and records of the oracle
laid out in pages.  Nothing here comes from the kernels."""
import numpy as np
import torch

import oracle
from tests import layout_ref

KEY, VALUE = 0, 1


def cos_sin(n_pos, dim, base=10000.0):
    """float32 [n_pos, dim]: cosines, then sines."""
    a = np.arange(n_pos)[:, None] * base ** (-np.arange(0, dim, 2) / dim)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def rotate(x, positions, table, interleaved):
    """x [rows, heads, 128] float64, table float32 [n_pos, dim]"""
    dim, x = table.shape[1], x.copy()
    t = table[np.clip(positions, 0, table.shape[0] - 1)].astype(np.float64)[:, None]
    c, s = t[..., : dim // 2], t[..., dim // 2 :]
    i = np.arange(dim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
    u, v = x[..., a], x[..., b]
    x[..., a], x[..., b] = u * c - v * s, u * s + v * c
    return x


def page_table(rng, n_pages, lens, ld=None, fill=-1):
    """Distinct pages in random order for sequences of these lengths -> int32 [n_seq, ld]; entries behind a sequence's last are `fill`."""
    need = [(n + 63) // 64 for n in lens]
    order = rng.permutation(n_pages)[: sum(need)]
    t = np.full((len(lens), ld or max(1, max(need, default=1))), fill, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at : at + n]
        at += n
    return t


class Format:
    """A context and what the oracle needs of it."""

    def __init__(self, ctx, bits=None):
        self.ctx, self.bits, self.S = ctx, bits, ctx.preconditioner()
        self.cb = np.concatenate([ctx.codebook(l)[0] for l in (1, 2, 3, 4)])
        self.record = 50 if bits else 62
        self.cbt = None
        if bits:
            self.cbt = np.zeros((3, 8))
            for l in (5, 6, 7):
                c = ctx.upper_codebook(l)[1]
                self.cbt[l - 5, : c.size] = c

    def encode(self, x, **want):
        if self.bits:
            return oracle.encode_deep(x, self.S, self.cb, self.bits, self.cbt, **want)
        return oracle.encode(x, self.S, self.cb, **want)

    def decode(self, rec):
        if self.bits:
            return oracle.decode_deep(rec, self.S, self.cb, self.bits, self.cbt)
        return oracle.decode(rec, self.S, self.cb)

    def tiles(self, kind, rec, fill):
        """rec [H, n, record] -> codes uint8 [H, T, 2944], radii uint16 [H, T, halves]"""
        if not self.bits:
            return layout_ref.canonical_to_tiles_planes(kind, rec, None, fill)
        both = [layout_ref.canonical_to_tiles_deep(kind, rec[h], None, fill) for h in range(rec.shape[0])]
        return np.stack([c for c, _ in both]), np.stack([r for _, r in both])

    def records(self, kind, codes, radii):
        """The records that pages hold: codes [H, T, 2944], radii [H, T, halves] -> [H, 64 T, record]"""
        read = layout_ref.tiles_to_canonical_deep if self.bits else layout_ref.tiles_to_canonical
        return np.stack([read(kind, codes[h], radii[h], 64 * codes.shape[1]) for h in range(codes.shape[0])])

    def code_bytes(self, rec):
        """A record without its radius: its last two bytes at full depth, its last sixteen otherwise."""
        return rec[..., :48] if self.bits else rec[..., :46]

    def radii(self, rec):
        return np.ascontiguousarray(rec[..., 48:] if self.bits else rec[..., 46:]).view(np.uint16)


class Cache:
    """A paged cache on the device."""

    def __init__(self, fmt, heads, n_pages, fill=0xFF, device="cuda"):
        self.fmt, self.heads = fmt, heads
        self.kc, self.kr = fmt.ctx.alloc_cache_for(heads, 64 * n_pages, device)
        self.vc, self.vr = fmt.ctx.alloc_cache_for(heads, 64 * n_pages, device)
        for t in self.all:
            t.view(torch.uint8).fill_(fill)

    @property
    def all(self):
        return self.kc, self.kr, self.vc, self.vr

    def put(self, kind, rec, pages, fill=0xFF):
        """rec [H, n, record] to the pages given, in order; the rest of the last page gets `fill`."""
        if rec.shape[1] == 0:
            return
        c, r = self.fmt.tiles(kind, rec, fill)
        at = torch.as_tensor(np.asarray(pages[: c.shape[1]]), dtype=torch.long, device=self.kc.device)
        codes, radii = (self.kc, self.kr) if kind == KEY else (self.vc, self.vr)
        codes[:, at] = torch.from_numpy(c).to(codes.device)
        radii[:, at] = torch.from_numpy(r.view(np.int16)).to(radii.device)

    def read(self):
        """What the pages hold: [keys, values], each records [H, pages, 64, record]"""
        both = []
        for kind, codes, radii in ((KEY, self.kc, self.kr), (VALUE, self.vc, self.vr)):
            rec = self.fmt.records(kind, codes.cpu().numpy(), radii.cpu().numpy().view(np.uint16))
            both.append(rec.reshape(rec.shape[0], -1, 64, rec.shape[2]))
        return both


def tokens(held, pages, first, last):
    """Records [H, last - first, record] of tokens first .. last - 1 of a sequence, from one of Cache.read's"""
    t = np.arange(first, last)
    return held[:, np.asarray(pages)[t >> 6], t & 63]


def attention(q, K, V, scale, M):
    """q [M, Hq, 128], K, V lists over kv heads of [n, 128] with, for query m, how many tokens take part: K[h], V[h] are functions of m."""
    out = np.zeros(q.shape)
    G = q.shape[1] // len(K)
    for h in range(len(K)):
        for m in range(M):
            k, v = K[h](m), V[h](m)
            if not len(k):
                continue
            s = q[m, h * G : (h + 1) * G] @ k.T * scale
            p = np.exp(s - s.max(1, keepdims=True))
            out[m, h * G : (h + 1) * G] = p @ v / p.sum(1, keepdims=True)
    return out
