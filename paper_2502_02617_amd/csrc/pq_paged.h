/*
 * pq_paged.h -- device code shared by the kernels of the paged cache: which
 * sequence, page and slot a row of a ragged batch belongs to, and the position
 * rotation of queries and keys.
 */
#ifndef PQ_PAGED_H
#define PQ_PAGED_H

#include "pq_common.h"

/* A paged cache's tables: page p of a head plane is its tile p; token t of sequence b lies in slot t & 63 of page
 * pages[b * ld_pages + (t >> 6)]. */
struct PagedTable {
    const int32_t *pages;
    int64_t ld_pages;
    int64_t pool_pages;
};

/* Ragged rows: row_start[b] .. row_start[b + 1] - 1 are the newest tokens of sequence b, the last one its token ctx_len[b] - 1. */
struct PagedRows {
    const int32_t *row_start, *ctx_len;
    int n_seq;
    int64_t n_rows;
};

/* Position rotation; cs NULL: none.  Row p of the table: dim / 2 cosines, then dim / 2 sines. */
struct RotaryArgs {
    const float *cs;
    int64_t n_pos;
    int dim;
    int interleaved;
};

static inline RotaryArgs pq_rotary_args(const pq_rotary *r)
{
    return r ? RotaryArgs{r->cos_sin, r->n_pos, r->dim, r->interleaved} : RotaryArgs{nullptr, 0, 0, 0};
}

static inline pq_status pq_check_rotary(const pq_rotary *r)
{
    if (!r) return PQ_OK;
    if (!r->cos_sin || r->n_pos <= 0 || r->n_pos > 0x7FFFFFFF || r->dim <= 0 || r->dim > PQ_D) return PQ_EINVAL;
    if (r->dim % 16) return PQ_EUNSUPPORTED;
    return pq_aligned16(r->cos_sin) ? PQ_OK : PQ_EALIGN;
}

#if defined(__HIPCC__)

/* Entries of the table outside the pool name no page. */
__device__ __forceinline__ int64_t paged_page(const PagedTable &t, int b, int64_t token)
{
    if (token < 0 || (token >> 6) >= t.ld_pages) return -1;
    const int32_t p = t.pages[(int64_t)b * t.ld_pages + (token >> 6)];
    return p >= 0 && p < t.pool_pages ? p : -1;
}

/* The number of entries of the non-decreasing start[0 .. n] at or below `value`, less one: the last sequence that starts there or
 * before (n if value lies behind the last row, -1 ahead of the first).  All lanes of the wavefront take part and get the same. */
template <typename At>
__device__ __forceinline__ int paged_find(int n, int64_t value, int lane, At start_at)
{
    int cnt = 0;
    for (int base = 0; base <= n; base += 64) {
        const int i = base + lane;
        cnt += __popcll(__ballot(i <= n && start_at(min(i, n)) <= value));
    }
    return __builtin_amdgcn_readfirstlane(cnt) - 1;
}

/* A page with rows: its slot tau is row row0 + tau, as far as that is in [lo, hi), and token token0 + tau of its sequence.
 * page -1: the sequence has none there. */
struct PagedTile {
    int64_t page, row0, lo, hi, token0;
};

/* The tiles of sequence b that hold rows are numbered from row_start[b] / 64 + 2 b on -- n rows that begin anywhere in a tile lie
 * in n / 64 + 2 tiles at most, so the ranges do not meet, and no running sum has to be built first.  Numbers run below paged_tile_numbers;
 * those without a tile have no rows (lo == hi).  All lanes of the wavefront take part. */
static inline int64_t paged_tile_numbers(int64_t n_rows, int n_seq) { return n_rows / 64 + 2 * (int64_t)n_seq; }

__device__ __forceinline__ PagedTile paged_tile(const PagedTable &t, const PagedRows &r, int64_t u, int lane)
{
    PagedTile p{-1, 0, 0, 0, 0};
    auto offset = [&](int i) { return (int64_t)(max(r.row_start[i], 0) >> 6) + 2 * i; };
    const int b = paged_find(r.n_seq, u, lane, offset);
    if (b < 0 || b >= r.n_seq) return p;
    const int64_t end = r.row_start[b + 1], n = end - r.row_start[b], ctx = r.ctx_len[b];
    const int64_t first = max(ctx - n, (int64_t)0);
    const int64_t t0 = ((first >> 6) + (u - offset(b))) * 64;
    if (n <= 0 || t0 >= ctx) return p;
    p.page = paged_page(t, b, t0);
    p.row0 = end - ctx + t0;
    p.lo = max(end - ctx + first, (int64_t)0);
    p.hi = min(end, r.n_rows);
    p.token0 = t0;
    return p;
}

/* Where coordinate j of a rotated vector comes from: x_j cos + sign x_partner sin, entries `at` of the two halves of a table row.
 * Pairs are (2 i, 2 i + 1) or (i, i + dim / 2). */
struct RotaryPair {
    int partner, at;
    bool minus;
};

__device__ __forceinline__ RotaryPair rotary_pair(const RotaryArgs &r, int j)
{
    if (r.interleaved) return RotaryPair{j ^ 1, j >> 1, (j & 1) == 0};
    const int h = r.dim >> 1;
    return j < h ? RotaryPair{j + h, j, true} : RotaryPair{j - h, j - h, false};
}

__device__ __forceinline__ const float *rotary_row(const RotaryArgs &r, int64_t position)
{
    const int64_t p = position < 0 ? 0 : (position >= r.n_pos ? r.n_pos - 1 : position);
    return r.cs + p * r.dim;
}

#endif /* __HIPCC__ */
#endif /* PQ_PAGED_H */
