/*
 * pq_prefix.h -- attention of groups of sequences over their common prefix (part of pq_attn.hip, whose tables, plan
 * and partial results it uses): the prefix's keys and values are rebuilt once per block of query rows of a group
 * instead of once per sequence.
 *
 * The query rows of a group and a kv head -- every (sequence, query token, head) of it, all of which see the whole
 * prefix -- are cut into blocks; a workgroup works through the tiles of its share of a (group, block, kv head)
 * stream.  Per 64-token tile its wavefronts rebuild the keys and values once, as binary16 in LDS, and multiply
 * them by all rows on v_mfma_f32_32x32x16_f16:
 *   scores     S^T = K Q^T   (tokens x rows): lane (H, r) holds row r of its block, tokens 8 j + 4 H + {0..3}
 *   values     O^T = V^T P^T (coordinates x rows): the contraction takes the tokens in the order in which the
 *              scores lie in a lane's registers, so the weights are its operand as they are; V is
 *              laid out in that order.
 * Rounding: keys are rebuilt as the values are, radius times block table and that times quarter table in binary16 (the kernel for
 * single sequences scales its keys in fp32); weights and values as there.  Maxima, sums and results stay in fp32.
 */
#ifndef PQ_PREFIX_H
#define PQ_PREFIX_H

typedef float f16x __attribute__((ext_vector_type(16)));

constexpr int kPrefixThreads = 512;

/* A block of query rows, as the launch that builds the plan leaves it for this one: rows first .. first + rows - 1 of the group that begins with
 * sequence seq0, and the tokens of its prefix. */
struct BlockRows {
    int group, first, rows, seq0, tokens;
};

struct PrefixArgs {
    const uint16_t *qrot; /* [B][M][Hq][128] binary16 */
    const uint8_t *k_codes, *v_codes;
    const uint16_t *k_radii, *v_radii;
    int up_b5, up_b6, up_b7;
    PagedTable table; /* one row per group */
    PrefixGroups groups;
    int B, Hq, Hkv, M;
    const int32_t *plan; /* as the other kernel's, of row blocks instead of sequences and their pieces instead of tiles */
    const BlockRows *blocks;
    int n_blocks;        /* row blocks that the plan counts */
    float *ws_ml; /* [piece][ROWS][2], ROWS query rows in a block */
    float *ws_o;  /* [piece][ROWS][128] */
    const PqDeviceConsts *consts;
};

/* Row blocks of `rows` rows are numbered without a running sum: those of group g begin at start[g] * pairs / rows + g, which leaves room
 * for them (pairs = M * G rows per sequence); numbers without rows have no tokens.  Sequences ahead of start[0] and behind start[n] have no prefix. */
__device__ __forceinline__ int64_t first_block(const PrefixGroups &g, int i, int pairs, int rows)
{
    return (int64_t)max(g.start[i], 0) * pairs / rows + i;
}

/* thread by thread (no wavefront operation) */
__device__ __forceinline__ BlockRows row_block(const PrefixGroups &g, int block, int B, int pairs, int rows)
{
    BlockRows r{-1, 0, 0, 0, 0};
    int lo = 0, hi = g.n; /* the last group that begins at or ahead of the block */
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (first_block(g, mid, pairs, rows) <= block) lo = mid + 1;
        else hi = mid;
    }
    if (lo == 0) return r;
    const int i = lo - 1;
    const int s0 = min(max(g.start[i], 0), B), s1 = min(g.start[i + 1], B);
    const int64_t first = (block - first_block(g, i, pairs, rows)) * (int64_t)rows, all = (int64_t)max(s1 - s0, 0) * pairs;
    if (first >= all) return r;
    r.group = i;
    r.first = (int)first;
    r.rows = (int)min(all - first, (int64_t)rows);
    r.seq0 = s0;
    r.tokens = prefix_length(g, i);
    return r;
}

/* A sequence's rows in its group's blocks: the block that the group begins with (-1: no group) and the sequence's first row in the group. */
struct SequenceRows {
    int block, row;
};

__device__ __forceinline__ SequenceRows sequence_rows(const PrefixGroups &g, int b, int pairs, int rows)
{
    int lo = 0, hi = g.n; /* the last group that begins with the sequence or ahead of it */
    while (lo <= hi) {
        const int mid = (lo + hi) >> 1;
        if (g.start[mid] <= b) lo = mid + 1;
        else hi = mid - 1;
    }
    const int i = lo - 1;
    if (i < 0 || i >= g.n) return SequenceRows{-1, 0};
    return SequenceRows{(int)first_block(g, i, pairs, rows), (b - max(g.start[i], 0)) * pairs};
}

/* Row `i` of a group -> row of q: (sequence, query token, head of the kv head's group) */
__device__ __forceinline__ int query_row(int seq0, int i, int M, int Hq, int G, int hk)
{
    const int s = i / (M * G), rest = i - s * (M * G), m = rest / G;
    return ((seq0 + s) * M + m) * Hq + hk * G + (rest - m * G);
}

/* A tile as it is in memory, codes and radii behind them. */
struct RawTile { __attribute__((aligned(16))) uint32_t w[1024]; };

/* Place of eight tokens of a coordinate in the values' LDS: neighbouring coordinates are read together, every eighth is written together. */
__device__ __forceinline__ int value_place(int coordinate, int chunk) { return 8 * coordinate + (chunk ^ (((coordinate >> 1) ^ (coordinate >> 3)) & 7)); }

struct PrefixTables {
    __attribute__((aligned(16))) uint32_t tq[2048];
    __attribute__((aligned(16))) float tbf[64][4];
    __attribute__((aligned(16))) uint32_t tbh[128];
    float2 up[24];
};

/* What a wavefront rebuilds of a tile: block `wave` of the keys of all 64 tokens, a token per lane, and half-block n of the values of the two
 * tokens 16 i + 4 g + e0, + 1 per lane (g, n), i = wave / 2, e0 = 2 (wave % 2).  In three steps, so that other work covers their LDS
 * reads.  Tokens from nv on become zeros, whatever the page holds there; products are binary16, radius times block table times quarter table, as
 * the values' of the other kernel. */
/* Byte offsets of what it reads in a raw tile; those of the key's dwords depend on the wavefront's block. */
struct RebuildPlaces {
    uint32_t k0, k1, k2, half1, half2, v0, v1, v2, b0, b1, r;
    int ksh, vsh, bsh; /* the same in all lanes */

    __device__ __forceinline__ void set(int wave, int lane)
    {
        /* dword d of a key's string: planes of 16, 16, 12 and 2 bytes per token; of the last half what lies behind it is not looked at */
        const int bit = PQL_BLOCK_BITS * wave, d0 = bit >> 5;
        auto key = [&](int d) -> uint32_t {
            const int base = d < 4 ? PQL_OFF_P0 + 4 * d : (d < 8 ? PQL_OFF_P1 + 4 * (d - 4) : PQL_OFF_P2 + 4 * (d - 8));
            return (uint32_t)(d < 11 ? base + (d < 8 ? 16 : 12) * lane : PQL_OFF_KP3 + ((2 * lane) & ~3));
        };
        auto half = [&](int d) -> uint32_t { return d < 11 ? 0u : 16u * (lane & 1); };
        k0 = key(d0); k1 = key(d0 + 1); k2 = key(min(d0 + 2, 11));
        half1 = half(d0 + 1); half2 = half(min(d0 + 2, 11));
        ksh = bit & 31;
        /* slots s, s + 1 = 4 i + e0: bits [20 s, 20 s + 40) of the values' string, [6 s, 6 s + 12) of the block indices */
        const int s = 4 * (wave >> 1) + 2 * (wave & 1), e0 = (20 * s) >> 5;
        auto value = [&](int d) -> uint32_t {
            return (uint32_t)(d < 8 ? (d < 4 ? PQL_OFF_P0 + 4 * d : PQL_OFF_P1 + 4 * (d - 4)) + 16 * lane : PQL_OFF_P2 + 4 * (d - 8) + 8 * lane);
        };
        v0 = value(e0); v1 = value(min(e0 + 1, 9)); v2 = value(min(e0 + 2, 9));
        vsh = (20 * s) & 31;
        const int c0 = (6 * s) >> 5;
        b0 = (uint32_t)(PQL_OFF_VB + 12 * (lane >> 1) + 4 * c0);
        b1 = (uint32_t)(PQL_OFF_VB + 12 * (lane >> 1) + 4 * min(c0 + 1, 2));
        bsh = (6 * s) & 31;
        r = (uint32_t)(4 * kKeyRadii + 32 * (lane >> 1) + 2 * s);
    }
};

template <bool DEEP>
struct Rebuild {
    uint32_t kx0, kx1, vx0, vx1, vb, kr, vr;
    h2 kq[2], vq[2];   /* radii of the quarters: the key's four, the values' two of each token */
    uint2 kt[4], vt[4];

    /* the strings' dwords; `rk`, `rv` as in memory */
    __device__ __forceinline__ void fetch(const RawTile &rk, const RawTile &rv, const RebuildPlaces &at, int wave, int lane)
    {
        auto dword = [](const RawTile &t, uint32_t o) { return *reinterpret_cast<const uint32_t *>(reinterpret_cast<const char *>(t.w) + o); };
        const uint32_t w0 = dword(rk, at.k0), w1 = dword(rk, at.k1) >> at.half1, w2 = dword(rk, at.k2) >> at.half2;
        kx0 = __builtin_amdgcn_alignbit(w1, w0, at.ksh);
        kx1 = __builtin_amdgcn_alignbit(w2, w1, at.ksh);
        kr = DEEP ? rk.w[kKeyRadii + lane] : reinterpret_cast<const uint16_t *>(rk.w + kKeyRadii)[8 * lane + wave];
        const uint32_t v0 = dword(rv, at.v0), v1 = dword(rv, at.v1), v2 = dword(rv, at.v2);
        vx0 = __builtin_amdgcn_alignbit(v1, v0, at.vsh);
        vx1 = __builtin_amdgcn_alignbit(v2, v1, at.vsh);
        vb = __builtin_amdgcn_alignbit(dword(rv, at.b1), dword(rv, at.b0), at.bsh);
        if (!DEEP) vr = dword(rv, at.r);
    }

    /* the tables' entries */
    __device__ __forceinline__ void gather(const PrefixArgs &a, const PrefixTables &tab, const uint32_t *rv, int wave, int nv, int lane)
    {
        const int n = lane & 15, t0 = 16 * (wave >> 1) + 4 * (lane >> 4) + 2 * (wave & 1);
        float r = DEEP ? pq_deep_block_radius(kr, a.up_b5, a.up_b6, a.up_b7, tab.up, wave) : pq_half_bits_to_float(kr);
        if (lane >= nv) r = 0.f;
        const float4 t43 = *reinterpret_cast<const float4 *>(tab.tbf[(kx1 >> 8) & 63u]);
        if (DEEP) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) f[e] = pq_deep_block_radius(rv[kKeyRadii + t0 + e], a.up_b5, a.up_b6, a.up_b7, tab.up, n >> 1);
            vr = __builtin_bit_cast(uint32_t, h2{(_Float16)f[0], (_Float16)f[1]});
        }
        if (t0 >= nv) vr = 0u;
        else if (t0 + 1 >= nv) vr &= 0xFFFFu;
        const uint32_t h0 = tab.tbh[2 * (vb & 63u) + (n & 1)], h1 = tab.tbh[2 * ((vb >> 6) & 63u) + (n & 1)];
        const uint32_t K[4] = {kx0 & 1023u, (kx0 >> 10) & 1023u, (kx0 >> 20) & 1023u, __builtin_amdgcn_alignbit(kx1, kx0, 30) & 1023u};
        const uint32_t V[4] = {vx0 & 1023u, (vx0 >> 10) & 1023u, (vx0 >> 20) & 1023u, __builtin_amdgcn_alignbit(vx1, vx0, 30) & 1023u};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            kt[j] = *reinterpret_cast<const uint2 *>(tab.tq + 2 * K[j]);
            vt[j] = *reinterpret_cast<const uint2 *>(tab.tq + 2 * V[j]);
        }
        kq[0] = h2{(_Float16)(r * t43.x), (_Float16)(r * t43.y)};
        kq[1] = h2{(_Float16)(r * t43.z), (_Float16)(r * t43.w)};
        const h2 two = as_h2(vr);
        vq[0] = bcast_lo(two) * as_h2(h0);
        vq[1] = bcast_hi(two) * as_h2(h1);
    }

    /* their products, to LDS; token 4 g + e of sixteen goes to place 8 (g & 1) + 4 (g >> 1) + e, the order of the weights in the lanes */
    __device__ __forceinline__ void store(uint4 *sK, uint4 *sV, int wave, int lane)
    {
        H8 o[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const h2 f = (j & 1) ? bcast_hi(kq[j >> 1]) : bcast_lo(kq[j >> 1]);
            o[j >> 1].p[2 * (j & 1)] = f * as_h2(kt[j].x);
            o[j >> 1].p[2 * (j & 1) + 1] = f * as_h2(kt[j].y);
        }
        sK[16 * lane + ((2 * wave) ^ (lane & 15))] = o[0].q;
        sK[16 * lane + ((2 * wave + 1) ^ (lane & 15))] = o[1].q;
        const int g = lane >> 4, n = lane & 15, chunk = 2 * (wave >> 1) + (g & 1), part = 2 * (g >> 1) + (wave & 1);
#pragma unroll
        for (int c = 0; c < 4; ++c) { /* coordinates 2 c, 2 c + 1 of the half-block: quarter c / 2, product c % 2 */
            const h2 f0 = (c & 2) ? bcast_hi(vq[0]) : bcast_lo(vq[0]), f1 = (c & 2) ? bcast_hi(vq[1]) : bcast_lo(vq[1]);
            const uint2 t0 = vt[c >> 1], t1 = vt[2 + (c >> 1)];
            const uint32_t x = __builtin_bit_cast(uint32_t, f0 * as_h2((c & 1) ? t0.y : t0.x)), y = __builtin_bit_cast(uint32_t, f1 * as_h2((c & 1) ? t1.y : t1.x));
            reinterpret_cast<uint32_t *>(sV)[4 * value_place(8 * n + 2 * c, chunk) + part] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            reinterpret_cast<uint32_t *>(sV)[4 * value_place(8 * n + 2 * c + 1, chunk) + part] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
    }
};

/* ROWS query rows per workgroup, 32 per wavefront: of 256 a wavefront sees all tokens of a tile, of 128 two wavefronts share rows and have
 * half of the tokens each, and join their results in the end.  While a tile is multiplied the next one is rebuilt into the other half of LDS,
 * and the one after that is on its way there: one barrier per tile.  What bounds it is the chain of a wavefront's steps, two wavefronts per
 * SIMD: so all requests to LDS stand ahead of the work that covers them.  16384 tokens, 256 rows of 8 kv heads: 36 us (45 in blocks of
 * 128), 17 GFLOP at 0.48 PFLOP/s; of its cycles the matrix cores work 25 %, the vector ALU half, LDS 40 to 60 %, half of that on colliding
 * reads of the tables. */
template <bool DEEP, int ROWS>
__global__ __launch_bounds__(kPrefixThreads, 1) void pq_attn_prefix_kernel(PrefixArgs a)
{
    static_assert((ROWS == 128 || ROWS == 256) && kPrefixThreads == 512, "row groups of 32 by eight wavefronts");
    constexpr int kSlices = ROWS / 128; /* of 32 tokens, that a wavefront multiplies */
    __shared__ PrefixTables tab;
    __shared__ RawTile sRaw[2][2];                                 /* [buffer][keys, values] */
    __shared__ __attribute__((aligned(16))) uint4 sK[2][64 * 16];  /* [token][chunk of eight coordinates ^ token & 15] */
    __shared__ __attribute__((aligned(16))) uint4 sV[2][128 * 8];  /* value_place */
    __shared__ float sM[4][32][2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = (int)blockIdx.x;
    /* the plan's entries and the row blocks of up to 64 blocks lie in registers, one per lane, requested before anything else */
    const bool few = a.n_blocks < 64;
    const int total = a.plan[0], working = a.plan[1];
    const int pre = a.plan[kPlanHeader + min(lane, a.n_blocks)];
    const BlockRows mine = a.blocks[min(lane, a.n_blocks - 1)];
    {
        const uint32_t *src = a.consts->attn_tab;
        const uint4 t = reinterpret_cast<const uint4 *>(src + PQ_TAB_TQ)[tid];
        const uint32_t f = src[PQ_TAB_TBF + (tid & 255)], h = src[PQ_TAB_TBH + (tid & 127)], u = src[PQ_TAB_UP + min(tid, 47)];
        reinterpret_cast<uint4 *>(tab.tq)[tid] = t;
        if (tid < 256) (&tab.tbf[0][0])[tid] = __uint_as_float(f);
        if (tid < 128) tab.tbh[tid] = h;
        if (tid < 48) reinterpret_cast<uint32_t *>(tab.up)[tid] = u;
    }
    if (w >= working) return;
    const int base = total / working, rem = total - base * working;
    int gpos = w * base + min(w, rem);
    const int gend = min(gpos + base + (w < rem ? 1 : 0), total);
    auto prefix_at = [&](int i) { return few ? __builtin_amdgcn_readlane(pre, i) : a.plan[kPlanHeader + i]; };
    auto rows_of = [&](int i) {
        if (!few) return a.blocks[i];
        return BlockRows{__builtin_amdgcn_readlane(mine.group, i), __builtin_amdgcn_readlane(mine.first, i), __builtin_amdgcn_readlane(mine.rows, i),
                         __builtin_amdgcn_readlane(mine.seq0, i), __builtin_amdgcn_readlane(mine.tokens, i)};
    };
    /* the last row block whose streams start at or before gpos */
    int blk = few ? __popcll(__ballot(lane <= a.n_blocks && (int64_t)pre * a.Hkv <= gpos)) - 1
                  : paged_find(a.n_blocks, gpos, lane, [&](int i) { return (int64_t)a.plan[kPlanHeader + i] * a.Hkv; });
    blk = min(max(blk, 0), a.n_blocks - 1);
    int before = prefix_at(blk), block_pieces = prefix_at(blk + 1) - before;
    if (block_pieces <= 0) return; /* cannot happen with a consistent plan */
    int hk, unit; /* piece of the stream */
    {
        const int r = gpos - before * a.Hkv;
        hk = min(r / block_pieces, a.Hkv - 1);
        unit = r - hk * block_pieces;
    }
    RebuildPlaces places;
    places.set(wave, lane);
    const int G = a.Hq / a.Hkv;
    constexpr int kRadiiHalves = DEEP ? PQ_DEEP_RADII_HALVES : PQL_RADII;
    const int rg = kSlices == 1 ? wave >> 1 : wave, slice = kSlices == 1 ? wave & 1 : 0, H = lane >> 5, r32 = lane & 31;

    for (;;) { /* one piece per round */
        const BlockRows rb = rows_of(blk);
        const int units = min(block_pieces - unit, gend - gpos), tiles = (rb.tokens + 63) >> 6, c = (tiles + block_pieces - 1) / block_pieces;
        const int tile_lo = unit * c, tile_hi = min(tiles, tile_lo + units * c); /* ceil(tiles / c) is block_pieces again: none is empty */
        if (tile_lo >= tile_hi) return; /* cannot happen with a consistent plan */
        const int64_t piece = (int64_t)w + (int64_t)blk * a.Hkv + hk;
        /* keys by wavefront 0, values by wavefront 1 (wavefronts of two SIMDs); a tile without a page is passed over */
        int page_base = tile_lo; /* the table's entries of 64 tiles lie in a register, one per lane */
        int32_t page_reg = 0;
        auto fetch_pages = [&](int t) {
            page_base = t;
            page_reg = a.table.pages[(int64_t)rb.group * a.table.ld_pages + min(t + lane, tile_hi - 1)];
        };
        auto page_of = [&](int t) {
            if (t >= tile_hi) return -1;
            if (t - page_base >= 64) fetch_pages(t);
            const int p = __builtin_amdgcn_readlane(page_reg, t - page_base);
            return p >= 0 && p < a.table.pool_pages ? p : -1;
        };
        auto request = [&](int buffer, int page) {
            if (wave > 1 || page < 0) return;
            const int64_t at = (int64_t)hk * a.table.pool_pages + page;
            const uint8_t *codes = (wave ? a.v_codes : a.k_codes) + at * PQL_CODE_BYTES;
            const uint16_t *radii = (wave ? a.v_radii : a.k_radii) + at * kRadiiHalves;
            request_k_tile<DEEP>(sRaw[buffer][wave].w, stream_descriptor(codes, PQL_CODE_BYTES), stream_descriptor(radii, kRadiiHalves * 2), 0, lane);
        };
        fetch_pages(tile_lo);
        int page = page_of(tile_lo), page1 = page_of(tile_lo + 1); /* of the tile that is multiplied, and the next */
        request(tile_lo & 1, page);
        const bool real = 32 * rg + r32 < rb.rows;
        h8 q[8];
        {
            const int64_t at = (int64_t)query_row(rb.seq0, rb.first + (real ? 32 * rg + r32 : 0), a.M, a.Hq, G, hk) * PQ_D;
            const uint4 *qr = reinterpret_cast<const uint4 *>(a.qrot + at) + H;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                H8 v;
                v.q = qr[2 * ks];
                if (!real) v.q = make_uint4(0, 0, 0, 0);
                q[ks] = v.v;
            }
        }
        f16x acc[4];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
        float m_ref = 0.f, l_run = 0.f;
        float start = kProbShift; /* what a tile's scores begin with */
        bool have_ref = false;
        /* tokens of tile t that are looked at: a tile without a page has none */
        auto tokens_of = [&](int t, int p) { return p < 0 ? 0 : min(rb.tokens - 64 * t, 64); };
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads(); /* the tables and the first raw tile are there */
        request((tile_lo + 1) & 1, page1);
        {
            Rebuild<DEEP> r;
            r.fetch(sRaw[tile_lo & 1][0], sRaw[tile_lo & 1][1], places, wave, lane);
            r.gather(a, tab, sRaw[tile_lo & 1][1].w, wave, tokens_of(tile_lo, page), lane);
            r.store(sK[tile_lo & 1], sV[tile_lo & 1], wave, lane);
        }
        for (int tile = tile_lo; tile < tile_hi; ++tile) {
            const int cur = tile & 1, nxt = cur ^ 1;
            const int page2 = page_of(tile + 2);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads(); /* this tile is rebuilt, the next raw one has arrived, and nobody reads the tile before this one any more */
            request(cur, page2);
            int l = lane; /* addresses are formed where they are used: kept over the tile loop they would be spilled */
            asm volatile("" : "+v"(l));
            const int nv = tokens_of(tile, page), nv1 = tokens_of(tile + 1, page1);
            const int lH = l >> 5, lr = l & 31, tok = 32 * slice + lr;
            Rebuild<DEEP> r;
            r.fetch(sRaw[nxt][0], sRaw[nxt][1], places, wave, l);
            auto key = [&](int ks, int sl) { return sK[cur][16 * (tok + 32 * sl) + ((2 * ks + lH) ^ (tok & 15))]; };
            auto value = [&](int d, int k, int sl) { return sV[cur][value_place(32 * d + lr, 2 * (2 * (slice + sl) + k) + lH)]; };
            H8 ko[8];
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) ko[ks].q = key(ks, 0);
            r.gather(a, tab, sRaw[nxt][1].w, wave, nv1, l);
            f16x s[kSlices];
#pragma unroll
            for (int sl = 0; sl < kSlices; ++sl) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[sl][e] = start;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    s[sl] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ko[ks].v, q[ks], s[sl], 0, 0, 0);
                    if (sl + 1 < kSlices) ko[ks].q = key(ks, sl + 1);
                }
            }
            H8 vo[8];
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int k = 0; k < 2; ++k) vo[2 * d + k].q = value(d, k, 0);
            if (nv < 64) {
#pragma unroll
                for (int sl = 0; sl < kSlices; ++sl)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * (slice + sl) + 8 * (e >> 2) + 4 * lH + (e & 3) >= nv) s[sl][e] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int sl = 0; sl < kSlices; ++sl)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[sl][e]);
            /* the first tokens that this wavefront sees set the reference of its rows */
            if (nv > 32 * slice && (!have_ref || __ballot(top > kProbShift + kRefSlack) != 0ull)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                float delta = top == -INFINITY ? 0.f : top - kProbShift;
                if (have_ref) delta = fmaxf(delta, 0.f);
                const float alpha = have_ref ? __builtin_amdgcn_exp2f(-delta) : 1.f;
                m_ref += delta;
                l_run *= alpha;
                start = kProbShift - m_ref;
#pragma unroll
                for (int sl = 0; sl < kSlices; ++sl) s[sl] -= delta;
#pragma unroll
                for (int d = 0; d < 4; ++d) acc[d] *= alpha;
                have_ref = true;
            }
#pragma unroll
            for (int sl = 0; sl < kSlices; ++sl) {
                H8 p[2];
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float x = __builtin_amdgcn_exp2f(s[sl][e]), y = __builtin_amdgcn_exp2f(s[sl][e + 1]);
                    l_run += x + y;
                    p[e >> 3].p[(e & 7) >> 1] = h2{(_Float16)x, (_Float16)y};
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vo[2 * d + k].v, p[k].v, acc[d], 0, 0, 0);
                        if (sl + 1 < kSlices) vo[2 * d + k].q = value(d, k, sl + 1);
                    }
            }
            r.store(sK[nxt], sV[nxt], wave, l);
            page = page1;
            page1 = page2;
        }
        float l = l_run + __shfl_xor(l_run, 32), m = l > 0.f ? m_ref : -INFINITY;
        const int64_t out_row = piece * ROWS + 32 * rg + r32;
        if (kSlices == 2) {
            if (real) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const f16x &o = acc[k >> 2];
                    const int j = 4 * (k & 3);
                    *reinterpret_cast<float4 *>(a.ws_o + out_row * PQ_D + 8 * k + 4 * H) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                }
            }
            __syncthreads(); /* nobody reads this piece's last tile any more */
        } else {
            /* the slices' results joined (through LDS, half of the coordinates at a time), and stored */
            __syncthreads();
            if (slice == 1 && H == 0) {
                sM[rg][r32][0] = m;
                sM[rg][r32][1] = l;
            }
            float4 *theirs = reinterpret_cast<float4 *>(&sK[0][0]) + rg * 512 + lane; /* eight of 64 lanes each */
            float scale0 = 0.f, scale1 = 0.f;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (slice == 1) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const f16x &o = acc[2 * half + (k >> 2)];
                        theirs[64 * k] = make_float4(o[4 * (k & 3)], o[4 * (k & 3) + 1], o[4 * (k & 3) + 2], o[4 * (k & 3) + 3]);
                    }
                }
                __syncthreads();
                if (slice == 0) {
                    if (half == 0) {
                        const float m1 = sM[rg][r32][0], l1 = sM[rg][r32][1], mm = fmaxf(m, m1);
                        if (mm != -INFINITY) {
                            scale0 = __builtin_amdgcn_exp2f(m - mm);
                            scale1 = __builtin_amdgcn_exp2f(m1 - mm);
                        }
                        l = l * scale0 + l1 * scale1;
                        m = mm;
                    }
                    if (real) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const f16x &o = acc[2 * half + (k >> 2)];
                            const float4 t = theirs[64 * k];
                            const int j = k & 3;
                            const float4 sum = make_float4(o[4 * j] * scale0 + t.x * scale1, o[4 * j + 1] * scale0 + t.y * scale1,
                                                           o[4 * j + 2] * scale0 + t.z * scale1, o[4 * j + 3] * scale0 + t.w * scale1);
                            *reinterpret_cast<float4 *>(a.ws_o + out_row * PQ_D + 32 * (2 * half + (k >> 2)) + 8 * j + 4 * H) = sum;
                        }
                    }
                }
                __syncthreads();
            }
        }
        if (slice == 0 && real && H == 0) *reinterpret_cast<float2 *>(a.ws_ml + out_row * 2) = make_float2(m, l);

        gpos += units;
        if (gpos >= gend) return;
        unit = 0;
        if (++hk == a.Hkv) {
            hk = 0;
            do {
                if (++blk >= a.n_blocks) return;
                before = prefix_at(blk);
                block_pieces = prefix_at(blk + 1) - before;
            } while (block_pieces <= 0);
        }
    }
}

#endif /* PQ_PREFIX_H */
