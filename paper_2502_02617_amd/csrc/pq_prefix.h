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
 * Rounding: a key's element is rounded to binary16 once, as the rotated query's is; weights and values as in the
 * kernel for single sequences.  Maxima, sums and results stay in fp32.
 */
#ifndef PQ_PREFIX_H
#define PQ_PREFIX_H

typedef float f16x __attribute__((ext_vector_type(16)));

constexpr int kPrefixThreads = 512, kPrefixRows = 128;

struct PrefixArgs {
    const uint16_t *qrot; /* [B][M][Hq][128] binary16 */
    const uint8_t *k_codes, *v_codes;
    const uint16_t *k_radii, *v_radii;
    int up_b5, up_b6, up_b7;
    PagedTable table; /* one row per group */
    PrefixGroups groups;
    int B, Hq, Hkv, M;
    const int32_t *plan; /* as the other kernel's, of row blocks instead of sequences */
    int n_blocks;        /* row blocks that the plan counts */
    float *ws_ml; /* [piece][ROWS][2] */
    float *ws_o;  /* [piece][ROWS][128] */
    const PqDeviceConsts *consts;
};

/* Row blocks of `rows` rows, numbered without a running sum: those of group g begin at start[g] * pairs / rows + g, which leaves room
 * for them (pairs = M * G rows per sequence).  Sequences ahead of start[0] and behind start[n] have no prefix. */
struct RowBlock {
    int group;     /* -1: none */
    int first;     /* first row of the group in the block */
    int rows;      /* of the block */
    int seq0;      /* first sequence of the group */
    int tiles;     /* of the prefix */
};

__device__ __forceinline__ int64_t first_block(const PrefixGroups &g, int i, int pairs, int rows)
{
    return (int64_t)max(g.start[i], 0) * pairs / rows + i;
}

/* thread by thread (no wavefront operation) */
__device__ __forceinline__ RowBlock row_block(const PrefixGroups &g, int block, int B, int pairs, int rows)
{
    RowBlock r{-1, 0, 0, 0, 0};
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
    r.tiles = (prefix_length(g, i) + 63) >> 6;
    return r;
}

/* Row `i` of a group -> row of q: (sequence, query token, head of the kv head's group) */
__device__ __forceinline__ int query_row(int seq0, int i, int M, int Hq, int G, int hk)
{
    const int s = i / (M * G), rest = i - s * (M * G), m = rest / G;
    return ((seq0 + s) * M + m) * Hq + hk * G + (rest - m * G);
}

/* A tile as it is in memory, codes and radii, to LDS (8 loads in all of the wavefronts that call it). */
struct RawTile { __attribute__((aligned(16))) uint32_t w[1024]; };

/* ROWS = 32 * ROW_WAVES rows per workgroup; 8 / ROW_WAVES wavefronts share a tile's tokens. */
template <int ROW_WAVES, bool DEEP>
__global__ __launch_bounds__(kPrefixThreads, 1) void pq_attn_prefix_kernel(PrefixArgs a)
{
    constexpr int kRows = 32 * ROW_WAVES, kSlices = 8 / ROW_WAVES; /* token slices of 32 */
    static_assert(ROW_WAVES == 4 && kSlices == 2 && kRows == kPrefixRows, "a tile is two slices of 32 tokens");
    __shared__ __attribute__((aligned(16))) uint32_t sTQ[2048];
    __shared__ __attribute__((aligned(16))) float sTBF[64][4];
    __shared__ __attribute__((aligned(16))) uint32_t sTBH[128];
    __shared__ float2 sUp[24];
    __shared__ RawTile sRaw[2][2]; /* [buffer][keys, values] */
    __shared__ __attribute__((aligned(16))) uint4 sK[64 * 16];  /* [token][chunk of eight coordinates ^ token & 15] */
    __shared__ __attribute__((aligned(16))) uint4 sV[128 * 8];  /* [coordinate][chunk of eight tokens ^ value_swizzle] */
    __shared__ __attribute__((aligned(16))) uint16_t sVrad[DEEP ? 512 : 8];
    __shared__ float sM[ROW_WAVES][32][2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int total = a.plan[0], working = a.plan[1];
    const int w = (int)blockIdx.x;
    {
        const uint32_t *src = a.consts->attn_tab;
        reinterpret_cast<uint4 *>(sTQ)[tid] = reinterpret_cast<const uint4 *>(src + PQ_TAB_TQ)[tid];
        if (tid < 256) (&sTBF[0][0])[tid] = __uint_as_float(src[PQ_TAB_TBF + tid]);
        if (tid < 128) sTBH[tid] = src[PQ_TAB_TBH + tid];
        if (tid < 48) reinterpret_cast<uint32_t *>(sUp)[tid] = src[PQ_TAB_UP + tid];
    }
    __syncthreads();
    if (w >= working) return;
    const int base = total / working, rem = total - base * working;
    int gpos = w * base + min(w, rem);
    const int gend = min(gpos + base + (w < rem ? 1 : 0), total);
    /* the last row block whose streams start at or before gpos */
    int blk = paged_find(a.n_blocks, gpos, lane, [&](int i) { return (int64_t)a.plan[kPlanHeader + i] * a.Hkv; });
    blk = min(max(blk, 0), a.n_blocks - 1);
    int before = a.plan[kPlanHeader + blk], block_tiles = a.plan[kPlanHeader + blk + 1] - before;
    if (block_tiles <= 0) return;
    int hk, tile_lo;
    {
        const int r = gpos - before * a.Hkv;
        hk = min(r / block_tiles, a.Hkv - 1);
        tile_lo = r - hk * block_tiles;
    }
    const int G = a.Hq / a.Hkv, pairs = a.M * G;
    constexpr int kRadiiHalves = DEEP ? PQ_DEEP_RADII_HALVES : PQL_RADII;
    const int rg = wave / kSlices, slice = wave % kSlices, H = lane >> 5, r32 = lane & 31;
    auto value_swizzle = [](int c) { return ((c >> 1) ^ (c >> 3)) & 7; };

    for (;;) { /* one piece per round */
        const RowBlock rb = row_block(a.groups, blk, a.B, pairs, kRows);
        const int n_tok = rb.group >= 0 ? prefix_length(a.groups, rb.group) : 0;
        const int tile_hi = min((n_tok + 63) >> 6, tile_lo + (gend - gpos));
        const int piece_tiles = tile_hi - tile_lo;
        if (piece_tiles <= 0) return; /* cannot happen with a consistent plan */
        const int64_t piece = (int64_t)w + (int64_t)blk * a.Hkv + hk;
        const int row = rb.first + 32 * rg + r32; /* of the group */
        const bool real = 32 * rg + r32 < rb.rows;
        h8 q[8];
        {
            const int64_t at = (int64_t)query_row(rb.seq0, real ? row : rb.first, a.M, a.Hq, G, hk) * PQ_D;
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
        bool have_ref = false;

        /* keys by wavefront 0, values by wavefront 1; false: the tile has no page and is passed over */
        auto page_of = [&](int t) { return paged_page(a.table, rb.group, (int64_t)t * 64); };
        auto request = [&](int buffer, int64_t page) {
            if (wave > 1 || page < 0) return;
            const int64_t at = (int64_t)hk * a.table.pool_pages + page;
            const uint8_t *codes = (wave ? a.v_codes : a.k_codes) + at * PQL_CODE_BYTES;
            const uint16_t *radii = (wave ? a.v_radii : a.k_radii) + at * kRadiiHalves;
            request_k_tile<DEEP>(sRaw[buffer][wave].w, stream_descriptor(codes, PQL_CODE_BYTES), stream_descriptor(radii, kRadiiHalves * 2), 0, lane);
        };
        int64_t page = page_of(tile_lo);
        request(0, page);
        for (int tile = tile_lo; tile < tile_hi; ++tile) {
            const int buffer = (tile - tile_lo) & 1;
            const int64_t next_page = tile + 1 < tile_hi ? page_of(tile + 1) : -1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads(); /* the raw tile has arrived, and nobody reads the tile before it any more */
            request(buffer ^ 1, next_page);
            const bool missing = page < 0;
            page = next_page;
            if (missing) continue;
            const int nv = min(n_tok - 64 * tile, 64); /* tokens of the tile */
            const uint32_t *rk = sRaw[buffer][0].w, *rv = sRaw[buffer][1].w;
            if (DEEP && wave < 4) { /* radii of the blocks, in the order of a depth-4 tile */
                if (wave == 0) {
                    float r[8];
                    pq_deep_block_radii(rv[kKeyRadii + lane], a.up_b5, a.up_b6, a.up_b7, sUp, r);
                    const int i = lane >> 4, g = (lane >> 2) & 3, e = lane & 3;
#pragma unroll
                    for (int b = 0; b < 8; ++b) sVrad[(8 * g + b) * 16 + 4 * i + e] = __builtin_bit_cast(uint16_t, (_Float16)r[b]);
                }
            }
            if (DEEP) __syncthreads();
            if (wave >= 4) { /* keys: two blocks per wavefront, a token per lane */
                const int tau = lane;
                float r8[8];
                if (DEEP) pq_deep_block_radii(rk[kKeyRadii + tau], a.up_b5, a.up_b6, a.up_b7, sUp, r8);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int b = 2 * (wave - 4) + k;
                    auto dword = [&](int d) -> uint32_t {
                        if (d < 4) return rk[4 * tau + d];
                        if (d < 8) return rk[256 + 4 * tau + d - 4];
                        if (d < 11) return rk[512 + 3 * tau + d - 8];
                        return reinterpret_cast<const uint16_t *>(rk)[PQL_OFF_KP3 / 2 + tau];
                    };
                    const int bit = PQL_BLOCK_BITS * b, d0 = bit >> 5, sh = bit & 31;
                    const uint32_t w0 = dword(d0), w1 = dword(d0 + 1), w2 = d0 + 2 < 12 ? dword(d0 + 2) : 0u;
                    const uint32_t x[2] = {__builtin_amdgcn_alignbit(w1, w0, sh), __builtin_amdgcn_alignbit(w2, w1, sh)};
                    float r;
                    if (DEEP) {
                        r = r8[0];
#pragma unroll
                        for (int e = 1; e < 8; ++e) r = b == e ? r8[e] : r;
                    } else {
                        r = pq_half_bits_to_float(reinterpret_cast<const uint16_t *>(rk + kKeyRadii)[8 * tau + b]);
                    }
                    if (tau >= nv) r = 0.f;
                    const float4 t43 = *reinterpret_cast<const float4 *>(sTBF[(x[1] >> 8) & 63u]);
                    const float rq[4] = {r * t43.x, r * t43.y, r * t43.z, r * t43.w};
                    const uint32_t Q[4] = {x[0] & 1023u, (x[0] >> 10) & 1023u, (x[0] >> 20) & 1023u, __builtin_amdgcn_alignbit(x[1], x[0], 30) & 1023u};
                    H8 o[2];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint2 t = *reinterpret_cast<const uint2 *>(sTQ + 2 * Q[j]);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const h2 two = as_h2(c ? t.y : t.x);
                            o[j >> 1].p[2 * (j & 1) + c] = h2{(_Float16)(rq[j] * (float)two.x), (_Float16)(rq[j] * (float)two.y)};
                        }
                    }
                    sK[16 * tau + ((2 * b) ^ (tau & 15))] = o[0].q;
                    sK[16 * tau + ((2 * b + 1) ^ (tau & 15))] = o[1].q;
                }
            } else { /* values: sixteen tokens per wavefront, lane (g, n) four of them of half-block n */
                const int i = wave, g = lane >> 4, n = lane & 15;
                auto dword = [&](int d) { return d < 4 ? rv[4 * lane + d] : (d < 8 ? rv[256 + 4 * lane + d - 4] : rv[512 + 2 * lane + d - 8]); };
                /* slots 4 i .. 4 i + 3: bits [80 i, 80 i + 80) of the string, [24 i, 24 i + 24) of the block indices */
                const int d0 = (80 * i) >> 5, sh = (80 * i) & 31;
                const uint32_t w0 = dword(d0), w1 = dword(d0 + 1), w2 = dword(d0 + 2), w3 = d0 + 3 < 10 ? dword(d0 + 3) : 0u;
                const uint32_t x[3] = {__builtin_amdgcn_alignbit(w1, w0, sh), __builtin_amdgcn_alignbit(w2, w1, sh), __builtin_amdgcn_alignbit(w3, w2, sh)};
                const uint32_t *vb = rv + PQL_OFF_VB / 4 + 3 * (lane >> 1);
                const int e0 = (24 * i) >> 5, bs = (24 * i) & 31;
                const uint32_t bi = __builtin_amdgcn_alignbit(e0 + 1 < 3 ? vb[e0 + 1] : 0u, vb[e0], bs);
                const uint16_t *rad = DEEP ? sVrad : reinterpret_cast<const uint16_t *>(rv + kKeyRadii);
                const uint2 r4 = *reinterpret_cast<const uint2 *>(rad + (lane >> 1) * 16 + 4 * i);
                const uint32_t F[4] = {x[0] & 0xFFFFFu, __builtin_amdgcn_alignbit(x[1], x[0], 20) & 0xFFFFFu, (x[1] >> 8) & 0xFFFFFu,
                                       __builtin_amdgcn_alignbit(x[2], x[1], 28) & 0xFFFFFu};
                h2 ve[4][4]; /* [token][pair of coordinates] */
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const h2 two = as_h2((e & 2) ? r4.y : r4.x);
                    h2 r = (e & 1) ? bcast_hi(two) : bcast_lo(two);
                    if (16 * i + 4 * g + e >= nv) r = h2{(_Float16)0.f, (_Float16)0.f};
                    const h2 rq = r * as_h2(sTBH[2 * ((bi >> (6 * e)) & 63u) + (n & 1)]);
                    const uint2 ta = *reinterpret_cast<const uint2 *>(sTQ + 2 * (F[e] & 1023u));
                    const uint2 tb = *reinterpret_cast<const uint2 *>(sTQ + 2 * (F[e] >> 10));
                    ve[e][0] = bcast_lo(rq) * as_h2(ta.x);
                    ve[e][1] = bcast_lo(rq) * as_h2(ta.y);
                    ve[e][2] = bcast_hi(rq) * as_h2(tb.x);
                    ve[e][3] = bcast_hi(rq) * as_h2(tb.y);
                }
                /* token 16 i + 4 g + e of a group of sixteen goes to place 8 (g & 1) + 4 (g >> 1) + e of it */
                const int chunk = 2 * i + (g & 1), part = g >> 1;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
                    const uint32_t lo = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, ve[1][c >> 1]), __builtin_bit_cast(uint32_t, ve[0][c >> 1]), sel);
                    const uint32_t hi = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, ve[3][c >> 1]), __builtin_bit_cast(uint32_t, ve[2][c >> 1]), sel);
                    const int dim = 8 * n + c;
                    reinterpret_cast<uint2 *>(sV)[2 * (8 * dim + (chunk ^ value_swizzle(dim))) + part] = make_uint2(lo, hi);
                }
            }
            __syncthreads();
            f16x s;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = kProbShift - m_ref;
            const int tok = 32 * slice + r32;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, sK[16 * tok + ((2 * ks + H) ^ (tok & 15))]), q[ks], s, 0, 0, 0);
            if (nv < 64) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * slice + 8 * (e >> 2) + 4 * H + (e & 3) >= nv) s[e] = -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
            if (!have_ref || __ballot(top > kProbShift + kRefSlack) != 0ull) {
                top = fmaxf(top, __shfl_xor(top, 32));
                float delta = top == -INFINITY ? 0.f : top - kProbShift;
                if (have_ref) delta = fmaxf(delta, 0.f);
                const float alpha = have_ref ? __builtin_amdgcn_exp2f(-delta) : 1.f;
                m_ref += delta;
                l_run *= alpha;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] -= delta;
#pragma unroll
                for (int d = 0; d < 4; ++d) acc[d] *= alpha;
                have_ref = true;
            }
            H8 p[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x = __builtin_amdgcn_exp2f(s[e]);
                l_run += x;
                p[e >> 3].v[e & 7] = (_Float16)x;
            }
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int dim = 32 * d + r32, chunk = 2 * (2 * slice + k) + H;
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, sV[8 * dim + (chunk ^ value_swizzle(dim))]), p[k].v, acc[d], 0, 0, 0);
                }
        }
        /* ---- the slices' results joined (through the keys' and values' LDS, a quarter of the coordinates at a time), and stored ---- */
        float l = l_run + __shfl_xor(l_run, 32), m = l > 0.f ? m_ref : -INFINITY;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (slice == 1 && H == 0) {
            sM[rg][r32][0] = m;
            sM[rg][r32][1] = l;
        }
        __syncthreads();
        float scale0 = 0.f, scale1 = 0.f;
        {
            const float m1 = sM[rg][r32][0], l1 = sM[rg][r32][1];
            if (slice == 0) {
                const float mm = fmaxf(m, m1);
                if (mm != -INFINITY) {
                    scale0 = __builtin_amdgcn_exp2f(m - mm);
                    scale1 = __builtin_amdgcn_exp2f(m1 - mm);
                }
                l = l * scale0 + l1 * scale1;
                m = mm;
            }
        }
        float *mine = reinterpret_cast<float *>(sK) + (rg * 64 + lane) * 16;
        const int64_t out_row = piece * kRows + 32 * rg + r32;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if (slice == 1) {
#pragma unroll
                for (int e = 0; e < 16; ++e) mine[e] = acc[d][e];
            }
            __syncthreads();
            if (slice == 0 && real) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float4 o;
                    o.x = acc[d][4 * j] * scale0 + mine[4 * j] * scale1;
                    o.y = acc[d][4 * j + 1] * scale0 + mine[4 * j + 1] * scale1;
                    o.z = acc[d][4 * j + 2] * scale0 + mine[4 * j + 2] * scale1;
                    o.w = acc[d][4 * j + 3] * scale0 + mine[4 * j + 3] * scale1;
                    *reinterpret_cast<float4 *>(a.ws_o + out_row * PQ_D + 32 * d + 8 * j + 4 * H) = o;
                }
            }
            __syncthreads();
        }
        if (slice == 0 && real && H == 0) *reinterpret_cast<float2 *>(a.ws_ml + out_row * 2) = make_float2(m, l);

        gpos += piece_tiles;
        if (gpos >= gend) return;
        tile_lo = 0;
        if (++hk == a.Hkv) {
            hk = 0;
            do {
                if (++blk >= a.n_blocks) return;
                before = a.plan[kPlanHeader + blk];
                block_tiles = a.plan[kPlanHeader + blk + 1] - before;
            } while (block_tiles <= 0);
        }
    }
}

#endif /* PQ_PREFIX_H */
