/*
 * pq_paged.hip -- pq_append_paged: the keys and values of a ragged batch of new tokens to a paged cache, with the
 * position rotation of the keys on the way (Algorithm 1 lines 2 and 4 on k' = Rot(position) k and on v).
 *
 * Codes are settled in double precision: y = k' S with S, the rotation's products and the sums in 64 bits, and the
 * cell comparisons v > tan(t) u of procedure Quant as well (their squares above level 1).  A vector therefore gets
 * the codes of the definition whatever batch it comes in, and equal prefixes have equal pages.
 */
#include <type_traits>

#include "pq_common.h"
#include "pq_encode_tile.h"
#include "pq_paged.h"
#include "pq_polar.h"

namespace {

struct AppendPagedArgs {
    const void *x[2]; /* keys, values */
    uint8_t *codes[2];
    uint16_t *radii[2];
    int64_t ld_token, ld_head;
    int n_heads;
    PagedTable table;
    PagedRows rows;
    RotaryArgs rot;
    const int32_t *positions;
    const PqExact *exact;
    const PqDeviceConsts *consts;
};

/* A row of the batch: its sequence's token, and where that lies in the pool (page -1: nowhere, nothing is written). */
struct PagedPlace {
    int64_t page, position;
    int tau;
};

__device__ __forceinline__ PagedPlace paged_place(const AppendPagedArgs &a, int64_t row, int lane)
{
    PagedPlace p{-1, 0, 0};
    const int b = paged_find(a.rows.n_seq, row, lane, [&](int i) { return (int64_t)a.rows.row_start[i]; });
    if (b < 0 || b >= a.rows.n_seq) return p;
    const int64_t token = (int64_t)a.rows.ctx_len[b] - (a.rows.row_start[b + 1] - row);
    p.page = paged_page(a.table, b, token);
    p.tau = (int)(token & 63);
    p.position = a.positions ? (int64_t)a.positions[row] : token;
    return p;
}

/* procedure Quant inside a quadrant, in 64 bits: boundaries below atan(v / u), u, v >= 0 (or of squares, with squared tangents) */
__device__ __forceinline__ uint32_t quant3_exact(double u, double v, const double (&t)[3])
{
    return (v > t[0] * u ? 1u : 0u) + (v > t[1] * u ? 1u : 0u) + (v > t[2] * u ? 1u : 0u);
}

__device__ __forceinline__ uint32_t quant_upper_exact(double u2, double v2, const double *tan2, int n_bounds)
{
    uint32_t c = 0;
    for (int k = 0; k < n_bounds; ++k) c += v2 > tan2[k] * u2 ? 1u : 0u;
    return c;
}

/* level-1 code of (ya, yb): quadrant from the signs and the cell inside it, or the number of boundaries below its pseudo-angle */
__device__ __forceinline__ uint32_t level1_exact(double ya, double yb, const PqExact &E, bool general)
{
    const uint32_t sa = (uint32_t)(__double2hiint(ya)) >> 31, sb = (uint32_t)(__double2hiint(yb)) >> 31, f = sa ^ sb;
    const double a = fabs(ya), b = fabs(yb);
    if (!general) return (quant3_exact(a, b, E.tan1) ^ (f ? 7u : 0u)) | (sb << 3);
    const double sum = a + b;
    const double p = (double)(2u * sb + f) + (sum > 0.0 ? (f ? a : b) / sum : 0.0);
    uint32_t c = 0;
    for (int k = 0; k < 15; ++k) c += p > E.pseudo1[k] ? 1u : 0u;
    return c;
}

/* one rounding, to nearest even */
__device__ __forceinline__ uint16_t radius_exact(double q)
{
    return __builtin_bit_cast(uint16_t, (_Float16)fmin(sqrt(q), 65504.0));
}

__device__ __forceinline__ double shfl_xor_double(double x, int d)
{
    const int lo = __shfl_xor(__double2loint(x), d), hi = __shfl_xor(__double2hiint(x), d);
    return __hiloint2double(hi, lo);
}

/* One rotated vector, coordinates 2 p and 2 p + 1 in lane p, to slot tau of a page: the recursion of procedure Polar with the codes'
 * comparisons, the nodes above level 1 in the lanes of their first leaf (the others compute the same along). */
template <int KIND>
__device__ __forceinline__ void write_exact(const AppendPagedArgs &a, double ya, double yb, int64_t tile, int tau, int lane)
{
    const PqExact &E = *a.exact;
    const PqDeviceConsts &K = *a.consts;
    const int i = lane & 7, b = lane >> 3;
    const uint32_t code1 = level1_exact(ya, yb, E, K.general != 0);
    const double q1 = ya * ya + yb * yb, q1s = shfl_xor_double(q1, 1);
    const uint32_t c2 = quant3_exact(q1, q1s, E.tan2[0]);
    const double q2 = q1 + q1s, q2s = shfl_xor_double(q2, 2);
    const uint32_t c3 = quant3_exact(q2, q2s, E.tan2[1]);
    const double q3 = q2 + q2s, q3s = shfl_xor_double(q3, 4);
    PqBlockFields f;
    f.c4 = quant3_exact(q3, q3s, E.tan2[2]);
    const double q4 = q3 + q3s;
    f.radius = radius_exact(q4);
    /* level-1 codes at their nibbles; [c2(2h) | c3(h) | c2(2h+1)] of half-block h at bits [8 h, 8 h + 6) */
    uint32_t l1 = code1 << (4 * i);
    uint32_t gw = (i & 1) ? 0u : ((i & 2) ? c2 : ((c2 << 4) | (c3 << 2))) << (2 * (i & 4));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        l1 |= __shfl_xor(l1, d);
        gw |= __shfl_xor(gw, d);
    }
    f.l1 = l1;
    f.g6[0] = gw & 63u;
    f.g6[1] = (gw >> 8) & 63u;
    if (i == 0) {
        pql_put_block<true>(reinterpret_cast<uint32_t *>(a.codes[KIND] + tile * PQL_CODE_BYTES), KIND, tau, b, f);
        if (K.depth != 7) a.radii[KIND][tile * PQL_RADII + pql_pos(KIND, tau, b).radius_half] = f.radius;
    }
    if (K.depth == 7) { /* levels 5, 6, 7 over the block radii, and the vector's word of the radius plane */
        const int b5 = K.up_bits[0], b6 = K.up_bits[1], b7 = K.up_bits[2];
        const double q4s = shfl_xor_double(q4, 8), q5 = q4 + q4s;
        const uint32_t c5 = quant_upper_exact(q4, q4s, E.up_tan2[0], (1 << b5) - 1);
        const double q5s = shfl_xor_double(q5, 16), q6 = q5 + q5s;
        const uint32_t c6 = quant_upper_exact(q5, q5s, E.up_tan2[1], (1 << b6) - 1);
        const double q6s = shfl_xor_double(q6, 32);
        const uint32_t c7 = quant_upper_exact(q6, q6s, E.up_tan2[2], (1 << b7) - 1);
        uint32_t word = 0;
        for (int j = 0; j < 4; ++j) word |= (uint32_t)__shfl((int)c5, 16 * j) << (j * b5);
        for (int j = 0; j < 2; ++j) word |= (uint32_t)__shfl((int)c6, 32 * j) << (4 * b5 + j * b6);
        word |= (uint32_t)__shfl((int)c7, 0) << (4 * b5 + 2 * b6);
        word |= (uint32_t)radius_exact(q6 + q6s) << 16;
        if (lane == 0) reinterpret_cast<uint32_t *>(a.radii[KIND])[tile * (PQ_DEEP_RADII_HALVES / 2) + tau] = word;
    }
}

/* y = x S of up to NV vectors by 512 threads in 64 bits: thread (kq, j) sums a quarter of the products of column j.  S is fetched once for
 * the NV products (128 KB, what bounds a launch of few vectors); the thread's part is requested first, ahead of the vectors. */
struct ExactSlice {
    double m[32];
    __device__ __forceinline__ void load(const double *S, int tid)
    {
        const int kq = tid >> 7, j = tid & 127;
#pragma unroll
        for (int k = 0; k < 32; ++k) m[k] = S[(32 * kq + k) * PQ_D + j];
    }
};

struct ExactLds {
    double x[4][PQ_D];
    double part[4][4][PQ_D];
};

template <int NV>
__device__ __forceinline__ void multiply_exact(const ExactSlice &s, ExactLds &lds, int tid)
{
    const int kq = tid >> 7, j = tid & 127;
    double acc[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) acc[v] = 0.0;
#pragma unroll
    for (int k = 0; k < 32; ++k)
#pragma unroll
        for (int v = 0; v < NV; ++v) acc[v] = fma(lds.x[v][32 * kq + k], s.m[k], acc[v]);
#pragma unroll
    for (int v = 0; v < NV; ++v) lds.part[v][kq][j] = acc[v];
}

__device__ __forceinline__ double rotated_exact(const ExactLds &lds, int r, int c)
{
    return ((lds.part[r][0][c] + lds.part[r][1][c]) + lds.part[r][2][c]) + lds.part[r][3][c];
}

/* coordinate c of a vector, a key's rotated to its position */
template <int XT>
__device__ __forceinline__ double element_exact(const AppendPagedArgs &a, int kind, int64_t off, int64_t position, int c)
{
    auto element = [&](int k) -> double {
        if (XT == PQ_BF16) return (double)__uint_as_float((uint32_t) static_cast<const uint16_t *>(a.x[kind])[off + k] << 16);
        return (double)static_cast<const float *>(a.x[kind])[off + k];
    };
    double x = element(c);
    if (kind == PQ_KEY && c < a.rot.dim) {
        const RotaryPair p = rotary_pair(a.rot, c);
        const float *cs = rotary_row(a.rot, position);
        const double s = (double)cs[(a.rot.dim >> 1) + p.at] * element(p.partner);
        x = x * (double)cs[p.at] + (p.minus ? -s : s);
    }
    return x;
}

/* NV vectors (row, head) of kind KIND by one workgroup of 512 threads, vec0 .. vec0 + NV - 1 as far as they are below n_vec; wavefronts
 * 2 r and 2 r + 1 fetch vector r, the first of them runs its recursion. */
template <int XT, int KIND, int NV>
__device__ __forceinline__ void append_vectors_exact(const AppendPagedArgs &a, int64_t vec0, int64_t n_vec, ExactLds &lds)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    ExactSlice s;
    s.load(a.exact->S, tid);
    const int r = min(wave >> 1, NV - 1); /* a vector beyond the range repeats the last one and is not written */
    const int64_t vec = min(vec0 + r, n_vec - 1), row = vec / a.n_heads;
    const int head = (int)(vec - row * a.n_heads);
    const PagedPlace at = paged_place(a, row, lane);
    if ((wave >> 1) < NV)
        lds.x[r][tid & 127] = element_exact<XT>(a, KIND, row * a.ld_token + (int64_t)head * a.ld_head, at.position, tid & 127);
    __syncthreads();
    multiply_exact<NV>(s, lds, tid);
    __syncthreads();
    if ((wave & 1) == 0 && (wave >> 1) < NV && vec0 + r < n_vec && at.page >= 0)
        write_exact<KIND>(a, rotated_exact(lds, r, 2 * lane), rotated_exact(lds, r, 2 * lane + 1), head * a.table.pool_pages + at.page, at.tau, lane);
}

/* workgroups [0, n_blocks): keys, the rest: values */
template <int XT, int NV>
__global__ __launch_bounds__(512) void pq_append_paged_kernel(AppendPagedArgs a, int64_t n_vec, int n_blocks)
{
    __shared__ ExactLds lds;
    const int blk = (int)blockIdx.x;
    if (blk < n_blocks) append_vectors_exact<XT, PQ_KEY, NV>(a, (int64_t)NV * blk, n_vec, lds);
    else append_vectors_exact<XT, PQ_VALUE, NV>(a, (int64_t)NV * (blk - n_blocks), n_vec, lds);
}

/* ---- whole tiles: chunks of prompts ----
 * A workgroup per tile, as for short inputs of pq_encode_kv: rows are rotated in fp32 and left in LDS as matrix operands, eight threads
 * per vector; wavefront (v, rt) multiplies the 32 vectors of half v into row tile rt of S and runs the recursion of blocks rt and 4 + rt.
 *
 * Codes in doubt.  A rotated coordinate is off by E = 2^-22 |x| at most (derivation and measurement at kDoubt), so the code of a node is
 * certain if its inputs u, v are further from every boundary t than that: |tan t u - v| > (1 + tan t) E at level 1, and above it, where
 * squares are compared, |tan^2 t u^2 - v^2| > 2 sqrt 2 E |(u, v)| sin t (1 + tan t).  The square root is bounded from above by
 * (q / s + s) / 2, q = u^2 + v^2, with s the node's usual radius; doubt is therefore only ever found too often.  Of
 * vectors without a preferred direction 1 in 250 has a code in doubt; the workgroup marks them and, behind its last tile, codes them once more in
 * 64 bits, four at a time. */
constexpr float kDoubt = 0x1p-22f;
constexpr int kChunkItems = 512; /* tiles of one workgroup at most */

struct ChunkItem { /* a tile that the workgroup has written */
    int32_t page, row0, token0, head_kind;
};

/* what the certainty of a vector's codes is measured with */
struct Doubt {
    float e;          /* E */
    float b2, b3, b4; /* the vector's part of the bounds of levels 2, 3, 4 */
};

/* 2 sqrt 2 E (q / s + s) / 2 = c q + b |x|^2 with s = rho |x|, a node's radius among 128 coordinates; and 2^-21 q for the roundings of the
   squares and their sums */
template <int LEVEL>
__device__ __forceinline__ constexpr float doubt_rho() { return LEVEL == 2 ? 0.1767767f : (LEVEL == 3 ? 0.25f : 0.3535534f); }

__device__ __forceinline__ Doubt doubt_of(float norm2)
{
    const float k = 1.4142136f * kDoubt * norm2;
    return Doubt{kDoubt * __builtin_amdgcn_sqrtf(norm2), k * doubt_rho<2>(), k * doubt_rho<3>(), k * doubt_rho<4>()};
}

__device__ __forceinline__ float min3_abs(float a, float b, float c) { return fminf(fminf(fabsf(a), fabsf(b)), fabsf(c)); }

/* distance of a node above level 1 from its nearest boundary, less what it may be off */
template <int LEVEL>
__device__ __forceinline__ float doubt_node(float u, float v, float t1, float t2, float t3, const float (&w)[3], float b)
{
    constexpr float c = 1.4142136f * kDoubt / doubt_rho<LEVEL>() + 0x1p-21f;
    const float d = min3_abs(__builtin_fmaf(t1, u, -v) * w[0], __builtin_fmaf(t2, u, -v) * w[1], __builtin_fmaf(t3, u, -v) * w[2]);
    return __builtin_fmaf(-c, u + v, d) - b;
}

/* polar_quant_block, and whether a code is in doubt.  The weights of level 1 are 1 / (1 + tan t); a coordinate's sign is a boundary as well. */
template <bool GENERAL>
__device__ __forceinline__ BlockCodes quant_block_checked(const f32x16 &y, const Thresholds &th, const Doubt &d, const float (&w)[3][3], const float *pseudo,
                                                          bool &doubt)
{
    PolarState s;
    float near1 = INFINITY, near = INFINITY;
    const float t2b = GENERAL ? th.t2b : 1.f, t3b = GENERAL ? th.t3b : 1.f, t4b = GENERAL ? th.t4b : 1.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        polar_level1_a<GENERAL>(s, y, p, th);
        if (GENERAL) {
            /* pseudo-angle: off by 2 E / (|a| + |b|) and a rounding of numbers below 4 */
            const float a = fabsf(y[2 * p]), b = fabsf(y[2 * p + 1]), sum = a + b;
            const uint32_t ba = __float_as_uint(y[2 * p]), bb = __float_as_uint(y[2 * p + 1]), sb = bb >> 31, f = (ba ^ bb) >> 31;
            const float pa = (float)(2u * sb + f) + (sum > 0.f ? (f ? a : b) * __builtin_amdgcn_rcpf(sum) : 0.f);
            const float gap = fminf(pa - pseudo[s.mq], pseudo[s.mq + 1] - pa);
            near1 = fminf(near1, __builtin_fmaf(gap - 0x1p-20f, sum, -4.f * d.e));
        } else {
            const float a = fabsf(y[2 * p]), b = fabsf(y[2 * p + 1]);
            const float dist = min3_abs(__builtin_fmaf(th.t1a, a, -b) * 0.70710678f, (a - b) * 0.5f, __builtin_fmaf(th.t1c, a, -b) * 0.29289322f);
            near1 = fminf(near1, fminf(dist, fminf(a, b)) - d.e);
        }
        polar_level1_b<GENERAL>(s, y, p);
        polar_upper<GENERAL>(s, p, th);
        if (p & 1) {
            const int n = p >> 1;
            near = fminf(near, doubt_node<2>(s.q1[2 * n], s.q1[2 * n + 1], th.t2a, t2b, th.t2c, w[0], d.b2));
        }
        if ((p & 3) == 3) {
            const int h = p >> 2;
            near = fminf(near, doubt_node<3>(s.q2[2 * h], s.q2[2 * h + 1], th.t3a, t3b, th.t3c, w[1], d.b3));
        }
    }
    near = fminf(near, doubt_node<4>(s.q3[0], s.q3[1], th.t4a, t4b, th.t4c, w[2], d.b4));
    doubt = near1 < 0.f || near < 0.f;
    return s.out;
}

/* the same of a node of levels 5, 6, 7 */
__device__ __forceinline__ bool upper_in_doubt(float u2, float v2, const float *tan2, const float *w, int n_bounds, float e)
{
    const float q = u2 + v2, bound = 2.8284271f * e * __builtin_amdgcn_sqrtf(q) + 0x1p-20f * q;
    bool doubt = false;
#pragma unroll
    for (int k = 0; k < 7; ++k)
        if (k < n_bounds) doubt |= fabsf(__builtin_fmaf(tan2[k], u2, -v2)) * w[k] < bound;
    return doubt;
}

template <int XT, int NTERMS, bool GENERAL, bool DEEP>
__global__ __launch_bounds__(512) void pq_append_chunk_kernel(AppendPagedArgs a, const uint4 *S_terms, int64_t n_items)
{
    typedef Operands<PQ_F32, NTERMS> Op; /* rotated rows are fp32, whatever the input's type */
    constexpr int NXT = Op::x_terms, kIn = NTERMS == 1 ? 1 : 3, kThreads = 512;
    constexpr int kImgDwords = TileImage<DEEP>::dwords, kRadiiHalves = TileImage<DEEP>::radii_halves;
    constexpr int kRows = NXT * 8 * 2 * 64; /* a tile's rows, [term][k-step][half][lane] */
    constexpr int kRaw = XT == PQ_BF16 ? 2 : 4;
    __shared__ union {
        uint4 rows[2 * kRows];
        ExactLds exact;
    } lds;
    __shared__ __align__(16) uint32_t sImg[2][kWaveDwords];
    __shared__ float sQ4[DEEP ? 2 : 1][2][4][DEEP ? 64 : 1];
    __shared__ float sUnscale[2][64], sNorm2[2][64];
    __shared__ PqDeviceConsts::Lut1Cell sLut[GENERAL ? 512 : 1];
    __shared__ float sPseudo[17];
    __shared__ ChunkItem sItem[kChunkItems];
    __shared__ uint32_t sDoubt[kChunkItems][2];
    __shared__ uint32_t sList[256];
    __shared__ int sCount;
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, H = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), v = wave & 1, rt = wave >> 1;
    const int64_t item_end = (int64_t)(blockIdx.x + 1) * n_items / gridDim.x;

    /* items: tile numbers, for each the keys of all heads, then the values: a workgroup has consecutive ones, so a tile's place is looked
       up once for many of them and its rotation table's rows stay near */
    struct Item {
        int64_t index; /* item_end: none */
        int kind, head;
        PagedTile t;
    };
    const int per_tile = 2 * a.n_heads;
    auto find = [&](int64_t index, const Item &from) { /* the first item from `index` on that has something to write */
        Item it = from;
        int64_t u = index / per_tile;
        bool known = from.index < item_end && from.index >= 0 && from.index / per_tile == u;
        while (index < item_end) {
            if (!known) it.t = paged_tile(a.table, a.rows, u, lane);
            if (it.t.page >= 0 && it.t.lo < it.t.hi) break;
            known = false;
            ++u;
            index = u * per_tile;
        }
        it.index = index < item_end ? index : item_end;
        const int rest = (int)(it.index - u * per_tile);
        it.kind = rest >= a.n_heads ? PQ_VALUE : PQ_KEY;
        it.head = rest - (rest >= a.n_heads ? a.n_heads : 0);
        return it;
    };
    /* slots [tau_lo, tau_hi) of the tile are written */
    auto tau_lo = [](const Item &it) { return (int)max(it.t.lo - it.t.row0, (int64_t)0); };
    auto tau_hi = [](const Item &it) { return (int)min(it.t.hi - it.t.row0, (int64_t)64); };

    /* this thread's sixteen coordinates 16 part .. + 15 of vector vec, in two pieces of eight; a slot that is not written gets the first row
       that is */
    const int vec = 8 * wave + (lane & 7), part = lane >> 3, half_dim = a.rot.dim >> 1;
    uint4 raw[kRaw], other[kRaw];
    float4 co[4], si[4];
    auto load_row = [&](const Item &it) {
        const int lo = tau_lo(it), slot = vec >= lo && vec < tau_hi(it) ? vec : lo;
        const int64_t row = it.t.row0 + slot, off = row * a.ld_token + (int64_t)it.head * a.ld_head;
        constexpr int kBytes = XT == PQ_BF16 ? 2 : 4;
        const char *base = static_cast<const char *>(a.x[it.kind]) + off * kBytes;
#pragma unroll
        for (int k = 0; k < kRaw; ++k) raw[k] = reinterpret_cast<const uint4 *>(base + 16 * part * kBytes)[k];
        if (it.kind != PQ_KEY || 16 * part >= a.rot.dim) return;
        const float *cs = rotary_row(a.rot, a.positions ? (int64_t)a.positions[row] : it.t.token0 + slot);
#pragma unroll
        for (int k = 0; k < 2; ++k) { /* dim is a multiple of 16, its half one of 8: a piece lies in one half of the pairs */
            const int c = 16 * part + 8 * k;
            if (a.rot.interleaved) {
                co[2 * k] = *reinterpret_cast<const float4 *>(cs + c / 2);
                si[2 * k] = *reinterpret_cast<const float4 *>(cs + half_dim + c / 2);
            } else {
                const int at = c < half_dim ? c : c - half_dim, partner = c < half_dim ? c + half_dim : c - half_dim;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    co[2 * k + q] = *reinterpret_cast<const float4 *>(cs + at + 4 * q);
                    si[2 * k + q] = *reinterpret_cast<const float4 *>(cs + half_dim + at + 4 * q);
                }
#pragma unroll
                for (int q = 0; q < kRaw / 2; ++q) other[(kRaw / 2) * k + q] = reinterpret_cast<const uint4 *>(base + partner * kBytes)[q];
            }
        }
    };
    auto floats = [](const uint4 *r, float (&f)[8]) {
        if constexpr (XT == PQ_BF16) {
            const uint32_t w[4] = {r[0].x, r[0].y, r[0].z, r[0].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float((e & 1) ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        } else {
            const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
        }
    };
    auto leave_row = [&](int buffer, int kind) {
        float f[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            floats(raw + (kRaw / 2) * k, f[k]);
            const int c = 16 * part + 8 * k;
            if (kind == PQ_KEY && c < a.rot.dim) {
                if (a.rot.interleaved) {
                    const float cc[4] = {co[2 * k].x, co[2 * k].y, co[2 * k].z, co[2 * k].w}, ss[4] = {si[2 * k].x, si[2 * k].y, si[2 * k].z, si[2 * k].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = f[k][2 * e], y = f[k][2 * e + 1];
                        f[k][2 * e] = __builtin_fmaf(x, cc[e], -(y * ss[e]));
                        f[k][2 * e + 1] = __builtin_fmaf(x, ss[e], y * cc[e]);
                    }
                } else {
                    const float cc[8] = {co[2 * k].x, co[2 * k].y, co[2 * k].z, co[2 * k].w, co[2 * k + 1].x, co[2 * k + 1].y, co[2 * k + 1].z, co[2 * k + 1].w};
                    const float ss[8] = {si[2 * k].x, si[2 * k].y, si[2 * k].z, si[2 * k].w, si[2 * k + 1].x, si[2 * k + 1].y, si[2 * k + 1].z, si[2 * k + 1].w};
                    float o[8];
                    floats(other + (kRaw / 2) * k, o);
                    const float sign = c < half_dim ? -1.f : 1.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[k][e] = __builtin_fmaf(f[k][e], cc[e], sign * (o[e] * ss[e]));
                }
            }
        }
        /* k-steps 2 (part & 3), + 1 of lane half part >> 2 */
        uint4 *dst = lds.rows + buffer * kRows + (4 * (part & 3) + (vec >> 5)) * 64 + 32 * (part >> 2) + (vec & 31);
        uint32_t e = 0;
        float up = 1.f;
        if constexpr (Op::half) {
            float m = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[k][i]));
#pragma unroll
            for (int d = 8; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d)); /* the vector's eight parts */
            e = half_exponent(m);
            up = __uint_as_float(e << 23);
            if (part == 0) sUnscale[buffer][vec] = half_unscale<NTERMS>(e);
        }
        float n2 = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = f[k][i] * up;
                n2 = __builtin_fmaf(x, x, n2);
            }
#pragma unroll
        for (int d = 8; d < 64; d <<= 1) n2 += __shfl_xor(n2, d);
        /* |x|^2 as the products give it: with the 2^15 of two terms of S, or the sqrt(d) of entries +-1 */
        if (part == 0) sNorm2[buffer][vec] = n2 * (NTERMS == 2 ? 0x1p30f : (NTERMS == 1 ? 128.f : 1.f));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            BOperand t[NXT];
            if constexpr (Op::half) split_half(f[k], e, t);
            else split_bf16(f[k], t);
#pragma unroll
            for (int x = 0; x < NXT; ++x) dst[(8 * x + k) * 2 * 64] = t[x].q;
        }
    };

    Item it{-1, 0, 0, {}};
    it = find((int64_t)blockIdx.x * n_items / gridDim.x, it);
    if (it.index >= item_end) return;
    load_row(it);
    BOperand sa[8][NTERMS];
    {
        uint4 stage[8][kIn];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int k = 0; k < kIn; ++k) stage[ks][k] = S_terms[((k * 4 + rt) * 8 + ks) * 64 + lane];
        leave_row(0, it.kind);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            if (NTERMS == 2) __builtin_amdgcn_sched_barrier(0); /* one chunk after the other: all at once spills */
            s_operand<PQ_F32, NTERMS>(sa[ks], stage[ks]);
        }
    }
    Thresholds th = load_thresholds(*a.consts, NTERMS == 1 ? PQ_INV_SQRT_D : 1.0f);
    const float base_scale = th.radius_scale;
    UpperTables ut = {};
    if (DEEP) ut = load_upper_tables(*a.consts);
    float w[3][3];
#pragma unroll
    for (int l = 0; l < 3; ++l)
#pragma unroll
        for (int k = 0; k < 3; ++k) w[l][k] = a.exact->doubt[l][k];
    if (GENERAL) {
        sLut[tid] = a.consts->lut1[tid];
        th.lut1 = sLut;
        if (tid < 17) sPseudo[tid] = a.exact->pseudo1_f[tid];
    }
    for (int i = tid; i < 2 * kChunkItems; i += kThreads) (&sDoubt[0][0])[i] = 0;
    const int tau = 32 * v + j;
    Item next = find(it.index + 1, it);
    if (next.index < item_end) load_row(next);
    __syncthreads();
    int n_done = 0;
    /* buffers are used in turn: what a wavefront writes for the tile after the next is behind the next tile's barrier */
    for (int turn = 0, storer = 0;; turn ^= 1, storer = (storer + 1) & 7, ++n_done) {
        const int lo = tau_lo(it), hi = tau_hi(it), kind = it.kind;
        const bool full = lo == 0 && hi == 64, valid = tau >= lo && tau < hi;
        const int64_t plane_tile = (int64_t)it.head * a.table.pool_pages + it.t.page;
        uint8_t *gcodes = a.codes[kind] + plane_tile * PQL_CODE_BYTES;
        uint16_t *gradii = a.radii[kind] + plane_tile * kRadiiHalves;
        uint32_t *img = sImg[turn];
        if (tid == 0) sItem[n_done] = ChunkItem{(int32_t)it.t.page, (int32_t)it.t.row0, (int32_t)it.t.token0, 2 * it.head + kind};
        if (!full) { /* the tile's present contents */
            const uint32_t *gc = reinterpret_cast<const uint32_t *>(gcodes);
            const uint32_t *gr = reinterpret_cast<const uint32_t *>(gradii);
            for (int c = tid; c < PQL_CODE_BYTES / 4; c += kThreads) img[c] = gc[c];
            for (int c = tid; c < kRadiiHalves / 2; c += kThreads) img[PQL_CODE_BYTES / 4 + c] = gr[c];
            __syncthreads();
        }
        if (Op::half) th.radius_scale = base_scale * sUnscale[turn][tau];
        auto mark = [&](bool doubt) {
            const uint64_t m = __ballot(doubt && valid);
            const uint32_t bits = (uint32_t)m | (uint32_t)(m >> 32); /* both halves of the wavefront have the same vectors */
            if (bits && lane == 0) atomicOr(&sDoubt[n_done][v], bits);
        };
        if (32 * v < hi && 32 * v + 32 > lo) {
            f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                BOperand xb[NXT];
#pragma unroll
                for (int x = 0; x < NXT; ++x) xb[x].q = lds.rows[turn * kRows + ((x * 8 + ks) * 2 + v) * 64 + lane];
#pragma unroll
                for (int term = NTERMS - 1; term >= 0; --term)
#pragma unroll
                    for (int x = 0; x < NXT; ++x)
                        if (x + term <= Op::top) acc = multiply<PQ_F32, NTERMS>(sa[ks][term], xb[x], acc);
            }
            bool doubt;
            const BlockCodes bc = quant_block_checked<GENERAL>(acc, th, doubt_of(sNorm2[turn][tau]), w, sPseudo, doubt);
            mark(doubt);
            if (kind == PQ_KEY) {
                if (full) leave_block<PQ_KEY, DEEP>(img, tau, 4 * H + rt, bc);
                else if (valid) emit_block<PQ_KEY, DEEP>(img, tau, 4 * H + rt, bc);
            } else {
                if (full) leave_block<PQ_VALUE, DEEP>(img, tau, 4 * H + rt, bc);
                else if (valid) emit_block<PQ_VALUE, DEEP>(img, tau, 4 * H + rt, bc);
            }
            if (DEEP) sQ4[turn][v][rt][lane] = bc.q4;
        }
        const bool more = next.index < item_end;
        Item after = next;
        if (more) {
            leave_row(turn ^ 1, next.kind);
            after = find(next.index + 1, next);
            if (after.index < item_end) load_row(after);
        }
        __syncthreads();
        if (DEEP && rt == 3 && 32 * v < hi && 32 * v + 32 > lo) {
            float q4[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q4[k] = sQ4[turn][v][k][lane];
            const UpperHalf mine = polar_upper_half(q4, H, ut);
            UpperHalf far;
            far.codes = from_other_half(mine.codes, H);
            far.q6 = __uint_as_float(from_other_half(__float_as_uint(mine.q6), H));
            const uint32_t word = H == 0 ? polar_upper_join(mine, far, th.radius_scale, ut) : polar_upper_join(far, mine, th.radius_scale, ut);
            const float err = kDoubt * __builtin_amdgcn_sqrtf(sNorm2[turn][tau]);
            const PqExact &E = *a.exact;
            mark(upper_in_doubt(q4[0], q4[1], ut.tan2[0], E.up_doubt[0], (1 << ut.b5) - 1, err) ||
                 upper_in_doubt(q4[2], q4[3], ut.tan2[0], E.up_doubt[0], (1 << ut.b5) - 1, err) ||
                 upper_in_doubt(q4[0] + q4[1], q4[2] + q4[3], ut.tan2[1], E.up_doubt[1], (1 << ut.b6) - 1, err) ||
                 upper_in_doubt(H == 0 ? mine.q6 : far.q6, H == 0 ? far.q6 : mine.q6, ut.tan2[2], E.up_doubt[2], (1 << ut.b7) - 1, err));
            if (H == 0 && valid) {
                if (full) reinterpret_cast<uint32_t *>(gradii)[tau] = word;
                else img[PQL_CODE_BYTES / 4 + tau] = word;
            }
        }
        if (full) {
            if (wave == storer) {
                if (kind == PQ_KEY) store_tile<PQ_KEY, DEEP>(img, gcodes, gradii, lane);
                else store_tile<PQ_VALUE, DEEP>(img, gcodes, gradii, lane);
            }
        } else {
            if (DEEP) __syncthreads();
            const uint4 *src = reinterpret_cast<const uint4 *>(img);
            for (int c = tid; c < kImgDwords / 4; c += kThreads) {
                if (c < PQL_CODE_BYTES / 16) reinterpret_cast<uint4 *>(gcodes)[c] = src[c];
                else reinterpret_cast<uint4 *>(gradii)[c - PQL_CODE_BYTES / 16] = src[c];
            }
        }
        if (!more) break;
        it = next;
        next = after;
    }
    ++n_done;

    /* ---- the marked vectors in 64 bits: listed 256 at a time, four per turn ---- */
    __syncthreads(); /* the workgroup's stores of whole tiles come before its updates of single fields */
    for (int skip = 0;; skip += 256) {
        if (wave == 0) {
            int rank = 0; /* of the first marked vector of the 64 tiles */
            for (int base = 0; base < n_done; base += 64) {
                const int i = base + lane;
                uint64_t m = i < n_done ? (uint64_t)sDoubt[i][1] << 32 | sDoubt[i][0] : 0ull;
                int incl = __popcll(m);
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int up = __shfl_up(incl, d);
                    if (lane >= d) incl += up;
                }
                for (int at = rank + incl - __popcll(m) - skip; m; m &= m - 1, ++at)
                    if (at >= 0 && at < 256) sList[at] = (uint32_t)i << 6 | (uint32_t)__builtin_ctzll(m);
                rank += __shfl(incl, 63);
            }
            if (lane == 0) sCount = rank - skip;
        }
        __syncthreads();
        const int count = sCount;
        if (count <= 0) break;
        const int n = min(count, 256), r = wave >> 1;
        for (int k = 0; k < n; k += 4) {
            ExactSlice s;
            s.load(a.exact->S, tid);
            const uint32_t entry = __builtin_amdgcn_readfirstlane(sList[min(k + r, n - 1)]);
            const ChunkItem ci = sItem[entry >> 6];
            const int slot = (int)(entry & 63u), kind = ci.head_kind & 1, head = ci.head_kind >> 1;
            const int64_t row = (int64_t)ci.row0 + slot;
            const int64_t position = a.positions ? (int64_t)a.positions[row] : (int64_t)ci.token0 + slot;
            lds.exact.x[r][tid & 127] = element_exact<XT>(a, kind, row * a.ld_token + (int64_t)head * a.ld_head, position, tid & 127);
            __syncthreads();
            multiply_exact<4>(s, lds.exact, tid);
            __syncthreads();
            if ((wave & 1) == 0 && k + r < n) {
                const double ya = rotated_exact(lds.exact, r, 2 * lane), yb = rotated_exact(lds.exact, r, 2 * lane + 1);
                const int64_t tile = (int64_t)head * a.table.pool_pages + ci.page;
                if (kind == PQ_KEY) write_exact<PQ_KEY>(a, ya, yb, tile, slot, lane);
                else write_exact<PQ_VALUE>(a, ya, yb, tile, slot, lane);
            }
            __syncthreads();
        }
    }
}

template <int XT>
void launch_chunks(const pq_ctx *ctx, const PqDeviceState *ds, const AppendPagedArgs &a, hipStream_t s)
{
    const int64_t n_items = 2 * (int64_t)a.n_heads * paged_tile_numbers(a.rows.n_rows, a.rows.n_seq);
    int64_t blocks = n_items < 256 ? n_items : 256; /* one workgroup per CU */
    if (n_items > blocks * kChunkItems) blocks = (n_items + kChunkItems - 1) / kChunkItems;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(512), 0, s, a, reinterpret_cast<const uint4 *>(ds->S_bf16x3), n_items);
    };
    auto with = [&](auto general, auto deep) {
        constexpr bool G = decltype(general)::value, D = decltype(deep)::value;
        if (ctx->unit_entries) launch(pq_append_chunk_kernel<XT, 1, G, D>);
        else if (ctx->mixing) launch(pq_append_chunk_kernel<XT, 2, G, D>);
        else launch(pq_append_chunk_kernel<XT, 3, G, D>);
    };
    auto with_books = [&](auto deep) {
        if (ctx->general_codebooks) with(std::true_type{}, deep);
        else with(std::false_type{}, deep);
    };
    if (ctx->depth == 7) with_books(std::true_type{});
    else with_books(std::false_type{});
}

} // namespace

extern "C" pq_status pq_append_paged(const pq_ctx *ctx, const void *xk, const void *xv, pq_dtype xt, int64_t n_rows, int n_heads,
                                     int64_t ld_token, int64_t ld_head, const pq_rotary *rotary, const int32_t *positions,
                                     uint8_t *k_codes, uint16_t *k_radii, uint8_t *v_codes, uint16_t *v_radii, int64_t pool_tokens,
                                     const int32_t *pages, int64_t ld_pages, const int32_t *row_start, const int32_t *ctx_len, int n_seq,
                                     void *hip_stream)
{
    if (!ctx) return PQ_EINVAL;
    if (n_rows == 0 || n_seq == 0) return PQ_OK;
    if (!xk || !xv || !k_codes || !k_radii || !v_codes || !v_radii || !pages || !row_start || !ctx_len) return PQ_EINVAL;
    if (xt != PQ_F32 && xt != PQ_BF16) return PQ_EINVAL;
    if (n_rows < 0 || n_seq < 0 || n_heads <= 0 || pool_tokens <= 0 || (pool_tokens & 63) || ld_pages <= 0) return PQ_EINVAL;
    if (ld_token < 0 || ld_head < 0) return PQ_EINVAL;
    if (n_rows > 0x7FFFFFFF / 2 / n_heads || pool_tokens / 64 > 0x7FFFFFFF) return PQ_EUNSUPPORTED;
    const pq_status rs = pq_check_rotary(rotary);
    if (rs != PQ_OK) return rs;
    const int64_t elems16 = xt == PQ_BF16 ? 8 : 4;
    if (!pq_aligned16(xk) || !pq_aligned16(xv) || !pq_aligned16(k_codes) || !pq_aligned16(k_radii) || !pq_aligned16(v_codes) ||
        !pq_aligned16(v_radii) || (ld_token % elems16) || (ld_head % elems16))
        return PQ_EALIGN;
    const PqDeviceState *ds = nullptr;
    const pq_status st = pq_device_state(ctx, &ds);
    if (st != PQ_OK) return st;
    AppendPagedArgs a{{xk, xv}, {k_codes, v_codes}, {k_radii, v_radii}, ld_token, ld_head, n_heads,
                      PagedTable{pages, ld_pages, pool_tokens / 64}, PagedRows{row_start, ctx_len, n_seq, n_rows},
                      pq_rotary_args(rotary), positions, ds->exact, ds->consts};
    const int64_t n_vec = n_rows * n_heads;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (n_rows >= 8 * (int64_t)n_seq) {
        if (xt == PQ_BF16) launch_chunks<PQ_BF16>(ctx, ds, a, s);
        else launch_chunks<PQ_F32>(ctx, ds, a, s);
        PQ_HIP_TRY(hipGetLastError());
        return PQ_OK;
    }
    const int nv = append_vectors_per_block(2 * n_vec);
    const int n_blocks = (int)((n_vec + nv - 1) / nv);
    const dim3 grid(2u * (unsigned)n_blocks), block(512);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, n_vec, n_blocks); };
    if (xt == PQ_BF16) nv == 1 ? launch(pq_append_paged_kernel<PQ_BF16, 1>) : launch(pq_append_paged_kernel<PQ_BF16, 4>);
    else nv == 1 ? launch(pq_append_paged_kernel<PQ_F32, 1>) : launch(pq_append_paged_kernel<PQ_F32, 4>);
    PQ_HIP_TRY(hipGetLastError());
    return PQ_OK;
}
